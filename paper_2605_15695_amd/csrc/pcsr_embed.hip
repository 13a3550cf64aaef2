// Rows of a table by id, scaled, and the table's gradient (see pcsr_train.h).
//
// Forward: out_i = s t_{id_i}.  Bound by memory: each row is read and written once.
//
// Backward: g_v = s sum_{i: id_i = v} d_i.  The ids are sorted (stable, so that equal ids stay in the order they came),
// the sorted positions are cut into tiles of a few dozen, and a group of lanes walks a tile, adding rows of the same id
// in registers.  An id whose run begins and ends in a tile is written there; the pieces of one that crosses tiles go
// to a workspace, and a second kernel adds them in order.  So no atomics decide the order of a sum, a frequent id is shared by as
// many groups as it has tiles, and rows without an id are zeros that are written while the ids are being sorted.
#include <hip/hip_runtime.h>

#include "pcsr_num.h"

namespace pcsr {
namespace {

constexpr int kT = 256;          // threads of a workgroup
constexpr int kAhead = 4;        // rows of the table a group of lanes has on their way
constexpr int kRankMost = 16384; // ids that are sorted by counting the smaller ones
constexpr int kRankT = 1024;     // threads of that
constexpr int kRankKeys = 8192;  // of their keys in LDS at a time
constexpr int kTile = 1024;      // ids a workgroup of a sorting pass holds in registers
constexpr int kTiles = 512;      // workgroups of a sorting pass at most
constexpr int kDigit = 11;       // bits of a sorting pass at most
constexpr int kRounds = kTile / kT;
constexpr int kGradAhead = 8;    // rows of the gradient a group of lanes has on their way

struct EmbedArgs {
    int64_t n, rows, d, stride;
    const void *ids, *src;
    void *dst;
    float scale;
};

// A row's 16-byte piece number `piece`: its first number and how many it has.  The last piece of a row whose width is no multiple of one
// begins early, so that it is whole: two lanes then work out the same numbers.  (Rows of less than a piece have one short one.)
template <int N> __device__ __forceinline__ int64_t piece_at(int64_t piece, int64_t d, int *m)
{
    *m = d < N ? (int)d : N;
    const int64_t c = piece * N;
    return d < N ? 0 : (c <= d - N ? c : d - N);
}

template <typename I> __device__ __forceinline__ int64_t id_at(const void *ids, int64_t i)
{
    return (int64_t) reinterpret_cast<const I *>(ids)[i];
}

// L lanes to a row, 16 bytes each; kAhead rows at a time (8: 19.7 us for 17.0).  32,768 rows of 768 in bf16: 17 us, 5.9 TB/s.  300,000 rows
// of 64 in fp32: 40 us, 3.9 TB/s, bound by rows of 256 bytes at random places of 268 MB (16 us out of a table of 1000 rows).
template <typename T, typename I, int L> __global__ void __launch_bounds__(kT) lookup_kernel(EmbedArgs p)
{
    constexpr int N = kPer16<T>, G = kT / L;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t first = ((int64_t)blockIdx.x * G + group) * kAhead;
    const T *table = static_cast<const T *>(p.src);
    T *out = static_cast<T *>(p.dst);
    int64_t row[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        row[k] = first + k < p.n ? id_at<I>(p.ids, first + k) : -1;
        if (row[k] >= p.rows) row[k] = -1;
    }
    const int64_t pieces = (p.d + N - 1) / N;
    for (int64_t piece = lane; piece < pieces; piece += L) {
        int m;
        const int64_t c = piece_at<N>(piece, p.d, &m);
        float x[kAhead][N];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (row[k] >= 0) {
                load_upto<T, N>(table + row[k] * p.stride + c, m, x[k]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] = 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (row[k] >= 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] *= p.scale;
            }
            if (first + k < p.n) store_upto<T, N>(out + (first + k) * p.d + c, m, x[k]);
        }
    }
}

// ------------------------------------------------------------------ sorted ids
// key of an id: itself, or `rows` for one that stands for no row, which sorts behind all others
template <typename I> __device__ __forceinline__ uint32_t key_of(const void *ids, int64_t i, int64_t rows)
{
    const int64_t id = id_at<I>(ids, i);
    return (uint32_t)(id >= 0 && id < rows ? id : rows);
}

// Zeros, by the workgroups behind those that sort: sorting waits for its round trips and leaves the memory idle, so every launch of it has
// a share.
struct Fill {
    char *p;
    int64_t bytes;
};
__device__ __forceinline__ void fill(const Fill &f, int64_t block, int64_t blocks)
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    const int64_t at = (block * blockDim.x + threadIdx.x) * 16, step = blocks * blockDim.x * 16;
    const int64_t head = (16 - (reinterpret_cast<uintptr_t>(f.p) & 15)) & 15; // up to 16-byte alignment
    const int64_t whole = f.bytes > head ? (f.bytes - head) / 16 * 16 : 0;
    for (int64_t i = at; i < whole; i += step) *reinterpret_cast<u4 *>(f.p + head + i) = u4{0, 0, 0, 0};
    if (block == 0 && threadIdx.x < 16) {
        if (threadIdx.x < head && threadIdx.x < f.bytes) f.p[threadIdx.x] = 0;
        if (head + whole + threadIdx.x < f.bytes) f.p[head + whole + threadIdx.x] = 0;
    }
}

// The place of an id among n sorted ones is the number of smaller ones and of equal ones before it.  64 ids to a
// workgroup, a sixteenth of the keys to each of its wavefronts, read from LDS four at a time.  Bound by the comparisons, 2.7e8 for 16,384 ids
// in one launch, where the passes below would be six: 33 us with 100 MB of zeros beside it, which alone take 16.  Gradients of 100,000 rows of 64
// in fp32, by ranks for by passes: 8192 ids 32 us for 42, 16,384 43 for 43 (60 for 67 of 50,000 rows of 1000 in bf16), 32,768 89 for 46.
template <typename I>
__global__ void __launch_bounds__(kRankT) rank_kernel(int64_t n_ids, int64_t rows, const void *ids, uint32_t *key, uint32_t *pos,
                                                      int sorters, Fill f)
{
    constexpr int W = kRankT / 64;
    __shared__ uint4 keys4[kRankKeys / 4];
    __shared__ int part[W][64];
    if ((int)blockIdx.x >= sorters) {
        fill(f, blockIdx.x - sorters, gridDim.x - sorters);
        return;
    }
    uint32_t *keys = reinterpret_cast<uint32_t *>(keys4);
    const int n = (int)n_ids, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int first = blockIdx.x * 64, i = first + lane; // first: a multiple of 4
    const uint32_t own = key_of<I>(ids, i < n ? i : n - 1, rows);
    int count = 0;
    for (int base = 0; base < n; base += kRankKeys) {
        const int here = n - base < kRankKeys ? n - base : kRankKeys, n4 = (here + 3) / 4;
        __syncthreads(); // the keys before are read
        for (int j = tid; j < n4 * 4; j += kRankT) keys[j] = j < here ? key_of<I>(ids, base + j, rows) : 0xffffffffu;
        __syncthreads();
        const int per = (n4 + W - 1) / W;
        const int hi = (wave + 1) * per < n4 ? (wave + 1) * per : n4, at = (first - base) / 4;
        int j = wave * per;
        const int end0 = hi < at ? hi : at, end1 = hi < at + 16 ? hi : at + 16;
#pragma unroll 8
        for (; j < end0; ++j) {
            const uint4 k = keys4[j];
            count += (k.x <= own) + (k.y <= own) + (k.z <= own) + (k.w <= own);
        }
        for (; j < end1; ++j) {
            const uint4 k = keys4[j];
            const int o = base + j * 4;
            count += (k.x < own || (k.x == own && o < i)) + (k.y < own || (k.y == own && o + 1 < i)) +
                     (k.z < own || (k.z == own && o + 2 < i)) + (k.w < own || (k.w == own && o + 3 < i));
        }
#pragma unroll 8
        for (; j < hi; ++j) {
            const uint4 k = keys4[j];
            count += (k.x < own) + (k.y < own) + (k.z < own) + (k.w < own);
        }
    }
    part[wave][lane] = count;
    __syncthreads();
    if (wave == 0 && i < n) {
        int to = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) to += part[w][lane];
        key[to] = own;
        pos[to] = i;
    }
}

struct SortArgs { // one pass over a digit of the keys
    int64_t n, chunk, rows; // chunk: of the ids to a workgroup, a multiple of kTile
    int shift, bits, tiles;
    const void *ids;        // in the first pass
    const uint32_t *kin, *vin;
    uint32_t *kout, *vout;
    int32_t *counts, *totals; // [tile][digit], [digit]
};
template <typename I, bool FIRST> __device__ __forceinline__ uint32_t sort_key(const SortArgs &p, int64_t t)
{
    return FIRST ? key_of<I>(p.ids, t, p.rows) : p.kin[t];
}

// Sorting passes of kDigit bits: counts of a digit by tile, sums of them over the tiles, places.  300,000 ids below 2^20: two passes, 75 us
// with 268 MB of zeros beside them, which alone take 39: what the launches wait for (counts, then their sums) is not hidden.
template <typename I, bool FIRST> __global__ void __launch_bounds__(kT) count_kernel(SortArgs p, Fill f)
{
    __shared__ int32_t cnt[1 << kDigit];
    if ((int)blockIdx.x >= p.tiles) {
        fill(f, blockIdx.x - p.tiles, gridDim.x - p.tiles);
        return;
    }
    const int bins = 1 << p.bits;
    for (int d = threadIdx.x; d < bins; d += kT) cnt[d] = 0;
    __syncthreads();
    const int64_t t0 = (int64_t)blockIdx.x * p.chunk, t1 = t0 + p.chunk < p.n ? t0 + p.chunk : p.n;
    for (int64_t t = t0 + threadIdx.x; t < t1; t += kT)
        atomicAdd(&cnt[(sort_key<I, FIRST>(p, t) >> p.shift) & (bins - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kT) p.counts[(int64_t)blockIdx.x * bins + d] = cnt[d];
}

__device__ __forceinline__ int32_t wave_upto(int32_t v, int lane)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int32_t o = __shfl_up(v, m);
        if (lane >= m) v += o;
    }
    return v;
}

// Counts of a digit, summed over the tiles before (in place); its total.  64 digits to a workgroup, a stretch of the tiles to each of its wavefronts.
constexpr int kTilesT = 1024;
__global__ void __launch_bounds__(kTilesT) tiles_kernel(int bins, int tiles, int32_t *counts, int32_t *totals, int sorters, Fill f)
{
    if ((int)blockIdx.x >= sorters) {
        fill(f, blockIdx.x - sorters, gridDim.x - sorters);
        return;
    }
    constexpr int W = kTilesT / 64, N = kTiles / W;
    __shared__ int32_t sums[W][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane, per = (tiles + W - 1) / W, t0 = wave * per;
    int32_t v[N], all = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = k < per && t0 + k < tiles && d < bins ? counts[(int64_t)(t0 + k) * bins + d] : 0;
#pragma unroll
    for (int k = 0; k < N; ++k) all += v[k];
    sums[wave][lane] = all;
    __syncthreads();
    int32_t before = 0;
    for (int w = 0; w < wave; ++w) before += sums[w][lane];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (k < per && t0 + k < tiles && d < bins) counts[(int64_t)(t0 + k) * bins + d] = before;
        before += v[k];
    }
    if (wave == W - 1 && d < bins) totals[d] = before;
}

// A wavefront ranks 64 ids at a time by ballots over the digit's bits, in the order they come, and keeps its own
// running counts; the wavefronts' counts are then added up in order.
template <typename I, bool FIRST> __global__ void __launch_bounds__(kT) scatter_kernel(SortArgs p, Fill f)
{
    if ((int)blockIdx.x >= p.tiles) {
        fill(f, blockIdx.x - p.tiles, gridDim.x - p.tiles);
        return;
    }
    constexpr int W = kT / 64, N = (1 << kDigit) / kT;
    __shared__ int32_t cnt[W][1 << kDigit];
    __shared__ int32_t next[1 << kDigit]; // where the next id of a digit goes
    __shared__ int32_t waves[W];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = 1 << p.bits;
    const unsigned long long below = (1ull << lane) - 1;
    { // ids of smaller digits, then those of this one in the tiles before
        int32_t v[N], own = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) own += v[k] = tid * N + k < bins ? p.totals[tid * N + k] : 0;
        const int32_t upto = wave_upto(own, lane);
        if (lane == 63) waves[wave] = upto;
        __syncthreads();
        int32_t ex = upto - own;
        for (int w = 0; w < wave; ++w) ex += waves[w];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int d = tid * N + k;
            if (d < bins) next[d] = ex + p.counts[(int64_t)blockIdx.x * bins + d];
            ex += v[k];
        }
    }
    const int64_t t0 = (int64_t)blockIdx.x * p.chunk, t1 = t0 + p.chunk < p.n ? t0 + p.chunk : p.n;
    for (int64_t sub = t0; sub < t1; sub += kTile) {
        const int64_t at = sub + wave * (kTile / W) + lane;
        uint32_t key[kRounds], val[kRounds];
        int rank[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int64_t t = at + r * 64;
            key[r] = t < t1 ? sort_key<I, FIRST>(p, t) : 0;
            val[r] = FIRST ? (uint32_t)t : (t < t1 ? p.vin[t] : 0);
        }
        for (int d = tid; d < bins; d += kT)
#pragma unroll
            for (int w = 0; w < W; ++w) cnt[w][d] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const bool ok = at + r * 64 < t1;
            const uint32_t digit = (key[r] >> p.shift) & (bins - 1);
            unsigned long long same = __ballot(ok);
            for (int b = 0; b < p.bits; ++b) {
                const bool bit = (digit >> b) & 1;
                const unsigned long long m = __ballot(bit);
                same &= bit ? m : ~m;
            }
            rank[r] = 0;
            if (ok) {
                const int had = cnt[wave][digit];
                rank[r] = had + __popcll(same & below);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); // all have read before the first of them writes
                if ((same & below) == 0) cnt[wave][digit] = had + __popcll(same);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        for (int d = tid; d < bins; d += kT) {
            int32_t to = next[d];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const int32_t c = cnt[w][d];
                cnt[w][d] = to;
                to += c;
            }
            next[d] = to;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (at + r * 64 < t1) {
                const int64_t to = cnt[wave][(key[r] >> p.shift) & (bins - 1)] + rank[r];
                p.kout[to] = key[r];
                p.vout[to] = val[r];
            }
        }
        __syncthreads(); // the counts are read
    }
}

// ------------------------------------------------------------------ sums of rows of the same id
struct GradArgs {
    int64_t n, rows, d, stride;
    int tile; // sorted ids to a group of lanes
    const uint32_t *key, *pos;
    const void *dout;
    void *grad;
    float *part; // [tile][2][d]: of a run that began before the tile; of one that goes on behind it
    float scale;
};

template <typename T, int N> __device__ __forceinline__ void put(const GradArgs &p, uint32_t row, int64_t c, int m, float (&sum)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] *= p.scale;
    store_upto<T, N>(static_cast<T *>(p.grad) + (int64_t)row * p.d + c, m, sum);
}

// A group of lanes to a tile.  300,000 gradients of 64 in fp32: 42 us (77 MB read at random, 3 MB of sums at most to the workspace);
// 16,384 of 1000 in fp16: 14 us, 2.8 TB/s.
template <typename T, int L> __global__ void __launch_bounds__(kT) runs_kernel(GradArgs p)
{
    constexpr int N = kPer16<T>, G = kT / L;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t g = (int64_t)blockIdx.x * G + group, piece = (int64_t)blockIdx.y * L + lane;
    const int64_t t0 = g * p.tile, t1 = t0 + p.tile < p.n ? t0 + p.tile : p.n;
    if (t0 >= p.n || piece * N >= p.d) return;
    int m;
    const int64_t c = piece_at<N>(piece, p.d, &m);
    const T *dout = static_cast<const T *>(p.dout);
    uint32_t cur = p.key[t0];
    bool before = t0 > 0 && p.key[t0 - 1] == cur; // the run of cur began before the tile
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
    float *part = p.part + g * 2 * p.d + c;
    for (int64_t t = t0; t < t1; t += kGradAhead) {
        uint32_t key[kGradAhead], pos[kGradAhead];
        float x[kGradAhead][N];
#pragma unroll
        for (int k = 0; k < kGradAhead; ++k) {
            key[k] = t + k < t1 ? p.key[t + k] : 0xffffffffu;
            pos[k] = t + k < t1 ? p.pos[t + k] : 0;
        }
#pragma unroll
        for (int k = 0; k < kGradAhead; ++k)
            if (key[k] < p.rows) load_upto<T, N>(dout + (int64_t)pos[k] * p.stride + c, m, x[k]);
#pragma unroll
        for (int k = 0; k < kGradAhead; ++k) {
            if (key[k] >= p.rows) continue; // behind the last one that has a row
            if (key[k] != cur) {
                if (before)
                    store_upto<float, N>(part, m, sum);
                else
                    put<T, N>(p, cur, c, m, sum);
                before = false;
                cur = key[k];
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += x[k][i];
        }
    }
    if (cur >= p.rows) return;
    if (before)
        store_upto<float, N>(part, m, sum);
    else if (t1 < p.n && p.key[t1] == cur)
        store_upto<float, N>(part + p.d, m, sum);
    else
        put<T, N>(p, cur, c, m, sum);
}

// The run that goes on behind a tile and did not begin before it: its pieces, in order.  Runs of more than kJoinAlone
// tiles are left to the whole workgroup, whose groups take a stretch of them each.  11 us after the 42 above, 8 after the 14: a chain of
// round trips (key, its run's end, pieces).  kJoinAlone of 8, 32 and 128: gradients of 300,000 ids in 100,000 rows of 32 in bf16, many ids frequent,
// 67, 65 and 74 us; of 20,000 in 1000 rows of 64 27, 28 and 32; all the same where ten rows have all ids.
constexpr int kJoinAlone = 32;
template <typename T, int L> __global__ void __launch_bounds__(kT) join_kernel(GradArgs p)
{
    constexpr int N = kPer16<T>, G = kT / L;
    __shared__ float shared[G][L * N];
    __shared__ int64_t last_of[G];
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t g0 = (int64_t)blockIdx.x * G, g = g0 + group, piece = (int64_t)blockIdx.y * L + lane;
    const bool in = piece * N < p.d;
    int m;
    const int64_t c = piece_at<N>(piece, p.d, &m);
    const int64_t t0 = g * p.tile, t1 = t0 + p.tile;
    int64_t last = 0; // the last tile of the run, 0 = none begins here
    uint32_t row = 0;
    if (t1 < p.n) {
        row = p.key[t1 - 1];
        if (row < p.rows && p.key[t1] == row && !(p.key[t0] == row && t0 > 0 && p.key[t0 - 1] == row)) {
            int64_t lo = t1, hi = p.n; // key[lo] == row
            for (int64_t step = p.tile; lo + step < hi; step *= 2) {
                if (p.key[lo + step] != row) hi = lo + step;
                else lo += step;
            }
            while (hi - lo > 1) {
                const int64_t mid = (lo + hi) >> 1;
                if (p.key[mid] == row) lo = mid;
                else hi = mid;
            }
            last = lo / p.tile;
        }
    }
    auto add = [&](int64_t from, int64_t to, float (&sum)[N]) { // pieces of tiles [from, to)
        for (int64_t h = from; h < to; h += kGradAhead) {
            float x[kGradAhead][N];
#pragma unroll
            for (int k = 0; k < kGradAhead; ++k)
                if (h + k < to) load_upto<float, N>(p.part + (h + k) * 2 * p.d + c, m, x[k]);
#pragma unroll
            for (int k = 0; k < kGradAhead; ++k)
                if (h + k < to)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += x[k][i];
        }
    };
    const bool whole = last - g > kJoinAlone;
    if (last && !whole && in) {
        float sum[N];
        load_upto<float, N>(p.part + (g * 2 + 1) * p.d + c, m, sum);
        add(g + 1, last + 1, sum);
        put<T, N>(p, row, c, m, sum);
    }
    if (lane == 0) last_of[group] = whole ? last : 0;
    __syncthreads();
    for (int k = 0; k < G; ++k) {
        const int64_t end = last_of[k] + 1, begin = g0 + k + 1;
        if (end == 1) continue; // the same for the whole workgroup
        const int64_t per = (end - begin + G - 1) / G, from = begin + group * per, to = from + per < end ? from + per : end;
        float sum[N];
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.0f;
        if (in && group == 0) load_upto<float, N>(p.part + ((g0 + k) * 2 + 1) * p.d + c, m, sum);
        if (in) add(from, to, sum);
#pragma unroll
        for (int i = 0; i < N; ++i) shared[group][lane * N + i] = sum[i];
        __syncthreads();
        if (group == 0 && in) {
            for (int o = 1; o < G; ++o)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += shared[o][lane * N + i];
            put<T, N>(p, p.key[(g0 + k + 1) * p.tile], c, m, sum);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ few ids
// With up to kOwnMost ids no order is made of them: a workgroup owns a stretch of rows, looks through all ids for those of its
// rows (each wavefront through a quarter, in order, into a list in LDS), and a group of lanes adds up a row or writes its zeros.  One launch, bound
// by its round trips and the zeros.  The whole workgroup takes a row, a stretch of its ids to each group, where the table has few, and
// where it has more than kOwnAlone ids; the parts of a sum are added in order.  777 ids of 75 numbers in a table of 1500: 6.2 us; 48 ids
// in 92,826 rows of 204 in bf16: 11 us, 38 MB (21 in slices of 4 lanes, which left fewer of them idle).
// Beside sorting, 100,000 rows of 64 in fp32: 512 ids 10 us for 14, 2048 14 for 19, 4096 20 for 23, 8192 36 for 28; where ids are skewed the two
// meet at 2048 already (19 for 20, 4096: 31 for 24), and an id that has nearly all of 4096 takes 425 for 39, since each group walks the whole list.
// kOwnAlone of 12, 48 and 192, 2000 rows of 64: 777 ids 10.8, 8.9 and 9.0 us, more skewed 28, 28 and 46.
constexpr int kOwnMost = 4096, kOwnAlone = 48;
struct OwnArgs {
    int64_t n, rows, d, stride;
    int own, whole; // rows of a workgroup; whether all of it takes each of them, not a group of lanes
    const void *ids, *dout;
    void *grad;
    float scale;
};
template <typename T, typename I, int L> __global__ void __launch_bounds__(kT) own_kernel(OwnArgs p)
{
    constexpr int N = kPer16<T>, G = kT / L, W = kT / 64;
    extern __shared__ uint32_t list[]; // [W][per]: position and row of ids in the stretch: position << 8 | row
    __shared__ int length[W];
    __shared__ float shared[G][L * N];
    __shared__ int heavy[256], met[256]; // rows: of many ids, of any
    const int tid = threadIdx.x, lane64 = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid % L, group = tid / L, n = (int)p.n, per = (n + W - 1) / W;
    const int64_t r0 = (int64_t)blockIdx.x * p.own, piece = (int64_t)blockIdx.y * L + lane;
    const int rows = p.rows - r0 < p.own ? (int)(p.rows - r0) : p.own;
    const bool in = piece * N < p.d;
    int m;
    const int64_t c = piece_at<N>(piece, p.d, &m);
    const T *dout = static_cast<const T *>(p.dout);
    T *grad = static_cast<T *>(p.grad) + r0 * p.d + c;
    uint32_t *mine = list + wave * per;
    int have = 0;
    const int end = (wave + 1) * per < n ? (wave + 1) * per : n;
    constexpr int U = 8; // ids of a lane on their way
    for (int i = wave * per; i < end; i += U * 64) {
        int64_t row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) row[u] = i + u * 64 + lane64 < end ? id_at<I>(p.ids, i + u * 64 + lane64) - r0 : -1;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool hit = row[u] >= 0 && row[u] < rows;
            const unsigned long long all = __ballot(hit);
            if (hit) mine[have + __popcll(all & ((1ull << lane64) - 1))] = (uint32_t)(i + u * 64 + lane64) << 8 | (uint32_t)row[u];
            have += __popcll(all);
        }
    }
    if (lane64 == 0) length[wave] = have;
    heavy[tid] = met[tid] = 0; // (256 of each, and threads)
    __syncthreads();
    for (int i = lane64; i < have; i += 64) met[mine[i] & 255] = 1;
    __syncthreads();
    // f(position) for the ids of a row in order, `share` of `shares` of them: every lane sees the same
    auto each = [&](int row, int share, int shares, auto f) {
        int seen = 0, total = 0;
        if (shares > 1) {
            for (int w = 0; w < W; ++w)
                for (int i = 0; i < length[w]; i += L) {
                    const bool hit = i + lane < length[w] && (list[w * per + i + lane] & 255) == (uint32_t)row;
                    total += __popcll(__ballot(hit) >> (lane64 - lane) & (L == 64 ? ~0ull : (1ull << L) - 1));
                }
        }
        const int each_of = (total + shares - 1) / shares, lo = share * each_of, hi = shares > 1 ? lo + each_of : INT32_MAX;
        for (int w = 0; w < W; ++w)
            for (int i = 0; i < length[w]; i += L) {
                const bool hit = i + lane < length[w] && (list[w * per + i + lane] & 255) == (uint32_t)row;
                unsigned long long all = __ballot(hit) >> (lane64 - lane) & (L == 64 ? ~0ull : (1ull << L) - 1);
                while (all) {
                    const int k = __ffsll(all) - 1;
                    all &= all - 1;
                    if (seen >= lo && seen < hi) f((int)(list[w * per + i + k] >> 8));
                    ++seen;
                }
            }
        return seen;
    };
    auto sum_row = [&](int row, int share, int shares, float (&sum)[N]) {
        int at[kGradAhead], held = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.0f;
        auto flush = [&] {
            float x[kGradAhead][N];
#pragma unroll
            for (int k = 0; k < kGradAhead; ++k)
                if (k < held && in) load_upto<T, N>(dout + (int64_t)at[k] * p.stride + c, m, x[k]);
#pragma unroll
            for (int k = 0; k < kGradAhead; ++k)
                if (k < held && in)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += x[k][i];
            held = 0;
        };
        each(row, share, shares, [&](int position) {
#pragma unroll
            for (int k = 0; k < kGradAhead; ++k)
                if (k == held) at[k] = position;
            if (++held == kGradAhead) flush();
        });
        flush();
    };
    auto finish = [&](int row, float (&sum)[N]) {
        if (met[row]) { // the others are zeros whatever the scale
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] *= p.scale;
        }
        if (in) store_upto<T, N>(grad + (int64_t)row * p.d, m, sum);
    };
    if (!p.whole) {
        bool any = false; // rows left to the whole workgroup
        for (int row = group; row < rows; row += G) {
            if (!met[row]) { // most rows of a large table: nothing but the store
                float zero[N] = {};
                finish(row, zero);
                continue;
            }
            int count = 0;
            for (int w = 0; w < W; ++w)
                for (int i = 0; i < length[w]; i += L) {
                    const bool hit = i + lane < length[w] && (list[w * per + i + lane] & 255) == (uint32_t)row;
                    count += __popcll(__ballot(hit) >> (lane64 - lane) & (L == 64 ? ~0ull : (1ull << L) - 1));
                }
            if (count > kOwnAlone) {
                if (lane == 0) heavy[row] = 1;
                any = true;
                continue;
            }
            float sum[N];
            sum_row(row, 0, 1, sum);
            finish(row, sum);
        }
        if (!__syncthreads_or(any)) return; // (looking at 256 rows one by one took longer than all the rest)
    }
    for (int row = 0; row < rows; ++row) { // the whole workgroup; the same branch for all of it
        if (!p.whole && !heavy[row]) continue;
        float sum[N];
        sum_row(row, group, G, sum);
#pragma unroll
        for (int i = 0; i < N; ++i) shared[group][lane * N + i] = sum[i];
        __syncthreads();
        if (group == 0) {
            for (int o = 1; o < G; ++o)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += shared[o][lane * N + i];
            finish(row, sum);
        }
        __syncthreads();
    }
}

// lanes to a row of `vectors` of 16 bytes: as many as leave the fewest idle, the most of those; where rows are so few that lanes are
// idle anyhow, enough to have all of a row on its way at once
int lanes_for(int64_t vectors, int64_t rows)
{
    int best = 64;
    if (rows * vectors < (1 << 17)) {
        while (best > 4 && best / 2 >= vectors) best /= 2;
        return best;
    }
    int64_t cost = INT64_MAX;
    for (int l = 64; l >= 4; l /= 2) {
        const int64_t c = (vectors + l - 1) / l * l;
        if (c < cost) cost = c, best = l;
    }
    return best;
}

template <template <int> class F, typename... A> void for_lanes(int lanes, A... a)
{
    switch (lanes) {
    case 4: F<4>::run(a...); break;
    case 8: F<8>::run(a...); break;
    case 16: F<16>::run(a...); break;
    case 32: F<32>::run(a...); break;
    default: F<64>::run(a...); break;
    }
}

int key_bits_of(int64_t rows) // keys 0 to rows
{
    int b = 1;
    while (b < 32 && (int64_t(1) << b) <= rows) ++b;
    return b;
}

struct GradPlan {
    int lanes, tile;
    int64_t slices, groups, chunk;
    int tiles, passes, bits;
};
template <typename V> GradPlan grad_plan(int64_t n, int64_t rows, int64_t d, V per16)
{
    GradPlan q;
    const int64_t vectors = (d + per16 - 1) / per16;
    q.lanes = lanes_for(vectors, n > kOwnMost ? n : 0); // few ids: whole rows, since a slice of them looks through all ids again
    q.slices = (vectors + q.lanes - 1) / q.lanes;
    // enough groups to keep the memory busy, long enough tiles that few runs cross them
    q.tile = 64;
    while (q.tile > 8 && n / q.tile * q.slices * q.lanes < 16384 * 16) q.tile /= 2;
    q.groups = (n + q.tile - 1) / q.tile;
    const int64_t subs = (n + kTile - 1) / kTile, per = (subs + kTiles - 1) / kTiles;
    q.chunk = (per < 1 ? 1 : per) * kTile;
    q.tiles = (int)((n + q.chunk - 1) / q.chunk);
    const int bits = key_bits_of(rows);
    q.passes = (bits + kDigit - 1) / kDigit;
    q.bits = (bits + q.passes - 1) / q.passes;
    return q;
}

int64_t up16(int64_t b) { return (b + 15) / 16 * 16; }

struct GradSpace { // offsets into the workspace
    int64_t key, pos, key2, pos2, counts, totals, part, bytes;
    GradSpace(int64_t n, const GradPlan &q, int64_t d)
    {
        int64_t at = 0;
        auto take = [&](int64_t b) { const int64_t o = at; at += up16(b); return o; };
        key = take(4 * n), pos = take(4 * n);
        const bool passes = n > kRankMost;
        key2 = take(passes && q.passes > 1 ? 4 * n : 0), pos2 = take(passes && q.passes > 1 ? 4 * n : 0);
        counts = take(passes ? (int64_t)q.tiles * (4 << q.bits) : 0), totals = take(passes ? 4 << q.bits : 0);
        part = take(8 * q.groups * d);
        bytes = at;
    }
};

bool sizes_ok(int64_t n, int64_t rows, int64_t d) { return n >= 0 && rows >= 0 && d >= 1; }
bool sizes_fit(int64_t n, int64_t rows, int64_t d)
{
    return n < (int64_t(1) << 31) - kTile && rows < (int64_t(1) << 31) && d <= (int64_t(1) << 23) &&
           (rows == 0 || d <= (int64_t(1) << 60) / rows) && (n == 0 || d <= (int64_t(1) << 60) / n);
}

template <typename T, typename I> struct Lookup {
    template <int L> struct Of {
        static void run(EmbedArgs p, hipStream_t s)
        {
            const int64_t per = (int64_t)(kT / L) * kAhead;
            hipLaunchKernelGGL((lookup_kernel<T, I, L>), dim3((unsigned)((p.n + per - 1) / per)), dim3(kT), 0, s, p);
        }
    };
};
template <typename T> struct Runs {
    template <int L> struct Of {
        static void run(GradArgs p, GradPlan q, hipStream_t s)
        {
            const dim3 grid((unsigned)((q.groups + kT / L - 1) / (kT / L)), (unsigned)q.slices);
            hipLaunchKernelGGL((runs_kernel<T, L>), grid, dim3(kT), 0, s, p);
            if (q.groups > 1) hipLaunchKernelGGL((join_kernel<T, L>), grid, dim3(kT), 0, s, p);
        }
    };
};

template <typename T, typename I> struct Own {
    template <int L> struct Of {
        static void run(OwnArgs p, int64_t slices, hipStream_t s)
        {
            constexpr int G = kT / L;
            // A workgroup to a row below 512 rows: 4000 ids of 64 in 200 rows 9.6 us (26 by groups), 400 9.0 (16.5), 1000 9.0 (10.7), 1500 12.8 (9.2).
            // 1024 workgroups, a look through all ids each, where that leaves every group a row: 4000 ids in 30,000 rows of 64 11 us (21 with 256 of
            // them, 14 with 4096), 50 ids in 90,000 rows of 204 in bf16 10.9 (12.6, 14.8).
            p.whole = p.rows < 512;
            const int64_t per = p.rows / 1024;
            p.own = p.whole ? 1 : (int)(per < G ? G : per > 256 ? 256 : per);
            const dim3 grid((unsigned)((p.rows + p.own - 1) / p.own), (unsigned)slices);
            hipLaunchKernelGGL((own_kernel<T, I, L>), grid, dim3(kT), (size_t)((p.n + kT / 64 - 1) / (kT / 64) * (kT / 64) * 4), s, p);
        }
    };
};

template <typename I> int sort_ids(int64_t n, int64_t rows, const void *ids, const GradPlan &q, const GradSpace &w, char *ws, Fill f,
                                   hipStream_t s)
{
    const auto fillers = [](int64_t bytes, int threads) {
        const int64_t want = ((bytes + 15) / 16 + threads * 4 - 1) / (threads * 4), most = 2048 * kT / threads; // one at least, unless there is nothing
        return (unsigned)(want < most ? want : most);
    };
    uint32_t *key = reinterpret_cast<uint32_t *>(ws + w.key), *pos = reinterpret_cast<uint32_t *>(ws + w.pos);
    if (n <= kRankMost) {
        const int sorters = (int)((n + 63) / 64);
        hipLaunchKernelGGL((rank_kernel<I>), dim3(sorters + fillers(f.bytes, kRankT)), dim3(kRankT), 0, s, n, rows, ids, key, pos,
                           sorters, f);
        return PCSR_OK;
    }
    SortArgs p;
    p.n = n, p.chunk = q.chunk, p.rows = rows, p.bits = q.bits, p.tiles = q.tiles, p.ids = ids;
    p.counts = reinterpret_cast<int32_t *>(ws + w.counts), p.totals = reinterpret_cast<int32_t *>(ws + w.totals);
    uint32_t *key2 = reinterpret_cast<uint32_t *>(ws + w.key2), *pos2 = reinterpret_cast<uint32_t *>(ws + w.pos2);
    // Shares of the zeros, as long as the launches take without (300,000 ids: 6, 4 and 12 us).  Gradients of 20,000 ids in 2^20 rows of 64 in fp32: 85 us
    // (all with the last launch 91, all with the first 100); of 300,000: 125 (125, 137); smaller tables: within 3 %.
    constexpr int kShares[3] = {3, 2, 5};
    int64_t filled = 0;
    int parts = 0;
    const auto share = [&](int which) {
        parts += kShares[which];
        int64_t to = f.bytes * parts / (10 * q.passes) / 4096 * 4096;
        if (parts == 10 * q.passes) to = f.bytes;
        const Fill part = {f.p + filled, to - filled};
        filled = to;
        return part;
    };
    for (int i = 0; i < q.passes; ++i) {
        p.shift = i * q.bits;
        p.kin = p.kout, p.vin = p.vout;
        const bool here = (q.passes - 1 - i) % 2 == 0; // the last pass ends in key and pos
        p.kout = here ? key : key2, p.vout = here ? pos : pos2;
        Fill part = share(0);
        dim3 grid(p.tiles + fillers(part.bytes, kT));
        if (i == 0) {
            p.kin = p.vin = nullptr;
            hipLaunchKernelGGL((count_kernel<I, true>), grid, dim3(kT), 0, s, p, part);
        } else {
            hipLaunchKernelGGL((count_kernel<I, false>), grid, dim3(kT), 0, s, p, part);
        }
        const int bins = 1 << p.bits, sorters = (bins + 63) / 64;
        part = share(1);
        hipLaunchKernelGGL(tiles_kernel, dim3(sorters + fillers(part.bytes, kTilesT)), dim3(kTilesT), 0, s, bins, p.tiles, p.counts, p.totals, sorters, part);
        part = share(2);
        grid = dim3(p.tiles + fillers(part.bytes, kT));
        if (i == 0)
            hipLaunchKernelGGL((scatter_kernel<I, true>), grid, dim3(kT), 0, s, p, part);
        else
            hipLaunchKernelGGL((scatter_kernel<I, false>), grid, dim3(kT), 0, s, p, part);
    }
    return PCSR_OK;
}

template <typename I> __global__ void __launch_bounds__(kT) fill_kernel(Fill f) { fill(f, blockIdx.x, gridDim.x); }

} // namespace
} // namespace pcsr

using namespace pcsr;

extern "C" {

int pcsr_embed(int64_t n, int64_t rows, int64_t d, int32_t type, const void *ids, int32_t wide, const void *table,
               int64_t stride, float scale, void *out, void *stream)
{
    if (!sizes_ok(n, rows, d) || stride < d || (n && (!ids || !out)) || (n && rows && !table)) return PCSR_E_INVALID_ARG;
    if (!sizes_fit(n, rows, d) || stride > (int64_t(1) << 31)) return PCSR_E_TOO_LARGE;
    if (type < PCSR_F32 || type > PCSR_F16) return PCSR_E_UNSUPPORTED;
    if (n == 0) return PCSR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    EmbedArgs p = {n, rows, d, stride, ids, table, out, scale};
    return for_type(type, [&](auto t) {
        typedef decltype(t) T;
        int lanes = lanes_for((d + kPer16<T> - 1) / kPer16<T>, n);
        while (lanes > 4 && (n + kAhead - 1) / kAhead * lanes >= (int64_t(1) << 32) - kT) lanes /= 2; // no launch has 2^32 threads
        if (wide)
            for_lanes<Lookup<T, int64_t>::template Of>(lanes, p, s);
        else
            for_lanes<Lookup<T, int32_t>::template Of>(lanes, p, s);
        return launched();
    });
}

int64_t pcsr_embed_workspace(int64_t n, int64_t rows, int64_t d)
{
    if (!sizes_ok(n, rows, d) || !sizes_fit(n, rows, d) || n <= kOwnMost) return 0;
    int64_t most = 0;
    for (int per16 : {4, 8}) {
        const GradPlan q = grad_plan(n, rows, d, per16);
        const int64_t b = GradSpace(n, q, d).bytes;
        most = b > most ? b : most;
    }
    return most;
}

int pcsr_embed_backward(int64_t n, int64_t rows, int64_t d, int32_t type, const void *ids, int32_t wide, const void *dout,
                        int64_t stride, float scale, void *grad, void *ws, void *stream)
{
    if (!sizes_ok(n, rows, d) || stride < d || (n && (!ids || !dout)) || (n > kOwnMost && !ws) || (rows && !grad)) return PCSR_E_INVALID_ARG;
    if (!sizes_fit(n, rows, d) || stride > (int64_t(1) << 31)) return PCSR_E_TOO_LARGE;
    if (type < PCSR_F32 || type > PCSR_F16) return PCSR_E_UNSUPPORTED;
    if (rows == 0) return PCSR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return for_type(type, [&](auto t) {
        typedef decltype(t) T;
        Fill f = {static_cast<char *>(grad), rows * d * (int64_t)sizeof(T)};
        if (n == 0) {
            hipLaunchKernelGGL(fill_kernel<int>, dim3(2048), dim3(kT), 0, s, f);
            return launched();
        }
        const GradPlan q = grad_plan(n, rows, d, kPer16<T>);
        if (n <= kOwnMost) {
            const OwnArgs o = {n, rows, d, stride, 0, 0, ids, dout, grad, scale};
            if (wide)
                for_lanes<Own<T, int64_t>::template Of>(q.lanes, o, q.slices, s);
            else
                for_lanes<Own<T, int32_t>::template Of>(q.lanes, o, q.slices, s);
            return launched();
        }
        const GradSpace w(n, q, d);
        char *at = static_cast<char *>(ws);
        int rc = wide ? sort_ids<int64_t>(n, rows, ids, q, w, at, f, s) : sort_ids<int32_t>(n, rows, ids, q, w, at, f, s);
        if (rc != PCSR_OK) return rc;
        GradArgs p = {n, rows, d, stride, q.tile, reinterpret_cast<uint32_t *>(at + w.key), reinterpret_cast<uint32_t *>(at + w.pos),
                      dout, grad, reinterpret_cast<float *>(at + w.part), scale};
        for_lanes<Runs<T>::template Of>(q.lanes, p, q, s);
        return launched();
    });
}

} // extern "C"
