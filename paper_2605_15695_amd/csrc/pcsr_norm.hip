// Group norm with an activation over rows of channels (see pcsr_train.h).
//
// In a group of m numbers (the rows of a graph times the channels of a group): xhat = (x - mean) rstd, z = xhat w + b, y =
// act(z).  Backward, with dz = dy act'(z): db = sum dz, dw = sum dz xhat, and in each group
// dx = rstd (w dz - (S1 + xhat S2) / m), S1 = sum w dz, S2 = sum w dz xhat.
//
// Bound by memory.  A thread owns 16 bytes of channels of every few rows.  A short graph belongs to a team (a wavefront where graphs are
// a few kilobytes, a workgroup otherwise), which keeps it in registers between its sums and its results: read once.  Long graphs are
// cut into chunks of rows whose sums go to a workspace; a second kernel adds those of a graph, a third reads the rows again,
// the last chunks first, since those are in the memory-side cache.  Which graph is long is found out on the GPU: the host does not know the
// offsets.  A long graph has more rows than a chunk, so that a chunk meets two of them at most, and there are two places for its sums.
// Sums of x and x^2 are held in 64 bits: the variance is a difference, and of numbers far from 0 32 bits would leave little.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "pcsr_num.h"

namespace pcsr {
namespace {

constexpr int kMost = 512;     // threads of a workgroup at most
constexpr int kKept = 8;       // 16-byte pieces a thread keeps of a short graph (of its rows and of their gradients, each)
constexpr int kAhead = 4;      // pieces a thread has on their way
constexpr int kSlots = 2;      // long graphs that meet a chunk
constexpr int kGroupsOf = 8;   // groups that a workgroup adds up over the chunks at a time
constexpr int kPartsMost = 8192; // workgroups to a chunk or graph for all its groups: with 1024 chunks and 2^22 channels fewer than 2^24 of 256 threads

// how a kernel's threads lie over rows and channels
struct Shape {
    int threads, team, slices; // of a workgroup; that work together; of the channels
    int cs, tpr, rpp;          // channels of a slice (whole groups), threads to a row, rows to a pass
    int lanes;                 // that add up one group
};
struct NormArgs {
    int64_t rows, C, graphs, length; // length: of a graph, where there are no offsets
    int groups, cpg;                 // channels of a group
    const void *offsets;
    int wide, ptype, act;
    const void *x;
    int64_t xs;
    const void *w, *b;
    float eps;
    float *mean, *rstd;
    void *y;
    // backward
    const void *dy;
    int64_t dys;
    void *dx;
    float *sums;  // [workgroup][2][C]: of dz and dz xhat; first those of short graphs
    float *means; // [graphs][groups][2]: S1 / m and S2 / m of long graphs
    void *dw, *db;
    // shape of the launch
    Shape few, many; // for short graphs, for chunks
    int64_t longer, chunk; // a graph of more rows is long; rows of a chunk, no more than that
    int shorts, chunks;    // workgroups for short graphs, for chunks
    void *part;            // [chunk][kSlots][groups] pairs of doubles (forward) or floats (backward)
    int32_t *met;          // [chunk]: whether it meets a long graph, for the kernels behind the first
};

__device__ __forceinline__ int64_t begin_of(const NormArgs &a, int64_t s)
{
    if (s <= 0) return 0;
    if (s >= a.graphs) return a.rows;
    if (!a.offsets) return s * a.length;
    const int64_t o = a.wide ? static_cast<const int64_t *>(a.offsets)[s] : (int64_t) static_cast<const int32_t *>(a.offsets)[s];
    return o < 0 ? 0 : (o < a.rows ? o : a.rows);
}
// The last graphs that begin at or before two rows, found by a wavefront: 64 probes at a time and for both, since such a search is bound by
// its round trips (20,000 graphs: three of them).  All lanes ask for the same rows.
__device__ __forceinline__ void graphs_of(const NormArgs &a, const int64_t (&row)[2], int64_t (&graph)[2])
{
    if (!a.offsets) {
        for (int k = 0; k < 2; ++k) graph[k] = a.length > 0 ? row[k] / a.length : 0;
        return;
    }
    const int lane = threadIdx.x & 63;
    int64_t lo[2] = {0, 0}, hi[2] = {a.graphs, a.graphs}; // lo begins there or before
    while (hi[0] - lo[0] > 1 || hi[1] - lo[1] > 1) {
        int64_t step[2], at[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            step[k] = (hi[k] - lo[k] + 63) / 64;
            const int64_t probe = lo[k] + lane * step[k];
            at[k] = begin_of(a, probe < hi[k] ? probe : a.graphs); // (behind the end: all rows, more than any)
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int below = __popcll(__ballot(at[k] <= row[k])); // 1 at least: lane 0's
            lo[k] += (int64_t)(below > 0 ? below - 1 : 0) * step[k];
            hi[k] = hi[k] < lo[k] + step[k] ? hi[k] : lo[k] + step[k];
            if (lo[k] >= hi[k]) lo[k] = hi[k] - 1; // offsets that do not ascend
        }
    }
    graph[0] = lo[0], graph[1] = lo[1];
}

__device__ __forceinline__ float param(const void *p, int type, int64_t c)
{
    return type == PCSR_F32 ? static_cast<const float *>(p)[c]
                            : type == PCSR_BF16 ? (float)static_cast<const bfloat_t *>(p)[c] : (float)static_cast<const half_t *>(p)[c];
}
__device__ __forceinline__ void put_param(void *p, int type, int64_t c, float v)
{
    if (type == PCSR_F32) static_cast<float *>(p)[c] = v;
    else if (type == PCSR_BF16) static_cast<bfloat_t *>(p)[c] = (bfloat_t)v;
    else static_cast<half_t *>(p)[c] = (half_t)v;
}

// 16 bytes of a row as they are
template <typename T> using Raw = typename Pack<T, kPer16<T>>::type;
template <typename T> __device__ __forceinline__ Raw<T> raw(const T *p, int m)
{
    constexpr int N = kPer16<T>;
    if (m >= N) return *reinterpret_cast<const Raw<T> *>(p);
    Raw<T> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < m ? p[i] : (T)0.0f;
    return v;
}

// The share of the normal distribution below z; bell: exp(-z^2 / 2), which the slope of gelu needs as well.  Below zero the share over the
// bell is t P(t) with t = 1 / (1 + 0.346 |z|), P of degree 8 by weighted least squares for the smallest relative error over z from -14 to 0 (3.5e-8;
// in fp32 5 u (1 + z^2), u = 2^-24, of which z^2 is the exponential's), so that gelu keeps its digits far below zero, where it is small.
__device__ __forceinline__ float below_normal(float z, float bell)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.346f, fabsf(z), 1.0f));
    constexpr float P[8] = {0.14520301f, -0.26838204f, 0.18176714f, -0.03471449f, 0.1105235f, 0.11777047f, 0.13838688f, 0.13801986f};
    float h = -0.02857433f;
#pragma unroll
    for (int k = 0; k < 8; ++k) h = __builtin_fmaf(h, t, P[k]);
    const float q = bell * t * h;
    return z < 0.0f ? q : 1.0f - q;
}
template <int N> __device__ __forceinline__ void activate(float (&z)[N], int act)
{
    switch (act) { // the same for the whole launch
    case PCSR_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i]; // a NaN stays one
        break;
    case PCSR_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] * __builtin_amdgcn_rcpf(1.0f + __expf(-z[i]));
        break;
    case PCSR_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] * below_normal(z[i], __expf(-0.5f * z[i] * z[i]));
        break;
    }
}
// z becomes the activation's slope there
template <int N> __device__ __forceinline__ void slopes(float (&z)[N], int act)
{
    switch (act) {
    case PCSR_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] > 0.0f ? 1.0f : z[i] <= 0.0f ? 0.0f : z[i];
        break;
    case PCSR_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-z[i]));
            z[i] = p * (1.0f + z[i] * (1.0f - p));
        }
        break;
    case PCSR_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float bell = __expf(-0.5f * z[i] * z[i]);
            z[i] = below_normal(z[i], bell) + z[i] * 0.39894228f * bell;
        }
        break;
    default:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = 1.0f;
    }
}

// a thread's place in a slice
template <bool WAVE> struct Place {
    int t;           // thread of the team
    int r, unit, m;  // row of a pass, 16-byte piece of the row, channels of it (0: the thread has none)
    int64_t c;       // first channel
    int c0, c1, g0, ng; // the slice's channels and groups
    const Shape &sh;
    __device__ Place(const NormArgs &a, const Shape &of, int per16) : sh(of)
    {
        t = WAVE ? threadIdx.x & 63 : threadIdx.x;
        c0 = blockIdx.y * sh.cs, c1 = c0 + sh.cs < a.C ? c0 + sh.cs : (int)a.C;
        g0 = c0 / a.cpg, ng = (c1 - c0) / a.cpg;
        r = t / sh.tpr, unit = t - r * sh.tpr;
        c = c0 + unit * per16;
        m = r < sh.rpp && c < c1 ? (c1 - (int)c < per16 ? c1 - (int)c : per16) : 0;
    }
};
// what was written to LDS can be read by the team
template <bool WAVE> __device__ __forceinline__ void team_sync()
{
    if (WAVE) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// Sums of a pair over the threads of each group: a thread's pairs (one for each of its channels; ONE: its channels are of one group, and
// there is one pair) go through LDS; `lanes` lanes then add up a group and the first of them calls done(group, pair).
// Pairs of the same place among the threads' channels lie side by side: with a row's channels one behind the other all lanes of a wavefront
// wrote to the same banks.
template <bool ONE, int N> __host__ __device__ __forceinline__ int pairs_of(const Shape &sh) { return sh.rpp * sh.tpr * (ONE ? 1 : N); }
template <bool WAVE, bool ONE, int N, int A, typename V, typename F>
__device__ __forceinline__ void group_sums(const NormArgs &a, const Place<WAVE> &at, V *shared, const V (&s)[A], const V (&q)[A], F done)
{
    const Shape &sh = at.sh;
    const int width = sh.rpp * sh.tpr;
#pragma unroll
    for (int i = 0; i < A; ++i)
        if (i < at.m) {
            V *to = shared + (i * width + at.r * sh.tpr + at.unit) * 2;
            to[0] = s[i], to[1] = q[i];
        }
    team_sync<WAVE>();
    const int per = ONE ? a.cpg / N : a.cpg;
    const float over = __builtin_amdgcn_rcpf((float)per); // e / per below: e is 4096 at most, half a unit outweighs the roundings
    const int lane = at.t & (sh.lanes - 1), mine = at.t / sh.lanes, step = sh.team / sh.lanes;
    for (int g = mine; g - mine < at.ng; g += step) { // all lanes of a wavefront stay
        V s1 = 0, q1 = 0;
        if (g < at.ng) {
            for (int e = lane; e < per * sh.rpp; e += sh.lanes) {
                const int r = (int)(((float)e + 0.5f) * over), c = g * per + e - r * per; // unit, or channel
                const V *from = shared + (ONE ? r * sh.tpr + c : (c % N) * width + r * sh.tpr + c / N) * 2;
                s1 += from[0], q1 += from[1];
            }
        }
        for (int m = 1; m < sh.lanes; m <<= 1) s1 += __shfl_xor(s1, m), q1 += __shfl_xor(q1, m);
        if (g < at.ng && lane == 0) done(g, s1, q1);
    }
    team_sync<WAVE>();
}

// what a thread's channels need: weight, bias; mean and rstd of their groups (ONE: of one, so that 8 channels take 2 registers for 16)
template <int N, bool ONE> struct Channel {
    static constexpr int A = ONE ? 1 : N;
    float mean[A], rstd[A], w[N], b[N];
    int group[A]; // of the slice
    template <bool WAVE> __device__ __forceinline__ void params(const NormArgs &a, const Place<WAVE> &at)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i] = a.w && i < at.m ? param(a.w, a.ptype, at.c + i) : 1.0f;
            b[i] = a.b && i < at.m ? param(a.b, a.ptype, at.c + i) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < A; ++i) group[i] = i < at.m ? ((int)at.c - at.c0 + i) / a.cpg : 0;
    }
    // stat: pairs of the slice's groups
    __device__ __forceinline__ void pairs(const float *stat, float (&first)[A], float (&second)[A]) const
    {
#pragma unroll
        for (int i = 0; i < A; ++i) first[i] = stat[group[i] * 2], second[i] = stat[group[i] * 2 + 1];
    }
    __device__ __forceinline__ void stats(const float *stat) { pairs(stat, mean, rstd); }
    // as a kernel before left them
    template <bool WAVE> __device__ __forceinline__ void stats_of(const NormArgs &a, const Place<WAVE> &at, int64_t graph)
    {
        const int64_t g0 = graph * a.groups + at.g0;
#pragma unroll
        for (int i = 0; i < A; ++i) mean[i] = a.mean[g0 + group[i]], rstd[i] = a.rstd[g0 + group[i]];
    }
};
// mean and 1 / sqrt(variance + eps) from sums in 64 bits; the variance is never below 0, and a NaN stays one
__device__ __forceinline__ void mean_rstd(double s, double q, double over, float eps, float *mean, float *rstd)
{
    const double mu = s * over, var = q * over - mu * mu, v = (var < 0.0 ? 0.0 : var) + (double)eps;
    double r = __builtin_amdgcn_rsq(v); // to half its bits, then twice as many
    r = r * (1.5 - 0.5 * v * r * r);
    r = r * (1.5 - 0.5 * v * r * r);
    *mean = (float)mu;
    *rstd = (float)r;
}

template <typename T, bool ONE>
__device__ __forceinline__ void apply(const NormArgs &a, const Raw<T> &v, const Channel<kPer16<T>, ONE> &ch, T *y, int m)
{
    constexpr int N = kPer16<T>;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = ((float)v[i] - ch.mean[ONE ? 0 : i]) * ch.rstd[ONE ? 0 : i] * ch.w[i] + ch.b[i];
    activate(z, a.act);
    store_upto<T, N>(y, m, z);
}

// f(row, piece of x [, piece of dy]) for the thread's rows of [lo, hi), kAhead pieces on their way
template <typename T, bool WAVE, typename F>
__device__ __forceinline__ void each_row(const NormArgs &a, const Place<WAVE> &at, int64_t lo, int64_t hi, F f)
{
    const T *x = static_cast<const T *>(a.x);
    const int rpp = at.sh.rpp;
    for (int64_t row = lo + at.r; row < hi; row += (int64_t)kAhead * rpp) {
        Raw<T> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (row + k * rpp < hi) v[k] = raw(x + (row + k * rpp) * a.xs + at.c, at.m);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (row + k * rpp < hi) f(row + k * rpp, v[k]);
    }
}
template <typename T, int U = kAhead / 2, bool WAVE, typename F>
__device__ __forceinline__ void each_pair(const NormArgs &a, const Place<WAVE> &at, int64_t lo, int64_t hi, F f)
{
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    const int rpp = at.sh.rpp;
    for (int64_t row = lo + at.r; row < hi; row += (int64_t)U * rpp) {
        Raw<T> v[U], g[U];
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (row + k * rpp < hi) {
                v[k] = raw(x + (row + k * rpp) * a.xs + at.c, at.m);
                g[k] = raw(dy + (row + k * rpp) * a.dys + at.c, at.m);
            }
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (row + k * rpp < hi) f(row + k * rpp, v[k], g[k]);
    }
}

template <typename T, bool ONE, int A> __device__ __forceinline__ void add_squares(const Raw<T> &v, double (&s)[A], double (&q)[A])
{
#pragma unroll
    for (int i = 0; i < kPer16<T>; ++i) {
        const double x = (double)(float)v[i];
        s[ONE ? 0 : i] += x;
        q[ONE ? 0 : i] = fma(x, x, q[ONE ? 0 : i]);
    }
}

// The parts of the graphs that have a chunk's first (slot 0) and last row (slot 1) that lie in the chunk, if those graphs are long; the second only
// if it is another one.
struct ChunkPart {
    int64_t lo, hi, graph, first, end; // rows of the part, its graph and the graph's rows
    bool any;
};
struct ChunkParts {
    ChunkPart part[kSlots];
    __device__ __forceinline__ ChunkPart at(int slot) const { return slot ? part[1] : part[0]; } // (in registers)
    __device__ ChunkParts(const NormArgs &a, int64_t j)
    {
        const int64_t lo = j * a.chunk, hi = lo + a.chunk < a.rows ? lo + a.chunk : a.rows;
        const int64_t row[2] = {lo, hi - 1};
        int64_t graph[2];
        graphs_of(a, row, graph);
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            ChunkPart &p = part[k];
            p.graph = graph[k], p.first = begin_of(a, graph[k]), p.end = begin_of(a, graph[k] + 1);
            p.any = p.end - p.first > a.longer && (k == 0 || p.first > lo);
            p.lo = lo > p.first ? lo : p.first, p.hi = hi < p.end ? hi : p.end;
        }
    }
};

// sums of a chunk
template <typename T, bool ONE> __device__ __forceinline__ void chunk_sums(const NormArgs &a, int64_t j, double *memory)
{
    constexpr int N = kPer16<T>, A = ONE ? 1 : N;
    if ((int)blockIdx.y >= a.many.slices) return;
    const Place<false> at(a, a.many, N);
    const ChunkParts parts(a, j);
    if (threadIdx.x == 0 && blockIdx.y == 0) a.met[j] = parts.part[0].any || parts.part[1].any;
    for (int slot = 0; slot < kSlots; ++slot) {
        const ChunkPart p = parts.at(slot);
        if (!p.any) continue;
        double s[A], q[A];
#pragma unroll
        for (int i = 0; i < A; ++i) s[i] = q[i] = 0.0;
        if (at.m) each_row<T>(a, at, p.lo, p.hi, [&](int64_t, const Raw<T> &v) { add_squares<T, ONE>(v, s, q); });
        double *out = static_cast<double *>(a.part) + ((j * kSlots + slot) * a.groups + at.g0) * 2;
        group_sums<false, ONE, N>(a, at, memory, s, q, [&](int g, double s1, double q1) { out[g * 2] = s1, out[g * 2 + 1] = q1; });
    }
}

// chunks alone, with the registers that those need: 12 us for 16 x 4096 x 320 in bf16 (42 MB; 34 in the kernel below)
template <typename T, bool ONE> __global__ void __launch_bounds__(kMost) norm_chunk_kernel(NormArgs a)
{
    extern __shared__ double memory[];
    chunk_sums<T, ONE>(a, blockIdx.x, memory);
}

// short graphs, one to a team; behind them the chunks of long ones
template <typename T, bool ONE, bool WAVE> __global__ void __launch_bounds__(kMost) norm_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>, A = ONE ? 1 : N;
    extern __shared__ double memory[];
    if ((int)blockIdx.x >= a.shorts) {
        chunk_sums<T, ONE>(a, blockIdx.x - a.shorts, memory);
        return;
    }
    if ((int)blockIdx.y >= a.few.slices) return;
    const int each = pairs_of<ONE, N>(a.few) * 2, team = WAVE ? threadIdx.x >> 6 : 0;
    const Place<WAVE> at(a, a.few, N);
    double *shared = memory + (size_t)team * (each + at.ng);
    float *stat = reinterpret_cast<float *>(shared + each);
    const int64_t graph = WAVE ? (int64_t)blockIdx.x * (blockDim.x >> 6) + team : blockIdx.x;
    const int64_t lo = begin_of(a, graph), hi = begin_of(a, graph + 1);
    if (hi <= lo || hi - lo > a.longer) return;
    const double over = 1.0 / ((double)(hi - lo) * a.cpg);
    auto found = [&](int g, double s1, double q1) {
        float mu, rs;
        mean_rstd(s1, q1, over, a.eps, &mu, &rs);
        stat[g * 2] = mu, stat[g * 2 + 1] = rs;
        a.mean[graph * a.groups + at.g0 + g] = mu, a.rstd[graph * a.groups + at.g0 + g] = rs;
    };
    T *y = static_cast<T *>(a.y);
    const int rpp = a.few.rpp;
    double s[A], q[A];
#pragma unroll
    for (int i = 0; i < A; ++i) s[i] = q[i] = 0.0;
    Channel<N, ONE> ch;
    if (hi - lo <= (int64_t)kKept * rpp) {
        const T *x = static_cast<const T *>(a.x);
        const int mine = at.m && lo + at.r < hi ? ((int)(hi - lo) - at.r + rpp - 1) / rpp : 0; // rows of the thread
        Raw<T> v[kKept];
#pragma unroll
        for (int k = 0; k < kKept; ++k)
            if (k < mine) v[k] = raw(x + (lo + k * rpp + at.r) * a.xs + at.c, at.m);
        ch.params(a, at);
#pragma unroll
        for (int k = 0; k < kKept; ++k)
            if (k < mine) add_squares<T, ONE>(v[k], s, q);
        group_sums<WAVE, ONE, N>(a, at, shared, s, q, found);
        ch.stats(stat);
#pragma unroll
        for (int k = 0; k < kKept; ++k)
            if (k < mine) apply<T, ONE>(a, v[k], ch, y + (lo + k * rpp + at.r) * a.C + at.c, at.m);
        return;
    }
    ch.params(a, at);
    if (at.m) each_row<T>(a, at, lo, hi, [&](int64_t, const Raw<T> &v) { add_squares<T, ONE>(v, s, q); });
    group_sums<WAVE, ONE, N>(a, at, shared, s, q, found);
    if (!at.m) return;
    ch.stats(stat);
    each_row<T>(a, at, lo, hi, [&](int64_t row, const Raw<T> &v) { apply<T, ONE>(a, v, ch, y + row * a.C + at.c, at.m); });
}

// done(graph, its rows, group, pair), the pair added up over the chunks by 32 lanes, for the long graphs that begin in chunk j; without
// offsets for graph j.
template <typename V, typename F> __device__ __forceinline__ void add_chunks(const NormArgs &a, int64_t j, int64_t group, F done)
{
    const V *part = static_cast<const V *>(a.part);
    const int lane = threadIdx.x & 31;
    const auto add = [&](int64_t graph, int64_t first, int64_t end) {
        const int64_t j0 = first / a.chunk, j1 = (end - 1) / a.chunk;
        const int slot = first > j0 * a.chunk; // in its first chunk; 0 in the others
        V s = 0, q = 0;
        if (group < a.groups) {
#pragma unroll 8
            for (int64_t k = j0 + lane; k <= j1; k += 32) {
                const V *in = part + ((k * kSlots + (k == j0 ? slot : 0)) * a.groups + group) * 2;
                s += in[0], q += in[1];
            }
        }
        for (int m = 1; m < 32; m <<= 1) s += __shfl_xor(s, m), q += __shfl_xor(q, m);
        if (lane == 0 && group < a.groups) done(graph, end - first, group, s, q);
    };
    if (!a.offsets) {
        add(j, j * a.length, (j + 1) * a.length);
        return;
    }
    if (!a.met[j]) return;
    const ChunkParts parts(a, j);
    for (int slot = 0; slot < kSlots; ++slot) {
        const ChunkPart p = parts.at(slot);
        if (p.any && p.lo == p.first) add(p.graph, p.first, p.end);
    }
}
__global__ void __launch_bounds__(32 * kGroupsOf) norm_combine_kernel(NormArgs a)
{
    for (int64_t g0 = (int64_t)blockIdx.y * kGroupsOf; g0 < a.groups; g0 += (int64_t)gridDim.y * kGroupsOf)
        add_chunks<double>(a, blockIdx.x, g0 + (threadIdx.x >> 5), [&](int64_t graph, int64_t rows, int64_t g, double s, double q) {
            mean_rstd(s, q, 1.0 / ((double)rows * a.cpg), a.eps, a.mean + graph * a.groups + g, a.rstd + graph * a.groups + g);
        });
}

template <typename T, bool ONE> __global__ void __launch_bounds__(kMost) norm_apply_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>;
    const int64_t j = gridDim.x - 1 - blockIdx.x;
    if (!a.met[j]) return;
    const Place<false> at(a, a.many, N);
    Channel<N, ONE> ch;
    ch.params(a, at);
    T *y = static_cast<T *>(a.y);
    const ChunkParts parts(a, j);
    for (int slot = 0; slot < kSlots; ++slot) {
        const ChunkPart p = parts.at(slot);
        if (!p.any || !at.m) continue;
        ch.stats_of(a, at, p.graph);
        each_row<T>(a, at, p.lo, p.hi, [&](int64_t row, const Raw<T> &v) { apply<T, ONE>(a, v, ch, y + row * a.C + at.c, at.m); });
    }
}

// ---------------------------------------------------------------------------------- backward
// of a piece: its sums for the thread's channels, and for its groups
template <typename T, bool ONE, int N, int A>
__device__ __forceinline__ void add_pair(const NormArgs &a, const Raw<T> &v, const Raw<T> &g, const Channel<N, ONE> &ch, float (&cs)[N], float (&cq)[N],
                                         float (&s)[A], float (&q)[A])
{
    float xhat[N], dz[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        xhat[i] = ((float)v[i] - ch.mean[ONE ? 0 : i]) * ch.rstd[ONE ? 0 : i];
        dz[i] = xhat[i] * ch.w[i] + ch.b[i];
    }
    slopes(dz, a.act);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        dz[i] *= (float)g[i];
        cs[i] += dz[i];
        cq[i] += dz[i] * xhat[i];
        const float d = dz[i] * ch.w[i];
        s[ONE ? 0 : i] += d;
        q[ONE ? 0 : i] += d * xhat[i];
    }
}
// s1, s2: the group's sums over its count, for each channel.  Products are rounded by themselves: in a group of one number the
// difference is 0.
template <typename T, bool ONE, int N, int A>
__device__ __forceinline__ void put_dx(const NormArgs &a, const Raw<T> &v, const Raw<T> &g, const Channel<N, ONE> &ch, const float (&s1)[A],
                                       const float (&s2)[A], T *dx, int m)
{
#pragma clang fp contract(off)
    float o[N], xhat[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        xhat[i] = ((float)v[i] - ch.mean[ONE ? 0 : i]) * ch.rstd[ONE ? 0 : i];
        o[i] = __builtin_fmaf(xhat[i], ch.w[i], ch.b[i]);
    }
    slopes(o, a.act);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = (o[i] * (float)g[i]) * ch.w[i];
        o[i] = ch.rstd[ONE ? 0 : i] * ((d - s1[ONE ? 0 : i]) - xhat[i] * s2[ONE ? 0 : i]);
    }
    store_upto<T, N>(dx, m, o);
}
// a workgroup's sums of each channel, [2][all rows of its teams][cs] of LDS, to row `to` of a.sums
template <bool WAVE, int N>
__device__ __forceinline__ void put_sums(const NormArgs &a, const Place<WAVE> &at, float *col, const float (&cs)[N], const float (&cq)[N], int64_t to)
{
    const Shape &sh = at.sh;
    const int teams = WAVE ? blockDim.x >> 6 : 1, R = sh.rpp * teams, r = at.r + (WAVE ? threadIdx.x >> 6 : 0) * sh.rpp;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < at.m) {
            col[r * sh.cs + (int)at.c - at.c0 + i] = cs[i];
            col[(R + r) * sh.cs + (int)at.c - at.c0 + i] = cq[i];
        }
    __syncthreads();
    const int n = at.c1 - at.c0;
    for (int k = threadIdx.x; k < 2 * n; k += blockDim.x) {
        const int which = k >= n, c = k - which * n;
        float v = 0.0f;
        for (int o = 0; o < R; ++o) v += col[(which * R + o) * sh.cs + c];
        a.sums[(to * 2 + which) * a.C + at.c0 + c] = v;
    }
}

template <typename T, bool ONE> __device__ __forceinline__ void chunk_gradients(const NormArgs &a, int64_t j, float *room)
{
    constexpr int N = kPer16<T>, A = ONE ? 1 : N;
    if ((int)blockIdx.y >= a.many.slices) return;
    const Place<false> at(a, a.many, N);
    const ChunkParts parts(a, j);
    const bool met = parts.part[0].any || parts.part[1].any;
    if (threadIdx.x == 0 && blockIdx.y == 0) a.met[j] = met;
    if (!met) return;
    Channel<N, ONE> ch;
    ch.params(a, at);
    float cs[N], cq[N];
#pragma unroll
    for (int i = 0; i < N; ++i) cs[i] = cq[i] = 0.0f;
    for (int slot = 0; slot < kSlots; ++slot) {
        const ChunkPart p = parts.at(slot);
        if (!p.any) continue;
        float s[A], q[A];
#pragma unroll
        for (int i = 0; i < A; ++i) s[i] = q[i] = 0.0f;
        ch.stats_of(a, at, p.graph);
        if (at.m) each_pair<T>(a, at, p.lo, p.hi, [&](int64_t, const Raw<T> &v, const Raw<T> &g) { add_pair<T, ONE>(a, v, g, ch, cs, cq, s, q); });
        float *out = static_cast<float *>(a.part) + ((j * kSlots + slot) * a.groups + at.g0) * 2;
        if (a.dx) group_sums<false, ONE, N>(a, at, room, s, q, [&](int g, float s1, float q1) { out[g * 2] = s1, out[g * 2 + 1] = q1; });
    }
    if (a.sums) put_sums(a, at, room, cs, cq, a.shorts + j);
}

template <typename T, bool ONE> __global__ void __launch_bounds__(kMost) norm_backward_chunk_kernel(NormArgs a)
{
    extern __shared__ float room[];
    chunk_gradients<T, ONE>(a, blockIdx.x, room);
}

// As the forward kernel; rows are read twice, mostly from the memory-side cache: keeping them took 163 registers, three wavefronts a SIMD for
// four, and 137 us for 113.  20,000 graphs of 24 rows of 64 in fp32, with silu: 103 us, 573 MB (367 read and written once) at 5.6 TB/s.
// The bound of three wavefronts is for 8 channels of several groups in a thread, which would take two with a few registers more.
template <typename T, bool ONE, bool WAVE> __global__ void __launch_bounds__(WAVE ? 256 : kMost, 3) norm_backward_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>, A = ONE ? 1 : N;
    extern __shared__ float room[];
    if ((int)blockIdx.x >= a.shorts) {
        chunk_gradients<T, ONE>(a, blockIdx.x - a.shorts, room);
        return;
    }
    if ((int)blockIdx.y >= a.few.slices) return;
    const int each = pairs_of<ONE, N>(a.few) * 2, teams = WAVE ? blockDim.x >> 6 : 1, team = WAVE ? threadIdx.x >> 6 : 0;
    const Place<WAVE> at(a, a.few, N);
    float *shared = room + (size_t)team * (each + 2 * at.ng), *stat = shared + each;
    Channel<N, ONE> ch;
    ch.params(a, at);
    float cs[N], cq[N]; // of the thread's channels over all its rows
#pragma unroll
    for (int i = 0; i < N; ++i) cs[i] = cq[i] = 0.0f;
    T *dx = static_cast<T *>(a.dx);
    constexpr int U = ONE && sizeof(T) == 4 ? kAhead : kAhead / 2; // where registers allow four wavefronts a SIMD: 103 us for 113 with U = 2
    for (int64_t graph = (int64_t)blockIdx.x * teams + team; graph < a.graphs; graph += (int64_t)a.shorts * teams) {
        const int64_t lo = begin_of(a, graph), hi = begin_of(a, graph + 1);
        if (hi <= lo || hi - lo > a.longer) continue;
        const float over = 1.0f / ((float)(hi - lo) * (float)a.cpg);
        auto found = [&](int g, float s1, float q1) { stat[g * 2] = s1 * over, stat[g * 2 + 1] = q1 * over; };
        float s[A], q[A], s1[A], s2[A];
#pragma unroll
        for (int i = 0; i < A; ++i) s[i] = q[i] = 0.0f;
        ch.stats_of(a, at, graph);
        if (at.m) each_pair<T, U>(a, at, lo, hi, [&](int64_t, const Raw<T> &v, const Raw<T> &g) { add_pair<T, ONE>(a, v, g, ch, cs, cq, s, q); });
        if (!dx) continue; // the same for the whole launch
        group_sums<WAVE, ONE, N>(a, at, shared, s, q, found);
        ch.pairs(stat, s1, s2);
        if (at.m)
            each_pair<T, U>(a, at, lo, hi, [&](int64_t row, const Raw<T> &v, const Raw<T> &g) {
                put_dx<T, ONE, N, A>(a, v, g, ch, s1, s2, dx + row * a.C + at.c, at.m);
            });
        team_sync<WAVE>(); // stat is read
    }
    if (a.sums) put_sums(a, at, room, cs, cq, blockIdx.x);
}

// dx of the chunks
template <typename T, bool ONE> __global__ void __launch_bounds__(kMost) norm_dx_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>, A = ONE ? 1 : N;
    const int64_t j = gridDim.x - 1 - blockIdx.x;
    if (!a.met[j]) return;
    const Place<false> at(a, a.many, N);
    Channel<N, ONE> ch;
    ch.params(a, at);
    T *dx = static_cast<T *>(a.dx);
    const ChunkParts parts(a, j);
    for (int slot = 0; slot < kSlots; ++slot) {
        const ChunkPart p = parts.at(slot);
        if (!p.any || !at.m) continue;
        float s1[A], s2[A];
        ch.stats_of(a, at, p.graph);
        ch.pairs(a.means + (p.graph * a.groups + at.g0) * 2, s1, s2);
        each_pair<T>(a, at, p.lo, p.hi, [&](int64_t row, const Raw<T> &v, const Raw<T> &g) {
            put_dx<T, ONE, N, A>(a, v, g, ch, s1, s2, dx + row * a.C + at.c, at.m);
        });
    }
}

static_assert(2 * 128 == 32 * kGroupsOf, "one workgroup for both");
// dweight and dbias: column sums of [workgroups][2][C], kSumCols columns to a workgroup; behind those the sums of long graphs' groups
constexpr int kSumCols = 2, kSumRows = 128;
__global__ void __launch_bounds__(kSumCols * kSumRows) norm_finish_kernel(NormArgs a, int columns, int parts)
{
    __shared__ float part[kSumRows][kSumCols + 1];
    if ((int)blockIdx.x >= columns) {
        const int k = blockIdx.x - columns;
        for (int64_t g0 = (int64_t)(k % parts) * kGroupsOf; g0 < a.groups; g0 += (int64_t)parts * kGroupsOf)
            add_chunks<float>(a, k / parts, g0 + (threadIdx.x >> 5), [&](int64_t graph, int64_t rows, int64_t g, float s, float q) {
                const float over = 1.0f / ((float)rows * (float)a.cpg);
                a.means[(graph * a.groups + g) * 2] = s * over, a.means[(graph * a.groups + g) * 2 + 1] = q * over;
            });
        return;
    }
    const int lane = threadIdx.x % kSumCols, r = threadIdx.x / kSumCols;
    const int64_t k = (int64_t)blockIdx.x * kSumCols + lane; // column of 2 C
    float v = 0.0f;
    if (k < 2 * a.C) {
#pragma unroll 8
        for (int64_t i = r; i < a.shorts; i += kSumRows) v += a.sums[i * 2 * a.C + k];
#pragma unroll 8
        for (int64_t i = r; i < a.chunks; i += kSumRows) v += a.met[i] ? a.sums[(a.shorts + i) * 2 * a.C + k] : 0.0f;
    }
    part[r][lane] = v;
    __syncthreads();
    for (int half = kSumRows / 2; half; half /= 2) {
        if (r < half) part[r][lane] = v = v + part[r + half][lane];
        __syncthreads();
    }
    if (r == 0 && k < 2 * a.C) {
        void *to = k < a.C ? a.db : a.dw;
        if (to) put_param(to, a.ptype, k < a.C ? k : k - a.C, v);
    }
}

// ---------------------------------------------------------------------------------- launch shapes
// n: numbers of 16 bytes.  A slice is as many whole groups as `team` threads have 16-byte pieces of a row for, or fewer: halved while
// `count` workgroups a slice are too few and a row's piece stays a line.
Shape shape_of(const pcsr_norm_t &a, int n, int threads, int team, int64_t count, int want)
{
    const int cpg = (int)(a.channels / a.groups), size = 16 / n;
    int64_t gs = a.groups;
    while (gs > 1 && (gs * cpg + n - 1) / n > team) gs = (gs + 1) / 2;
    while (gs > 1 && count * ((a.groups + gs - 1) / gs) < want && (gs + 1) / 2 * cpg * size >= 128) gs = (gs + 1) / 2;
    Shape s;
    s.threads = threads, s.team = team;
    s.cs = (int)(gs * cpg), s.slices = (int)((a.groups + gs - 1) / gs);
    s.tpr = (s.cs + n - 1) / n, s.rpp = team / s.tpr;
    s.lanes = 1;
    while (s.lanes < 64 && s.lanes * 2 * gs <= team) s.lanes *= 2;
    return s;
}
struct NormPlan {
    Shape few, many; // for short graphs, for chunks
    int64_t longer, chunk;
    int shorts, chunks;
    bool one, wave;
};
NormPlan norm_plan(const pcsr_norm_t &a, int n, bool backward)
{
    NormPlan q;
    const int cpg = (int)(a.channels / a.groups), size = 16 / n;
    const int64_t mean = a.rows / (a.graphs > 0 ? a.graphs : 1), bytes = mean * a.channels * size, pieces = (cpg + n - 1) / n;
    q.one = cpg % n == 0;
    q.wave = a.graphs >= 512 && pieces <= 64 && bytes <= 64 * 16 * kKept;
    if (q.wave) {
        q.few = shape_of(a, n, 256, 64, a.graphs, 0);
    } else {
        const int t = pieces <= 256 ? 256 : kMost;
        q.few = shape_of(a, n, t, t, a.graphs, 512);
    }
    q.many = shape_of(a, n, q.few.threads, q.few.threads, 1024, 0);
    const int64_t keeps = (int64_t)kKept * q.few.rpp, least = (int64_t)kAhead * q.many.rpp;
    q.chunk = (a.rows + 1023) / 1024;
    if (q.chunk < least) q.chunk = least;
    q.longer = keeps > q.chunk ? keeps : q.chunk;
    const bool known = !a.offsets || a.graphs == 1; // every graph has `mean` rows
    const bool any_short = !known || mean <= q.longer, any_long = known ? mean > q.longer : a.rows > q.longer;
    const int teams = q.few.threads / q.few.team;
    const int64_t groups = (a.graphs + teams - 1) / teams, cap = backward ? 1024 : groups; // backward: as many as run at once
    q.shorts = any_short ? (int)(groups < cap ? groups : cap) : 0;
    q.chunks = any_long ? (int)((a.rows + q.chunk - 1) / q.chunk) : 0;
    return q;
}

bool norm_sizes_ok(const pcsr_norm_t *a)
{
    return a && a->rows >= 0 && a->channels >= 1 && a->groups >= 1 && a->graphs >= 0 && a->channels % a->groups == 0 &&
           (a->graphs > 0 || a->rows == 0) && (a->offsets || a->graphs == 0 || a->rows % a->graphs == 0);
}
int64_t widest(int type) { return kMost * (type == PCSR_F32 ? 4 : 8); } // channels of a group: a thread to each 16 bytes
int norm_check(const pcsr_norm_t *a)
{
    if (!norm_sizes_ok(a) || !(a->eps >= 0.0f) || a->x_stride < a->channels) return PCSR_E_INVALID_ARG;
    if (a->type < PCSR_F32 || a->type > PCSR_F16 || a->param_type < PCSR_F32 || a->param_type > PCSR_F16 || a->act < PCSR_ACT_NONE ||
        a->act > PCSR_ACT_GELU || a->channels / a->groups > widest(a->type))
        return PCSR_E_UNSUPPORTED;
    if (a->rows >= (int64_t(1) << 40) || a->channels > (1 << 22) || a->graphs >= (int64_t(1) << 31) - 65536 || a->x_stride > (int64_t(1) << 31) ||
        a->graphs * a->groups >= int64_t(1) << 40)
        return PCSR_E_TOO_LARGE;
    if (a->rows && (!a->x || !a->mean || !a->rstd)) return PCSR_E_INVALID_ARG;
    return PCSR_OK;
}

NormArgs norm_args(const pcsr_norm_t &a, const NormPlan &q, void *ws)
{
    NormArgs p = {};
    p.rows = a.rows, p.C = a.channels, p.graphs = a.graphs, p.length = a.graphs ? a.rows / a.graphs : 0;
    p.groups = (int)a.groups, p.cpg = (int)(a.channels / a.groups);
    p.offsets = a.graphs == 1 ? nullptr : a.offsets, p.wide = a.wide, p.ptype = a.param_type, p.act = a.act;
    p.x = a.x, p.xs = a.x_stride, p.w = a.weight, p.b = a.bias, p.eps = a.eps, p.mean = a.mean, p.rstd = a.rstd;
    p.longer = q.longer, p.chunk = q.chunk, p.shorts = q.shorts, p.chunks = q.chunks;
    p.few = q.few, p.many = q.many, p.part = ws;
    return p;
}

struct NormSpace { // of the workspace
    int64_t part, means, sums, met, bytes;
    NormSpace(const pcsr_norm_t &a, const NormPlan &q, bool backward)
    {
        auto up = [](int64_t b) { return (b + 15) / 16 * 16; };
        part = 0;
        means = up((int64_t)q.chunks * kSlots * a.groups * 2 * (backward ? 4 : 8));
        sums = means + (backward && q.chunks ? up(a.graphs * a.groups * 8) : 0);
        met = sums + (backward ? ((int64_t)q.shorts + q.chunks) * 2 * a.channels * 4 : 0);
        bytes = met + (int64_t)q.chunks * 4;
    }
};

int parts_of(int groups)
{
    const int parts = (groups + kGroupsOf - 1) / kGroupsOf;
    return parts < kPartsMost ? parts : kPartsMost;
}

unsigned slices(const NormPlan &q)
{
    const int few = q.shorts ? q.few.slices : 0, many = q.chunks ? q.many.slices : 0;
    return (unsigned)(few > many ? few : many);
}

// f<ONE, WAVE>
template <typename F> int for_plan(const NormPlan &q, F f)
{
    if (q.one) return q.wave ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    return q.wave ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

} // namespace
} // namespace pcsr

using namespace pcsr;

extern "C" {

int64_t pcsr_norm_workspace(const pcsr_norm_t *a, int32_t backward)
{
    if (!norm_sizes_ok(a) || a->rows == 0 || a->channels / a->groups > widest(a->type)) return 0;
    return NormSpace(*a, norm_plan(*a, a->type == PCSR_F32 ? 4 : 8, backward), backward).bytes;
}

int pcsr_norm(const pcsr_norm_t *a, void *y, void *ws, void *stream)
{
    const int rc = norm_check(a);
    if (rc != PCSR_OK) return rc;
    if (a->rows == 0) return PCSR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return for_type(a->type, [&](auto t) {
        typedef decltype(t) T;
        const NormPlan q = norm_plan(*a, kPer16<T>, false);
        if (!y || (q.chunks && !ws)) return (int)PCSR_E_INVALID_ARG;
        if (((int64_t)q.shorts + q.chunks) * q.few.threads >= int64_t(1) << 32) return (int)PCSR_E_TOO_LARGE; // threads of a launch
        NormArgs p = norm_args(*a, q, ws);
        p.y = y;
        p.met = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + NormSpace(*a, q, false).met);
        return for_plan(q, [&](auto one, auto wave) {
            constexpr bool ONE = decltype(one)::value, WAVE = decltype(wave)::value;
            const auto lds_of = [&](const Shape &sh, int teams, bool stat) {
                return sizeof(double) * teams * ((size_t)2 * pairs_of<ONE, kPer16<T>>(sh) + (stat ? sh.cs / p.cpg : 0));
            };
            const size_t lds0 = q.shorts ? lds_of(q.few, q.few.threads / q.few.team, true) : 0, lds1 = q.chunks ? lds_of(q.many, 1, false) : 0;
            const size_t lds = lds0 > lds1 ? lds0 : lds1;
            const dim3 grid(q.shorts + q.chunks, slices(q)), block(q.few.threads);
            if (q.shorts) {
                if (!allow_lds(&norm_kernel<T, ONE, WAVE>, lds)) return (int)PCSR_E_HIP;
                hipLaunchKernelGGL((norm_kernel<T, ONE, WAVE>), grid, block, lds, s, p);
            } else {
                if (!allow_lds(&norm_chunk_kernel<T, ONE>, lds)) return (int)PCSR_E_HIP;
                hipLaunchKernelGGL((norm_chunk_kernel<T, ONE>), grid, block, lds, s, p);
            }
            if (q.chunks) {
                hipLaunchKernelGGL(norm_combine_kernel, dim3(p.offsets ? q.chunks : (unsigned)p.graphs, parts_of(p.groups)),
                                   dim3(32 * kGroupsOf), 0, s, p);
                hipLaunchKernelGGL((norm_apply_kernel<T, ONE>), dim3(q.chunks, q.many.slices), dim3(q.many.threads), 0, s, p);
            }
            return launched();
        });
    });
}

int pcsr_norm_backward(const pcsr_norm_t *a, const void *dy, int64_t dy_stride, void *dx, void *dweight, void *dbias, void *ws,
                       void *stream)
{
    const int rc = norm_check(a);
    if (rc != PCSR_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool sums = dweight || dbias;
    if (a->rows && (!dy || dy_stride < a->channels)) return PCSR_E_INVALID_ARG;
    if (dy_stride > (int64_t(1) << 31)) return PCSR_E_TOO_LARGE;
    if (!dx && !sums) return PCSR_OK;
    const int columns = sums ? (int)((2 * a->channels + kSumCols - 1) / kSumCols) : 0;
    return for_type(a->type, [&](auto t) {
        typedef decltype(t) T;
        NormPlan q = {};
        if (a->rows) q = norm_plan(*a, kPer16<T>, true);
        const NormSpace w(*a, q, true);
        if (!ws && a->rows && (q.chunks || sums)) return (int)PCSR_E_INVALID_ARG;
        NormArgs p = norm_args(*a, q, ws);
        char *at = static_cast<char *>(ws);
        p.dy = dy, p.dys = dy_stride, p.dx = dx, p.dw = dweight, p.db = dbias;
        p.sums = sums ? reinterpret_cast<float *>(at + w.sums) : nullptr;
        p.means = reinterpret_cast<float *>(at + w.means);
        p.met = reinterpret_cast<int32_t *>(at + w.met);
        return for_plan(q, [&](auto one, auto wave) {
            constexpr bool ONE = decltype(one)::value, WAVE = decltype(wave)::value;
            const auto lds_of = [&](const Shape &sh, size_t teams, bool stat) {
                const size_t pairs = teams * ((size_t)2 * pairs_of<ONE, kPer16<T>>(sh) + (stat ? 2 * (sh.cs / p.cpg) : 0));
                const size_t col = sums ? teams * 2 * sh.rpp * sh.cs : 0;
                return sizeof(float) * (pairs > col ? pairs : col);
            };
            const size_t lds0 = q.shorts ? lds_of(q.few, q.few.threads / q.few.team, true) : 0, lds1 = q.chunks ? lds_of(q.many, 1, false) : 0;
            const size_t lds = lds0 > lds1 ? lds0 : lds1;
            const dim3 grid(q.shorts + q.chunks, slices(q)), block(q.few.threads);
            if (q.shorts) {
                if (!allow_lds(&norm_backward_kernel<T, ONE, WAVE>, lds)) return (int)PCSR_E_HIP;
                hipLaunchKernelGGL((norm_backward_kernel<T, ONE, WAVE>), grid, block, lds, s, p);
            } else if (q.chunks) {
                if (!allow_lds(&norm_backward_chunk_kernel<T, ONE>, lds)) return (int)PCSR_E_HIP;
                hipLaunchKernelGGL((norm_backward_chunk_kernel<T, ONE>), grid, block, lds, s, p);
            }
            const int parts = parts_of(p.groups), more = dx && q.chunks ? (p.offsets ? q.chunks : (int)p.graphs) * parts : 0;
            if (columns + more) hipLaunchKernelGGL(norm_finish_kernel, dim3(columns + more), dim3(kSumCols * kSumRows), 0, s, p, columns, parts);
            if (dx && q.chunks) hipLaunchKernelGGL((norm_dx_kernel<T, ONE>), dim3(q.chunks, q.many.slices), dim3(q.many.threads), 0, s, p);
            return launched();
        });
    });
}

} // extern "C"
