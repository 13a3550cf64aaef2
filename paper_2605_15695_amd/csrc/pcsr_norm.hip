// Group norm with an activation over rows of channels (see pcsr_train.h).
//
// In a group of m numbers (the rows of a graph times the channels of a group): xhat = (x - mean) rstd, z = xhat w + b, y =
// act(z).  Backward, with dz = dy act'(z): db = sum dz, dw = sum dz xhat, and in each group
// dx = rstd (w dz - (S1 + xhat S2) / m), S1 = sum w dz, S2 = sum w dz xhat.
//
// Bound by memory.  A thread owns 16 bytes of channels of every few rows.  A short graph belongs to one workgroup, which keeps it in
// registers between its sums and its results: read once.  Long graphs are cut into chunks of rows whose sums go to a
// workspace, and a second kernel adds those of its graph and reads the rows again: twice, the second time from the
// memory-side cache where they fit.  Which graph is short is found out on the GPU: the host does not know the offsets.  A graph is long
// if it has more rows than a chunk, so that a chunk meets two long graphs at most, and there are two places for its sums.
// Sums of x and x^2 are held in 64 bits: the variance is a difference, and of numbers far from 0 32 bits would leave little.
#include <hip/hip_runtime.h>

#include "pcsr_num.h"

namespace pcsr {
namespace {

constexpr int kMost = 512;     // threads of a workgroup at most
constexpr int kKept = 16;      // 16-byte pieces a thread keeps of a short graph
constexpr int kKeptBack = 8;   // of its rows and of their gradients, each
constexpr int kAhead = 4;      // pieces a thread has on their way
constexpr int kSlots = 2;      // long graphs that meet a chunk

struct NormArgs {
    int64_t rows, C, graphs, length; // length: of a graph, where there are no offsets
    int groups, cpg;                 // channels of a group
    const void *offsets;
    int wide, ptype;
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
    float *sums; // [workgroup][2][C]: of dz and dz xhat
    // shape of the launch
    int64_t chunk; // rows of a chunk
    int shorts, chunks; // workgroups for short graphs, for chunks
    int cs, tpr, rpp;   // channels of a slice (whole groups), threads to a row, rows to a pass
    int one;            // a thread's channels are of one group
    int lanes;          // that add up one group
    void *part;         // [chunk][kSlots][groups] pairs of doubles (forward) or floats (backward)
};

__device__ __forceinline__ int64_t begin_of(const NormArgs &a, int64_t s)
{
    if (s <= 0) return 0;
    if (s >= a.graphs) return a.rows;
    if (!a.offsets) return s * a.length;
    const int64_t o = a.wide ? static_cast<const int64_t *>(a.offsets)[s] : (int64_t) static_cast<const int32_t *>(a.offsets)[s];
    return o < 0 ? 0 : (o < a.rows ? o : a.rows);
}
// the last graph that begins at or before a row
__device__ __forceinline__ int64_t graph_of(const NormArgs &a, int64_t row)
{
    if (!a.offsets) return a.length > 0 ? row / a.length : 0;
    int64_t lo = 0, hi = a.graphs;
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (begin_of(a, mid) <= row) lo = mid;
        else hi = mid;
    }
    return lo;
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

template <int ACT> __device__ __forceinline__ float act(float z)
{
    if (ACT == PCSR_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (ACT == PCSR_ACT_SILU) return z / (1.0f + __expf(-z));
    if (ACT == PCSR_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    return z;
}
template <int ACT> __device__ __forceinline__ float slope(float z)
{
    if (ACT == PCSR_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == PCSR_ACT_SILU) {
        const float p = 1.0f / (1.0f + __expf(-z));
        return p * (1.0f + z * (1.0f - p));
    }
    if (ACT == PCSR_ACT_GELU) return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * 0.39894228f * __expf(-0.5f * z * z);
    return 1.0f;
}

// a thread's place in a slice
struct Place {
    int r, unit, m;  // row of a pass, 16-byte piece of the row, channels of it (0: the thread has none)
    int64_t c;       // first channel
    int c0, c1, g0, ng; // the slice's channels and groups
    __device__ Place(const NormArgs &a, int per16)
    {
        c0 = blockIdx.y * a.cs, c1 = c0 + a.cs < a.C ? c0 + a.cs : (int)a.C;
        g0 = c0 / a.cpg, ng = (c1 - c0) / a.cpg;
        r = threadIdx.x / a.tpr, unit = threadIdx.x - r * a.tpr;
        c = c0 + unit * per16;
        m = r < a.rpp && c < c1 ? (c1 - (int)c < per16 ? c1 - (int)c : per16) : 0;
    }
};

// Sums of a pair over the threads of each group: v (N pairs of a thread, one for each of its channels) go through LDS; `lanes`
// lanes then add up a group and the first of them calls done(group, pair).
template <int N, typename V, typename F>
__device__ __forceinline__ void group_sums(const NormArgs &a, const Place &at, V *shared, const V (&s)[N], const V (&q)[N], F done)
{
    const int units = a.one ? a.tpr : a.cs; // of a row
    if (a.one) {
        V s1 = 0, q1 = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < at.m) s1 += s[i], q1 += q[i];
        if (at.m) {
            shared[(at.r * units + at.unit) * 2] = s1;
            shared[(at.r * units + at.unit) * 2 + 1] = q1;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < at.m) {
                shared[(at.r * units + (int)at.c - at.c0 + i) * 2] = s[i];
                shared[(at.r * units + (int)at.c - at.c0 + i) * 2 + 1] = q[i];
            }
    }
    __syncthreads();
    const int per = a.one ? a.cpg / N : a.cpg, lane = threadIdx.x & (a.lanes - 1), step = blockDim.x / a.lanes;
    for (int g = threadIdx.x / a.lanes; g - (int)(threadIdx.x / a.lanes) < at.ng; g += step) { // all lanes of a wavefront stay
        V s1 = 0, q1 = 0;
        if (g < at.ng) {
            for (int r = 0; r < a.rpp; ++r)
                for (int k = lane; k < per; k += a.lanes) {
                    s1 += shared[(r * units + g * per + k) * 2];
                    q1 += shared[(r * units + g * per + k) * 2 + 1];
                }
        }
        for (int m = 1; m < a.lanes; m <<= 1) s1 += __shfl_xor(s1, m), q1 += __shfl_xor(q1, m);
        if (g < at.ng && lane == 0) done(g, s1, q1);
    }
    __syncthreads();
}

// what a thread's channels need: mean, rstd, weight, bias
template <int N> struct Channel {
    float mean[N], rstd[N], w[N], b[N];
    __device__ __forceinline__ void params(const NormArgs &a, const Place &at)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i] = a.w && i < at.m ? param(a.w, a.ptype, at.c + i) : 1.0f;
            b[i] = a.b && i < at.m ? param(a.b, a.ptype, at.c + i) : 0.0f;
        }
    }
    // stat: pairs of the slice's groups
    __device__ __forceinline__ void stats(const NormArgs &a, const Place &at, const float *stat)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int g = i < at.m ? ((int)at.c - at.c0 + i) / a.cpg : 0;
            mean[i] = stat[g * 2], rstd[i] = stat[g * 2 + 1];
        }
    }
};

// variance from sums in 64 bits; never below 0
__device__ __forceinline__ void mean_rstd(double s, double q, double m, float eps, float *mean, float *rstd)
{
    const double mu = s / m, var = q / m - mu * mu;
    *mean = (float)mu;
    *rstd = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)eps)); // a NaN stays one
}

template <typename T, int ACT> __device__ __forceinline__ void apply(const Raw<T> &v, const Channel<kPer16<T>> &ch, T *y, int m)
{
    constexpr int N = kPer16<T>;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = act<ACT>(((float)v[i] - ch.mean[i]) * ch.rstd[i] * ch.w[i] + ch.b[i]);
    store_upto<T, N>(y, m, z);
}

// f(row, piece of x [, piece of dy]) for the thread's rows of [lo, hi), kAhead of them on their way
template <typename T, typename F> __device__ __forceinline__ void each_row(const NormArgs &a, const Place &at, int64_t lo, int64_t hi, F f)
{
    const T *x = static_cast<const T *>(a.x);
    for (int64_t row = lo + at.r; row < hi; row += (int64_t)kAhead * a.rpp) {
        Raw<T> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (row + k * a.rpp < hi) v[k] = raw(x + (row + k * a.rpp) * a.xs + at.c, at.m);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (row + k * a.rpp < hi) f(row + k * a.rpp, v[k]);
    }
}
template <typename T, typename F>
__device__ __forceinline__ void each_pair(const NormArgs &a, const Place &at, int64_t lo, int64_t hi, F f)
{
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    constexpr int U = kAhead / 2;
    for (int64_t row = lo + at.r; row < hi; row += (int64_t)U * a.rpp) {
        Raw<T> v[U], g[U];
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (row + k * a.rpp < hi) {
                v[k] = raw(x + (row + k * a.rpp) * a.xs + at.c, at.m);
                g[k] = raw(dy + (row + k * a.rpp) * a.dys + at.c, at.m);
            }
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (row + k * a.rpp < hi) f(row + k * a.rpp, v[k], g[k]);
    }
}

template <typename T, int N> __device__ __forceinline__ void add_squares(const Raw<T> &v, double (&s)[N], double (&q)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const double x = (double)(float)v[i];
        s[i] += x;
        q[i] = fma(x, x, q[i]);
    }
}

// the part of the graph that has a chunk's first (slot 0) or last row (slot 1) that lies in the chunk, if the graph is long
struct ChunkPart {
    int64_t lo, hi, graph, first, end; // rows of the part, its graph and the graph's rows
    bool any;
    __device__ ChunkPart(const NormArgs &a, int64_t j, int slot)
    {
        lo = j * a.chunk, hi = lo + a.chunk < a.rows ? lo + a.chunk : a.rows;
        graph = graph_of(a, slot ? hi - 1 : lo);
        first = begin_of(a, graph), end = begin_of(a, graph + 1);
        any = end - first > a.chunk && (slot == 0 || first > lo);
        lo = lo > first ? lo : first, hi = hi < end ? hi : end;
    }
};

template <typename T, int ACT> __global__ void __launch_bounds__(kMost) norm_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>;
    extern __shared__ double shared[];
    float *stat = reinterpret_cast<float *>(shared + (size_t)2 * a.rpp * (a.one ? a.tpr : a.cs));
    const Place at(a, N);
    Channel<N> ch;
    double s[N], q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = q[i] = 0.0;
    if ((int64_t)blockIdx.x >= a.shorts) { // sums of a chunk
        const int64_t j = blockIdx.x - a.shorts;
        for (int slot = 0; slot < kSlots; ++slot) {
            const ChunkPart p(a, j, slot);
            if (!p.any) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = q[i] = 0.0;
            if (at.m) each_row<T>(a, at, p.lo, p.hi, [&](int64_t, const Raw<T> &v) { add_squares<T, N>(v, s, q); });
            double *out = static_cast<double *>(a.part) + ((j * kSlots + slot) * a.groups + at.g0) * 2;
            group_sums<N>(a, at, shared, s, q, [&](int g, double s1, double q1) { out[g * 2] = s1, out[g * 2 + 1] = q1; });
        }
        return;
    }
    const int64_t graph = blockIdx.x, lo = begin_of(a, graph), hi = begin_of(a, graph + 1);
    if (hi <= lo || hi - lo > a.chunk) return;
    const double count = (double)(hi - lo) * a.cpg;
    auto found = [&](int g, double s1, double q1) {
        float mu, rs;
        mean_rstd(s1, q1, count, a.eps, &mu, &rs);
        stat[g * 2] = mu, stat[g * 2 + 1] = rs;
        a.mean[graph * a.groups + at.g0 + g] = mu, a.rstd[graph * a.groups + at.g0 + g] = rs;
    };
    T *y = static_cast<T *>(a.y);
    ch.params(a, at);
    if (hi - lo <= (int64_t)kKept * a.rpp) {
        const T *x = static_cast<const T *>(a.x);
        Raw<T> v[kKept];
#pragma unroll
        for (int k = 0; k < kKept; ++k)
            if (lo + k * a.rpp < hi && at.m && lo + k * a.rpp + at.r < hi) v[k] = raw(x + (lo + k * a.rpp + at.r) * a.xs + at.c, at.m);
#pragma unroll
        for (int k = 0; k < kKept; ++k)
            if (lo + k * a.rpp < hi && at.m && lo + k * a.rpp + at.r < hi) add_squares<T, N>(v[k], s, q);
        group_sums<N>(a, at, shared, s, q, found);
        if (!at.m) return;
        ch.stats(a, at, stat);
#pragma unroll
        for (int k = 0; k < kKept; ++k)
            if (lo + k * a.rpp < hi && lo + k * a.rpp + at.r < hi)
                apply<T, ACT>(v[k], ch, y + (lo + k * a.rpp + at.r) * a.C + at.c, at.m);
        return;
    }
    if (at.m) each_row<T>(a, at, lo, hi, [&](int64_t, const Raw<T> &v) { add_squares<T, N>(v, s, q); });
    group_sums<N>(a, at, shared, s, q, found);
    if (!at.m) return;
    ch.stats(a, at, stat);
    each_row<T>(a, at, lo, hi, [&](int64_t row, const Raw<T> &v) { apply<T, ACT>(v, ch, y + row * a.C + at.c, at.m); });
}

// done(group, pair): sums of the chunks of the part's graph
template <typename V, typename F>
__device__ __forceinline__ void graph_sums(const NormArgs &a, const Place &at, const ChunkPart &p, F done)
{
    const int64_t j0 = p.first / a.chunk, j1 = (p.end - 1) / a.chunk;
    const int slot0 = p.first > j0 * a.chunk; // of the first chunk; 0 in the others
    const int lane = threadIdx.x & (a.lanes - 1), step = blockDim.x / a.lanes;
    const V *part = static_cast<const V *>(a.part);
    for (int g = threadIdx.x / a.lanes; g - (int)(threadIdx.x / a.lanes) < at.ng; g += step) {
        V s = 0, q = 0;
        if (g < at.ng) {
#pragma unroll 8
            for (int64_t j = j0 + lane; j <= j1; j += a.lanes) {
                const V *in = part + ((j * kSlots + (j == j0 ? slot0 : 0)) * a.groups + at.g0 + g) * 2;
                s += in[0], q += in[1];
            }
        }
        for (int m = 1; m < a.lanes; m <<= 1) s += __shfl_xor(s, m), q += __shfl_xor(q, m);
        if (g < at.ng && lane == 0) done(g, s, q);
    }
    __syncthreads();
}

template <typename T, int ACT> __global__ void __launch_bounds__(kMost) norm_apply_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>;
    extern __shared__ double shared[];
    float *stat = reinterpret_cast<float *>(shared);
    const Place at(a, N);
    Channel<N> ch;
    ch.params(a, at);
    const int64_t j = blockIdx.x;
    T *y = static_cast<T *>(a.y);
    for (int slot = 0; slot < kSlots; ++slot) {
        const ChunkPart p(a, j, slot);
        if (!p.any) continue;
        const double count = (double)(p.end - p.first) * a.cpg;
        graph_sums<double>(a, at, p, [&](int g, double s, double q) {
            float mu, rs;
            mean_rstd(s, q, count, a.eps, &mu, &rs);
            stat[g * 2] = mu, stat[g * 2 + 1] = rs;
            if (p.lo == p.first) a.mean[p.graph * a.groups + at.g0 + g] = mu, a.rstd[p.graph * a.groups + at.g0 + g] = rs;
        });
        if (at.m) {
            ch.stats(a, at, stat);
            each_row<T>(a, at, p.lo, p.hi, [&](int64_t row, const Raw<T> &v) { apply<T, ACT>(v, ch, y + row * a.C + at.c, at.m); });
        }
        __syncthreads(); // stat is read
    }
}

// ---------------------------------------------------------------------------------- backward
template <typename T, int ACT, int N>
__device__ __forceinline__ void add_pair(const Raw<T> &v, const Raw<T> &g, const Channel<N> &ch, float (&s)[N], float (&q)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float xhat = ((float)v[i] - ch.mean[i]) * ch.rstd[i];
        const float dz = (float)g[i] * slope<ACT>(xhat * ch.w[i] + ch.b[i]);
        s[i] += dz;
        q[i] += dz * xhat;
    }
}
// s1, s2: the group's sums over its count, for each channel.  Products are rounded by themselves: in a group of one number the
// difference is 0.
template <typename T, int ACT, int N>
__device__ __forceinline__ void put_dx(const Raw<T> &v, const Raw<T> &g, const Channel<N> &ch, const float (&s1)[N], const float (&s2)[N], T *dx,
                                       int m)
{
#pragma clang fp contract(off)
    float o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float xhat = ((float)v[i] - ch.mean[i]) * ch.rstd[i];
        const float dz = (float)g[i] * slope<ACT>(xhat * ch.w[i] + ch.b[i]);
        o[i] = ch.rstd[i] * ((dz * ch.w[i] - s1[i]) - xhat * s2[i]);
    }
    store_upto<T, N>(dx, m, o);
}
template <int N> __device__ __forceinline__ void group_means(const NormArgs &a, const Place &at, const float *stat, float (&s1)[N], float (&s2)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int g = i < at.m ? ((int)at.c - at.c0 + i) / a.cpg : 0;
        s1[i] = stat[g * 2], s2[i] = stat[g * 2 + 1];
    }
}
// mean and rstd as the forward call left them
template <int N> __device__ __forceinline__ void saved_stats(const NormArgs &a, const Place &at, int64_t graph, Channel<N> &ch)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t g = graph * a.groups + at.g0 + (i < at.m ? ((int)at.c - at.c0 + i) / a.cpg : 0);
        ch.mean[i] = a.mean[g], ch.rstd[i] = a.rstd[g];
    }
}

template <typename T, int ACT> __global__ void __launch_bounds__(kMost) norm_backward_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>;
    extern __shared__ double shared_[];
    float *shared = reinterpret_cast<float *>(shared_);
    const int units = a.one ? a.tpr : a.cs;
    float *stat = shared + (size_t)2 * a.rpp * units;
    const Place at(a, N);
    Channel<N> ch;
    ch.params(a, at);
    float all_s[N], all_q[N]; // of the thread's channels over all its rows
#pragma unroll
    for (int i = 0; i < N; ++i) all_s[i] = all_q[i] = 0.0f;
    T *dx = static_cast<T *>(a.dx);
    auto group_part = [&](float (&s)[N], float (&q)[N], auto done) {
        float ws[N], wq[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            all_s[i] += s[i], all_q[i] += q[i];
            ws[i] = s[i] * ch.w[i], wq[i] = q[i] * ch.w[i];
        }
        if (a.dx) group_sums<N>(a, at, shared, ws, wq, done);
    };
    if ((int64_t)blockIdx.x >= a.shorts) {
        const int64_t j = blockIdx.x - a.shorts;
        for (int slot = 0; slot < kSlots; ++slot) {
            const ChunkPart p(a, j, slot);
            if (!p.any) continue;
            float s[N], q[N];
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = q[i] = 0.0f;
            if (at.m) {
                saved_stats(a, at, p.graph, ch);
                each_pair<T>(a, at, p.lo, p.hi, [&](int64_t, const Raw<T> &v, const Raw<T> &g) { add_pair<T, ACT, N>(v, g, ch, s, q); });
            }
            float *out = static_cast<float *>(a.part) + ((j * kSlots + slot) * a.groups + at.g0) * 2;
            group_part(s, q, [&](int g, float s1, float q1) { out[g * 2] = s1, out[g * 2 + 1] = q1; });
        }
    } else {
        for (int64_t graph = blockIdx.x; graph < a.graphs; graph += a.shorts) {
            const int64_t lo = begin_of(a, graph), hi = begin_of(a, graph + 1);
            if (hi <= lo || hi - lo > a.chunk) continue;
            const float over = 1.0f / ((float)(hi - lo) * (float)a.cpg);
            auto found = [&](int g, float s1, float q1) { stat[g * 2] = s1 * over, stat[g * 2 + 1] = q1 * over; };
            float s[N], q[N], s1[N], s2[N];
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = q[i] = 0.0f;
            if (at.m) saved_stats(a, at, graph, ch);
            if (hi - lo <= (int64_t)kKeptBack * a.rpp) {
                const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
                Raw<T> v[kKeptBack], d[kKeptBack];
#pragma unroll
                for (int k = 0; k < kKeptBack; ++k)
                    if (lo + k * a.rpp < hi && at.m && lo + k * a.rpp + at.r < hi) {
                        v[k] = raw(x + (lo + k * a.rpp + at.r) * a.xs + at.c, at.m);
                        d[k] = raw(dy + (lo + k * a.rpp + at.r) * a.dys + at.c, at.m);
                    }
#pragma unroll
                for (int k = 0; k < kKeptBack; ++k)
                    if (lo + k * a.rpp < hi && at.m && lo + k * a.rpp + at.r < hi) add_pair<T, ACT, N>(v[k], d[k], ch, s, q);
                group_part(s, q, found);
                if (a.dx && at.m) {
                    group_means(a, at, stat, s1, s2);
#pragma unroll
                    for (int k = 0; k < kKeptBack; ++k)
                        if (lo + k * a.rpp < hi && lo + k * a.rpp + at.r < hi)
                            put_dx<T, ACT, N>(v[k], d[k], ch, s1, s2, dx + (lo + k * a.rpp + at.r) * a.C + at.c, at.m);
                }
            } else {
                if (at.m)
                    each_pair<T>(a, at, lo, hi, [&](int64_t, const Raw<T> &v, const Raw<T> &g) { add_pair<T, ACT, N>(v, g, ch, s, q); });
                group_part(s, q, found);
                if (a.dx && at.m) {
                    group_means(a, at, stat, s1, s2);
                    each_pair<T>(a, at, lo, hi, [&](int64_t row, const Raw<T> &v, const Raw<T> &g) {
                        put_dx<T, ACT, N>(v, g, ch, s1, s2, dx + row * a.C + at.c, at.m);
                    });
                }
            }
            __syncthreads(); // stat is read
        }
    }
    if (!a.sums) return;
    // the workgroup's sums of each channel
    __syncthreads();
    float *col = shared; // [2][rpp][cs]
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < at.m) {
            col[at.r * a.cs + (int)at.c - at.c0 + i] = all_s[i];
            col[(a.rpp + at.r) * a.cs + (int)at.c - at.c0 + i] = all_q[i];
        }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * (at.c1 - at.c0); k += blockDim.x) {
        const int which = k >= at.c1 - at.c0, c = k - which * (at.c1 - at.c0);
        float v = 0.0f;
        for (int r = 0; r < a.rpp; ++r) v += col[(which * a.rpp + r) * a.cs + c];
        a.sums[((int64_t)blockIdx.x * 2 + which) * a.C + at.c0 + c] = v;
    }
}

// dx of the chunks
template <typename T, int ACT> __global__ void __launch_bounds__(kMost) norm_dx_kernel(NormArgs a)
{
    constexpr int N = kPer16<T>;
    extern __shared__ double shared[];
    float *stat = reinterpret_cast<float *>(shared);
    const Place at(a, N);
    Channel<N> ch;
    ch.params(a, at);
    const int64_t j = blockIdx.x;
    T *dx = static_cast<T *>(a.dx);
    for (int slot = 0; slot < kSlots; ++slot) {
        const ChunkPart p(a, j, slot);
        if (!p.any) continue;
        const float over = 1.0f / ((float)(p.end - p.first) * (float)a.cpg);
        graph_sums<float>(a, at, p, [&](int g, float s, float q) { stat[g * 2] = s * over, stat[g * 2 + 1] = q * over; });
        if (at.m) {
            float s1[N], s2[N];
            saved_stats(a, at, p.graph, ch);
            group_means(a, at, stat, s1, s2);
            each_pair<T>(a, at, p.lo, p.hi, [&](int64_t row, const Raw<T> &v, const Raw<T> &g) {
                put_dx<T, ACT, N>(v, g, ch, s1, s2, dx + row * a.C + at.c, at.m);
            });
        }
        __syncthreads();
    }
}

// dweight and dbias: column sums of [groups of workgroups][2][C], 32 columns to a workgroup
constexpr int kSumRows = 32;
__global__ void __launch_bounds__(1024) norm_params_kernel(const float *sums, int64_t n, int64_t C, void *dw, void *db, int ptype)
{
    __shared__ float part[kSumRows][33];
    const int lane = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int64_t k = (int64_t)blockIdx.x * 32 + lane; // column of 2 C
    float v = 0.0f;
    if (k < 2 * C) {
#pragma unroll 8
        for (int64_t i = r; i < n; i += kSumRows) v += sums[i * 2 * C + k];
    }
    part[r][lane] = v;
    __syncthreads();
    if (r == 0 && k < 2 * C) {
        for (int o = 1; o < kSumRows; ++o) v += part[o][lane];
        void *to = k < C ? db : dw;
        if (to) put_param(to, ptype, k < C ? k : k - C, v);
    }
}

// ---------------------------------------------------------------------------------- launch shapes
struct NormPlan {
    int threads, slices;
    int shorts, chunks, cs, tpr, rpp, one, lanes;
    int64_t chunk;
};


// n: numbers of 16 bytes.  Few rows are cut into slices of whole groups, so that more workgroups have them.
NormPlan norm_plan(const pcsr_norm_t &a, int n, bool backward)
{
    NormPlan q;
    const int cpg = (int)(a.channels / a.groups);
    const int64_t mean = a.rows / (a.graphs > 0 ? a.graphs : 1);
    const int size = 16 / n, kept = backward ? kKeptBack : kKept;
    const int64_t bytes = mean * a.channels * size;
    q.threads = bytes <= 64 * 16 * 8 ? 64 : bytes <= 256 * 16 * 8 ? 256 : kMost;
    // a slice: whole groups, a thread to each 16 bytes of a row
    int64_t gs = a.groups;
    auto too_wide = [&](int64_t g) { return (g * cpg + n - 1) / n > q.threads; };
    while (gs > 1 && too_wide(gs)) gs = (gs + 1) / 2;
    while (q.threads < kMost && too_wide(gs)) q.threads *= 2;
    const int64_t count = a.graphs > 256 ? a.graphs : a.rows * a.channels * size / (64 << 10) + a.graphs;
    while (gs > 1 && count * ((a.groups + gs - 1) / gs) < 512 && (gs + 1) / 2 * cpg * size >= 128) gs = (gs + 1) / 2;
    q.cs = (int)(gs * cpg);
    q.slices = (int)((a.groups + gs - 1) / gs);
    q.tpr = (q.cs + n - 1) / n;
    q.rpp = q.threads / q.tpr;
    q.one = cpg % n == 0;
    q.lanes = 1;
    while (q.lanes < 64 && q.lanes * 2 * gs <= q.threads) q.lanes *= 2;
    const int64_t target = q.threads == 64 ? 4096 : q.threads == 256 ? 1024 : 512, keeps = (int64_t)kept * q.rpp;
    q.chunk = (a.rows + target - 1) / target;
    if (q.chunk < keeps) q.chunk = keeps;
    const bool known = !a.offsets || a.graphs == 1; // every graph has `mean` rows
    const bool any_short = !known || mean <= q.chunk, any_long = known ? mean > q.chunk : a.rows > q.chunk;
    const int64_t most = backward ? 4096 * 64 / q.threads : a.graphs;
    q.shorts = any_short ? (int)(a.graphs < most ? a.graphs : most) : 0;
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
    p.offsets = a.graphs == 1 ? nullptr : a.offsets, p.wide = a.wide, p.ptype = a.param_type;
    p.x = a.x, p.xs = a.x_stride, p.w = a.weight, p.b = a.bias, p.eps = a.eps, p.mean = a.mean, p.rstd = a.rstd;
    p.chunk = q.chunk, p.shorts = q.shorts, p.chunks = q.chunks, p.cs = q.cs, p.tpr = q.tpr, p.rpp = q.rpp, p.one = q.one, p.lanes = q.lanes;
    p.part = ws;
    return p;
}

template <typename F> int for_act(int act, F f)
{
    switch (act) {
    case PCSR_ACT_RELU: return f(std::integral_constant<int, PCSR_ACT_RELU>{});
    case PCSR_ACT_SILU: return f(std::integral_constant<int, PCSR_ACT_SILU>{});
    case PCSR_ACT_GELU: return f(std::integral_constant<int, PCSR_ACT_GELU>{});
    }
    return f(std::integral_constant<int, PCSR_ACT_NONE>{});
}

int64_t part_bytes(const pcsr_norm_t &a, const NormPlan &q, bool backward)
{
    return ((int64_t)q.chunks * kSlots * a.groups * 2 * (backward ? 4 : 8) + 15) / 16 * 16;
}

} // namespace
} // namespace pcsr

using namespace pcsr;

extern "C" {

int64_t pcsr_norm_workspace(const pcsr_norm_t *a, int32_t backward)
{
    if (!norm_sizes_ok(a) || a->rows == 0 || a->channels / a->groups > widest(a->type)) return 0;
    const NormPlan q = norm_plan(*a, a->type == PCSR_F32 ? 4 : 8, backward);
    return part_bytes(*a, q, backward) + (backward ? ((int64_t)q.shorts + q.chunks) * 2 * a->channels * 4 : 0);
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
        NormArgs p = norm_args(*a, q, ws);
        p.y = y;
        const size_t stat = sizeof(float) * 2 * (q.cs / p.cpg), lds = sizeof(double) * 2 * q.rpp * (q.one ? q.tpr : q.cs) + stat;
        return for_act(a->act, [&](auto v) {
            constexpr int ACT = decltype(v)::value;
            if (!allow_lds(&norm_kernel<T, ACT>, lds)) return (int)PCSR_E_HIP;
            hipLaunchKernelGGL((norm_kernel<T, ACT>), dim3(q.shorts + q.chunks, q.slices), dim3(q.threads), lds, s, p);
            if (q.chunks) hipLaunchKernelGGL((norm_apply_kernel<T, ACT>), dim3(q.chunks, q.slices), dim3(q.threads), stat, s, p);
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
    const unsigned columns = (unsigned)((2 * a->channels + 31) / 32);
    if (a->rows == 0) {
        if (sums) hipLaunchKernelGGL(norm_params_kernel, dim3(columns), dim3(1024), 0, s, nullptr, 0, a->channels, dweight, dbias, a->param_type);
        return launched();
    }
    return for_type(a->type, [&](auto t) {
        typedef decltype(t) T;
        const NormPlan q = norm_plan(*a, kPer16<T>, true);
        if (!ws && (q.chunks || sums)) return (int)PCSR_E_INVALID_ARG;
        NormArgs p = norm_args(*a, q, ws);
        p.dy = dy, p.dys = dy_stride, p.dx = dx;
        p.sums = sums ? reinterpret_cast<float *>(static_cast<char *>(ws) + part_bytes(*a, q, true)) : nullptr;
        const size_t stat = sizeof(float) * 2 * (q.cs / p.cpg);
        const size_t first = sizeof(float) * 2 * q.rpp * (q.one ? q.tpr : q.cs) + stat, col = sizeof(float) * 2 * q.rpp * q.cs;
        const size_t lds = sums && col > first ? col : first;
        return for_act(a->act, [&](auto v) {
            constexpr int ACT = decltype(v)::value;
            if (!allow_lds(&norm_backward_kernel<T, ACT>, lds)) return (int)PCSR_E_HIP;
            hipLaunchKernelGGL((norm_backward_kernel<T, ACT>), dim3(q.shorts + q.chunks, q.slices), dim3(q.threads), lds, s, p);
            if (q.chunks && dx) hipLaunchKernelGGL((norm_dx_kernel<T, ACT>), dim3(q.chunks, q.slices), dim3(q.threads), stat, s, p);
            if (sums)
                hipLaunchKernelGGL(norm_params_kernel, dim3(columns), dim3(1024), 0, s, p.sums, (int64_t)q.shorts + q.chunks, a->channels, dweight, dbias,
                                   a->param_type);
            return launched();
        });
    });
}

} // extern "C"
