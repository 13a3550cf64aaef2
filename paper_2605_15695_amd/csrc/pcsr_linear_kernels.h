// Linear layers of any width with what follows them (see pcsr_train.h): the kernels and their launches for one type.  pcsr_linear_f32.hip,
// pcsr_linear_bf16.hip and pcsr_linear_f16.hip make them, side by side; pcsr_linear.hip has the entry points.
//
// y = r + f act(z), z = x w^T + b, f = 0 or c = 1 / (1 - p) (pcsr_drop.h).  Backward: dz = f / c act'(z) dy, dx = c dz w, dw = c dz^T x,
// db = c times the sums of dz's columns (dr = dy).  c multiplies sums in fp32 and not dz, which is rounded to x's type: fp16 ends at 65,504, and without an
// activation, or with relu, dz is dy's numbers or none.
//
// Products D[i][j] = sum over k of P(i, k) Q(j, k) run on the 16-bit matrix instructions, in tiles that go through LDS, summed in
// fp32.  An operand lies with its k side by side (x and w forward, dz for dx) or with its rows side by side (w for dx, dz and x for dw);
// the second kind is turned on its way to LDS, where k is always side by side.
//
// fp32 numbers are three bf16 numbers each, x = p0 + p1 + p2 exactly (8 bits each), and a product is the six p q of order 2^-16 and more,
// six instructions of 16 times the fp32 rate (the method: Henry, Tang and Heinecke, "Leveraging the bfloat16 Artificial Intelligence Datatype For
// Higher-Precision Computations", ARITH 2019).  Numbers are split 2^16 times as large, so that small ones keep all their pieces.  A tile that has
// met numbers of 2^31 and more is done again in fp32: of smaller ones 2^32 products, 2^94 each as they are split, stay in the range (an infinity's pieces are none).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "pcsr_act.h"
#include "pcsr_drop.h"
#include "pcsr_linear.h"
#include "pcsr_num.h"

namespace pcsr {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

constexpr int64_t up(int64_t n, int64_t by) { return (n + by - 1) / by; }
constexpr int kT = 256;
constexpr float kUp = 65536.0f, kDown = 1.0f / (65536.0f * 65536.0f), kHot = 0x1p47f; // 2^31 of a number as it is split

// what an operand's numbers are in LDS
template <typename T> struct Num {
    typedef T E;
    static constexpr int NP = 1, KS = 64; // pieces, numbers of k in a stage: 128 bytes a row
};
template <> struct Num<float> {
    typedef bfloat_t E;
    static constexpr int NP = 3, KS = 32;
};

typedef half_t h8 __attribute__((ext_vector_type(8)));
typedef bfloat_t b8 __attribute__((ext_vector_type(8)));
// 16x16x32: lane l holds A[i = l % 16][k = 8 (l / 16) ..] and B[k][j = l % 16] likewise; D[i = 4 (l / 16) + r][j = l % 16]
__device__ __forceinline__ f4 mfma(half_t, u4 a, u4 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f4 mfma(bfloat_t, u4 a, u4 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

struct Side { // an operand: number (row, k) is at[row * ld + k], turned: at[k * ld + row]
    const void *at;
    int64_t ld, n; // rows
};
template <typename T, bool TURN> __device__ __forceinline__ float number(const Side &s, int64_t row, int64_t k)
{
    const T *p = static_cast<const T *>(s.at);
    return (float)(TURN ? p[k * s.ld + row] : p[row * s.ld + k]);
}

// ---------------------------------------------------------------------------------- what follows a product
struct Tail {
    const void *bias, *residual;
    void *y, *slope;              // slope: null, or act'(z) as the backward pass reads it
    int64_t r_stride, rows, cols; // of y and slope, whose rows lie one behind the other
    int act, bias_type;
    Drop drop;
    float times; // of the sums of a backward pass's product
};

// Slopes as they are kept for the backward pass: fp32, or of 16-bit types 16 bits as well, 2^15 (s + 1/4) (0 and 1 are exact, others are 2^-16 off at
// most, gelu's up to 1.15 2^-16 more, by below_normal16; slopes are between -0.13 and 1.13, so that codes end at 45,187; 0 stands for none).  Those below zero become small far out, where a row or a column may have no others:
// from -2^-6 to -2^-45 (silu at -34) the codes from 45,312 on are their fp32 exponent and 9 bits behind it, 2^-10 off at most.  Kept in place of z: a
// slope costs eight operations beside the activation, and six to take, and forty apart from it.
template <typename T> struct Slope {
    typedef uint16_t type;
    static constexpr uint32_t first = 0xA9000000u, binades = 39, code = 45312; // -2^-45 as fp32
    static __device__ __forceinline__ uint16_t put(float s)
    {
        const uint32_t bits = __builtin_bit_cast(uint32_t, s), plain = (uint32_t)__builtin_fmaf(s, 32768.0f, 8192.5f); // (of no number 0)
        return (uint16_t)(bits - first < binades << 23 ? bits + ((code << 14) + (1u << 13) - first) >> 14 : plain);
    }
    static __device__ __forceinline__ float take(uint16_t q)
    {
        const float small = __builtin_bit_cast(float, ((uint32_t)q << 14) + (first - (code << 14))), plain = __builtin_fmaf((float)q, 1.0f / 32768.0f, -0.25f);
        return q >= code ? small : q ? plain : __builtin_nanf("");
    }
};
template <> struct Slope<float> {
    typedef float type;
    static __device__ __forceinline__ float put(float s) { return s; }
    static __device__ __forceinline__ float take(float s) { return s; }
};

// 8 numbers of x w^T at a row and a column that is a multiple of 8, m of them there (WHOLE: all); bias: theirs; r: the residual's (RES)
template <typename T, bool WHOLE, bool RES>
__device__ __forceinline__ void put8(const Tail &a, const DropKey &key, int64_t row, int64_t c, int m, float (&v)[8], const float (&bias)[8], const float (&r)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += bias[i];
    if (a.slope) {
        typedef typename Slope<T>::type S;
        float f[8];
        activate_for<sizeof(T) == 2, true>(v, f, a.act);
        S *to = static_cast<S *>(a.slope) + row * a.cols + c;
        typename Pack<S, 8>::type q;
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = Slope<T>::put(f[i]);
        if (WHOLE || m >= 8) {
            *reinterpret_cast<typename Pack<S, 8>::type *>(to) = q;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < m) to[i] = q[i];
        }
    } else {
        float none[8];
        activate_for<sizeof(T) == 2, false>(v, none, a.act);
    }
    if (a.drop.threshold) drop8(a.drop, key, (uint32_t)(c >> 3), (uint32_t)row, v);
    if (RES)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    T *to = static_cast<T *>(a.y) + row * a.cols + c;
    if (WHOLE) store<T, 8>(to, v);
    else store_upto<T, 8>(to, m, v);
}
template <typename T, bool WHOLE> __device__ __forceinline__ void bias8(const Tail &a, int64_t c, int m, float (&b)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = 0.0f;
    if (a.bias && m > 0) {
        if (a.bias_type == PCSR_F32) load_upto<float, 8>(static_cast<const float *>(a.bias) + c, WHOLE ? 8 : m, b);
        else load_upto<T, 8>(static_cast<const T *>(a.bias) + c, WHOLE ? 8 : m, b);
    }
}
// any place, on its own
template <typename T> __device__ __forceinline__ void put_one(const Tail &a, const DropKey &key, int64_t row, int64_t c, int m, float (&v)[8])
{
    float b[8], r[8];
    bias8<T, false>(a, c, m, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = 0.0f;
    if (a.residual) load_upto<T, 8>(static_cast<const T *>(a.residual) + row * a.r_stride + c, m, r);
    put8<T, false, true>(a, key, row, c, m, v, b, r);
}

// ---------------------------------------------------------------------------------- operands on their way to LDS
// Where a row's 16-byte chunk of k lies, so that what an instruction reads or writes lies in different banks.  128 bytes a row: chunks are exchanged by bits of the row's number.
// 64 bytes, four rows to all banks: likewise, by a permutation of four that suits both 16 lanes side by side and the 16 that a read of 64 x 16 bytes takes at once (four of each
// four rows, two chunks).  TURNED: 4 k of every fourth row are written at once, so 4 x 4 rows are exchanged as well (with the other's places 65 % of LDS cycles were lost to conflicts).
__device__ __forceinline__ int turn_of(int q) { return (q << 1 & 2) ^ (q & 2) ^ q >> 1; } // 0, 2, 3, 1
template <int KS, bool TURNED = false> __device__ __forceinline__ int place(int row, int chunk)
{
    if (KS == 64) return (row * 8 + (chunk ^ ((row ^ row >> 3) & 7))) * 16;
    if (TURNED) return (((row & ~15) | (row & 3) << 2 | (row >> 2 & 3)) * 4 + (chunk ^ ((row ^ row >> 4) & 3))) * 16;
    return (row * 4 + (chunk ^ turn_of(row >> 2 & 3))) * 16;
}

// two numbers side by side in k, in pieces
__device__ __forceinline__ void pieces(float x, float y, float &hot, uint32_t (&p)[3])
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef bfloat_t b2 __attribute__((ext_vector_type(2)));
    x *= kUp, y *= kUp;
    hot = __builtin_fmaxf(hot, __builtin_fmaxf(__builtin_fabsf(x), __builtin_fabsf(y)));
#pragma unroll
    for (int o = 0; o < 3; ++o) {
        p[o] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{x, y}), b2)); // both in one instruction
        if (o < 2) x -= __builtin_bit_cast(float, p[o] << 16), y -= __builtin_bit_cast(float, p[o] & 0xffff0000u);
    }
}

// R rows of KS numbers of k
template <typename T, bool TURN, int R, int THREADS> struct Loader {
    static constexpr int KS = Num<T>::KS, NP = Num<T>::NP, N = kPer16<T>;
    // a unit: 8 numbers of a row, or turned 4 of k in N rows
    static constexpr int across = TURN ? R / N : KS / 8, units = TURN ? R / N * (KS / 4) : R * (KS / 8), U = (units + THREADS - 1) / THREADS;
    static constexpr int parts = TURN ? 4 : 8 / N;
    static constexpr bool whole = units % THREADS == 0;
    typedef typename Pack<T, N>::type Raw;
    Raw raw[U][parts];

    __device__ __forceinline__ void fetch(const Side &s, int64_t row0, int64_t k0, int64_t k1, int tid)
    {
        const T *base = static_cast<const T *>(s.at);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = tid + u * THREADS;
            if (!whole && id >= units) break;
            if (TURN) {
                const int64_t row = row0 + id % across * N, k = k0 + id / across * 4;
                const int m = s.n - row >= N ? N : s.n > row ? (int)(s.n - row) : 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const T *p = base + (k + q) * s.ld + row;
                    if (k + q < k1 && m == N) raw[u][q] = *reinterpret_cast<const Raw *>(p);
                    else
#pragma unroll
                        for (int i = 0; i < N; ++i) raw[u][q][i] = k + q < k1 && i < m ? p[i] : (T)0.0f;
                }
            } else {
                int64_t row = row0 + id / across;
                row = row < s.n ? row : s.n - 1; // what comes of it is not stored
                const int64_t k = k0 + id % across * 8;
                const T *p = base + row * s.ld + k;
                if (k + 8 <= k1) {
#pragma unroll
                    for (int q = 0; q < parts; ++q) raw[u][q] = *reinterpret_cast<const Raw *>(p + q * N);
                } else {
#pragma unroll
                    for (int q = 0; q < parts; ++q)
#pragma unroll
                        for (int i = 0; i < N; ++i) raw[u][q][i] = k + q * N + i < k1 ? p[q * N + i] : (T)0.0f;
                }
            }
        }
    }
    __device__ __forceinline__ void put(char *lds, float &hot, int tid) const
    {
        constexpr int plane = R * KS * 2;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = tid + u * THREADS;
            if (!whole && id >= units) break;
            if constexpr (TURN) {
                const int row = id % across * N, kg = id / across;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    char *to = lds + place<KS, true>(row + i, kg >> 1) + (kg & 1) * 8;
                    if constexpr (NP == 3) {
                        uint32_t a[3], b[3];
                        pieces(raw[u][0][i], raw[u][1][i], hot, a);
                        pieces(raw[u][2][i], raw[u][3][i], hot, b);
#pragma unroll
                        for (int o = 0; o < 3; ++o) *reinterpret_cast<u2 *>(to + o * plane) = u2{a[o], b[o]};
                    } else {
                        typedef T t4 __attribute__((ext_vector_type(4)));
                        const t4 v = {raw[u][0][i], raw[u][1][i], raw[u][2][i], raw[u][3][i]};
                        *reinterpret_cast<t4 *>(to) = v;
                    }
                }
            } else {
                char *to = lds + place<KS>(id / across, id % across);
                if constexpr (NP == 3) {
                    uint32_t a[4][3];
#pragma unroll
                    for (int q = 0; q < 4; ++q) pieces(raw[u][q >> 1][(q & 1) * 2], raw[u][q >> 1][(q & 1) * 2 + 1], hot, a[q]);
#pragma unroll
                    for (int o = 0; o < 3; ++o) *reinterpret_cast<u4 *>(to + o * plane) = u4{a[0][o], a[1][o], a[2][o], a[3][o]};
                } else {
                    *reinterpret_cast<u4 *>(to) = __builtin_bit_cast(u4, raw[u][0]);
                }
            }
        }
    }
};

// ---------------------------------------------------------------------------------- tiles
struct TileArgs {
    Side p, q;
    int64_t K, stretch; // stretch: of k, for a workgroup
    int tiles_i, tiles_j, stretches;
    float *part; // [stretch][rows][cols] sums, null: whole sums, for `tail`
    Tail tail;
};

template <int BI_, int BJ_, int WI_, int WJ_, int PER_ = 1> struct Tiling { // PER: wavefronts to a SIMD at least
    static constexpr int per = PER_, BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_, threads = 64 * WI * WJ, FI = BI / 16 / WI, FJ = BJ / 16 / WJ;
};
typedef Tiling<128, 128, 2, 2> Wide;
typedef Tiling<128, 64, 2, 2> Tall;
typedef Tiling<64, 128, 2, 2> Flat;
typedef Tiling<64, 64, 2, 2> Small;
typedef Tiling<256, 256, 2, 4, 2> Large;
typedef Tiling<128, 256, 2, 4, 2> PiecesFlat;
typedef Tiling<256, 128, 4, 2, 2> PiecesTall;
typedef Tiling<128, 128, 2, 2, 2> StraightWide;
typedef Tiling<128, 64, 2, 2, 2> StraightTall;
typedef Tiling<64, 128, 2, 2, 2> StraightFlat;

// A workgroup's tile and stretch of k.  Workgroups are dealt to the 8 dies one by one, each with an L2 of its own: a die takes a run of tiles in
// blocks of four rows (32 of them read 12 strips of operands, side by side in one row 33), and the tiles of a stretch one after the other.
__device__ __forceinline__ void place_of(const TileArgs &a, int b, int *ti, int *tj, int *stretch)
{
    const int tiles = a.tiles_i * a.tiles_j, all = tiles * a.stretches, per = all / 8;
    const int t = b < per * 8 ? (b & 7) * per + (b >> 3) : b;
    *stretch = t / tiles;
    const int r = t - *stretch * tiles, block = r / (4 * a.tiles_j), in = r - block * 4 * a.tiles_j, n = a.tiles_i - block * 4 < 4 ? a.tiles_i - block * 4 : 4;
    *tj = in / n, *ti = block * 4 + in - *tj * n;
}


template <typename C> using Sums = f4[C::FI][C::FJ];

// Products of 32 numbers of k in pieces, with tiles side by side so that an instruction does not wait for the one before it.  They have a sum of
// their own, small ones first: the matrix instructions cut off what does not reach a sum's last bit, always downwards.
template <int N> __device__ __forceinline__ void products32(const u4 (&x)[3], const u4 (&y)[N][3], f4 (&s)[N])
{
    constexpr int P[6] = {2, 0, 1, 1, 0, 0}, Q[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int o = 0; o < 6; ++o)
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = mfma(bfloat_t(), x[P[o]], y[j][Q[o]], s[j]);
}
// 8 columns of a row in fp32, where pieces would leave the range
template <typename T, bool TP, bool TQ>
__device__ __forceinline__ void once_more(const TileArgs &a, int64_t row, int64_t col, int m, int64_t k0, int64_t k1, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
#pragma unroll 1
    for (int64_t k = k0; k < k1; ++k) {
        const float x = number<T, TP>(a.p, row, k);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < m) v[e] = __builtin_fmaf(x, number<T, TQ>(a.q, col + e, k), v[e]);
    }
}

// What becomes of a tile's sums.  They go through LDS, G times 16 rows of a wavefront at a time, so that a lane has 8 columns side by side: whole lines
// of y, and what one call of the generator is for.  again: the numbers are added up once more, in fp32.
template <typename C, int G> constexpr int out_bytes() { return C::WI * C::WJ * G * 16 * (C::FJ * 16 + 4) * 4; }

// Numbers that are used under a condition are waited for in front of it: where one path waits and another does not, a wait for everything follows behind them.
__device__ __forceinline__ void arrived(float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(x[i]));
}
struct Where { // of a wavefront's sums
    int64_t i0, col; // first row, a lane's column
    int m;           // columns that are there from it on
    int64_t k0, k1;
    int stretch;
    bool again;
};
// The rows that lie in LDS.  WHOLE: 8 columns are there or none.  RES: residuals come four rows ahead, since each is a round trip to memory.
template <typename T, bool TP, bool TQ, int ROWS, int LD, int PER, bool WHOLE, bool RES>
__device__ __forceinline__ void finish_rows(const TileArgs &a, const DropKey &key, const Where &w, const float *own, const float (&bias)[8], int lane)
{
    constexpr int NP = Num<T>::NP, step = 64 / PER, passes = ROWS / step, A = RES ? (passes < 4 ? passes : 4) : 1;
    const int r0 = lane / PER, c = lane % PER * 8;
    if (w.m <= 0) return;
#pragma unroll 1
    for (int n = 0; n < passes; n += A) {
        float res[A][8];
        if (RES)
#pragma unroll
            for (int u = 0; u < A; ++u) {
                const int64_t r = w.i0 + r0 + (n + u) * step, row = r < a.tail.rows ? r : a.tail.rows - 1;
                const T *p = static_cast<const T *>(a.tail.residual) + row * a.tail.r_stride + w.col;
                if (WHOLE) load<T, 8>(p, res[u]);
                else load_upto<T, 8>(p, w.m, res[u]);
            }
#pragma unroll
        for (int u = 0; u < A; ++u) {
            const int r = r0 + (n + u) * step;
            const int64_t row = w.i0 + r;
            float v[8];
            const f4 lo = *reinterpret_cast<const f4 *>(own + r * LD + c), hi = *reinterpret_cast<const f4 *>(own + r * LD + c + 4);
            if (RES) arrived(res[u]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = NP == 3 ? lo[e] * kDown : lo[e];
                v[e + 4] = NP == 3 ? hi[e] * kDown : hi[e];
            }
            if (row < a.tail.rows) {
                if (NP == 3 && w.again) once_more<T, TP, TQ>(a, row, w.col, w.m, w.k0, w.k1, v);
                if (!a.part) {
                    if (TQ) // (of backward passes alone)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= a.tail.times;
                    put8<T, WHOLE, RES>(a.tail, key, row, w.col, w.m, v, bias, res[u]);
                } else {
                    float *to = a.part + (w.stretch * a.tail.rows + row) * a.tail.cols + w.col;
                    if (WHOLE) store<float, 8>(to, v);
                    else store_upto<float, 8>(to, w.m, v);
                }
            }
        }
    }
}
template <typename T, bool TP, bool TQ, typename C, int G>
__device__ __forceinline__ void finish_tile(const TileArgs &a, const Sums<C> &sum, char *lds, int64_t i0, int64_t j0, int64_t k0, int64_t k1, int stretch, bool again, int tid)
{
    constexpr int FI = C::FI, FJ = C::FJ, LD = FJ * 16 + 4, per = FJ * 2; // lanes to a row
    static_assert(FI % G == 0, "whole passes");
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / C::WJ, wj = wave % C::WJ, at = lane & 15, chunk = lane >> 4;
    float *own = reinterpret_cast<float *>(lds) + wave * G * 16 * LD;
    DropKey key = {};
    if (!a.part && a.tail.drop.threshold) {
        key = key_of(a.tail.drop);
        if (blockIdx.x == 0 && tid == 0) tell_key(a.tail.drop, key);
    }
    const bool whole = a.tail.cols % 8 == 0, res = a.tail.residual && !a.part;
    Where w = {0, j0 + wj * FJ * 16 + lane % per * 8, 0, k0, k1, stretch, again};
    w.m = a.tail.cols - w.col >= 8 ? 8 : a.tail.cols > w.col ? (int)(a.tail.cols - w.col) : 0;
    float bias[8];
    bias8<T, false>(a.tail, w.col, a.part ? 0 : w.m, bias);
    arrived(bias);
    const auto pass = [&](auto g) { // (written out, not unrolled: loops of this length are not)
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) own[(i * 16 + chunk * 4 + e) * LD + j * 16 + at] = sum[g * G + i][j][e];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        w.i0 = i0 + (wi * FI + g * G) * 16;
        if (whole && res) finish_rows<T, TP, TQ, G * 16, LD, per, true, true>(a, key, w, own, bias, lane);
        else if (whole) finish_rows<T, TP, TQ, G * 16, LD, per, true, false>(a, key, w, own, bias, lane);
        else if (res) finish_rows<T, TP, TQ, G * 16, LD, per, false, true>(a, key, w, own, bias, lane);
        else finish_rows<T, TP, TQ, G * 16, LD, per, false, false>(a, key, w, own, bias, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    static_assert(FI / G <= 2, "two passes at most");
    pass(std::integral_constant<int, 0>());
    if constexpr (FI / G == 2) pass(std::integral_constant<int, 1>());
}

template <typename T, typename C> constexpr int lds_bytes()
{
    constexpr int stage = (C::BI + C::BJ) * Num<T>::KS * 2 * Num<T>::NP, out = out_bytes<C, 2>();
    return stage > out ? stage : out;
}

// Any operands.  They go through registers to LDS, one stage ahead; two to five workgroups on a compute unit fill one another's waits.  Bound by what an operand takes
// on its way (loads of single numbers at ends, turned writes, splits).  777 x 75 -> 333 in fp32 9.3 us in 78 tiles of 64 x 64 (with dropout, slopes, a residual);
// 4096 x 1001 -> 1001 in bf16 23 us, 0.35 PFLOP/s.
template <typename T, bool TP, bool TQ, typename C> __device__ __forceinline__ void tile_of(const TileArgs &a, int block, char *lds, int &met)
{
    typedef typename Num<T>::E E;
    constexpr int KS = Num<T>::KS, NP = Num<T>::NP, FI = C::FI, FJ = C::FJ;
    constexpr int planeP = C::BI * KS * 2, planeQ = C::BJ * KS * 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / C::WJ, wj = wave % C::WJ;
    int ti, tj, stretch;
    place_of(a, block, &ti, &tj, &stretch);
    const int64_t i0 = (int64_t)ti * C::BI, j0 = (int64_t)tj * C::BJ;
    const int64_t k0 = (int64_t)stretch * a.stretch, k1 = k0 + a.stretch < a.K ? k0 + a.stretch : a.K;
    if (tid == 0) met = 0;
    f4 sum[FI][FJ];
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) sum[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    float hot = 0.0f;
    Loader<T, TP, C::BI, C::threads> lp;
    Loader<T, TQ, C::BJ, C::threads> lq;
    char *ldsP = lds, *ldsQ = lds + NP * planeP;
    lp.fetch(a.p, i0, k0, k1, tid);
    lq.fetch(a.q, j0, k0, k1, tid);
    const int at = lane & 15, chunk = lane >> 4;
    for (int64_t k = k0; k < k1; k += KS) {
        lp.put(ldsP, hot, tid);
        lq.put(ldsQ, hot, tid);
        __syncthreads();
        if (k + KS < k1) {
            lp.fetch(a.p, i0, k + KS, k1, tid);
            lq.fetch(a.q, j0, k + KS, k1, tid);
        }
#pragma unroll
        for (int kk = 0; kk < KS / 32; ++kk) {
            u4 x[FI][NP], y[FJ][NP];
#pragma unroll
            for (int o = 0; o < NP; ++o) {
#pragma unroll
                for (int i = 0; i < FI; ++i)
                    x[i][o] = *reinterpret_cast<const u4 *>(ldsP + o * planeP + place<KS, TP>((wi * FI + i) * 16 + at, kk * 4 + chunk));
#pragma unroll
                for (int j = 0; j < FJ; ++j)
                    y[j][o] = *reinterpret_cast<const u4 *>(ldsQ + o * planeQ + place<KS, TQ>((wj * FJ + j) * 16 + at, kk * 4 + chunk));
            }
#pragma unroll
            for (int i = 0; i < FI; ++i) {
                if constexpr (NP == 3) {
                    f4 part[FJ];
                    products32<FJ>(x[i], y, part);
#pragma unroll
                    for (int j = 0; j < FJ; ++j) sum[i][j] += part[j];
                } else {
#pragma unroll
                    for (int j = 0; j < FJ; ++j) sum[i][j] = mfma(E(), x[i][0], y[j][0], sum[i][j]);
                }
            }
        }
        __syncthreads();
    }
    bool again = false;
    if constexpr (NP == 3) {
        if (hot >= kHot) met = 1; // (a NaN needs nothing: its pieces are NaN)
        __syncthreads();
        again = met;
    }
    finish_tile<T, TP, TQ, C, 2>(a, sum, lds, i0, j0, k0, k1, stretch, again, tid);
}
template <typename T, bool TP, bool TQ, typename C> __global__ void __launch_bounds__(C::threads) tile_kernel(TileArgs a)
{
    __shared__ __align__(16) char lds[lds_bytes<T, C>()];
    __shared__ int met;
    tile_of<T, TP, TQ, C>(a, blockIdx.x, lds, met);
}
// Both products of a backward pass side by side: where each leaves most of the chip idle.  777 x 75 -> 333 in fp32: 15 us for 13 and
// 15 (12 now that two numbers are split at once).
template <typename T> __global__ void __launch_bounds__(Small::threads) pair_kernel(TileArgs x, TileArgs w, int first)
{
    __shared__ __align__(16) char lds[lds_bytes<T, Small>()];
    __shared__ int met;
    if ((int)blockIdx.x < first) tile_of<T, false, true, Small>(x, blockIdx.x, lds, met);
    else tile_of<T, true, true, Small>(w, blockIdx.x - first, lds, met);
}

// Until at most N of the wavefront's loads are on their way and its LDS reads and writes are done, for all wavefronts.  Instructions that the compiler knows, so that its own
// waits go by what is left (behind an asm it waits for everything at the head of a loop).
template <int N> __device__ __forceinline__ void wait_for_all()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | (N >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------------------------- 16-bit numbers straight to LDS
// Tiles of operands whose rows are whole 16-byte pieces.  Pieces go from memory straight to LDS, two stages of 64 numbers of k, one of them on its way while
// the other is multiplied.  A load of a wavefront fills 1 KB.
//
// k side by side: 128 bytes a row, whose 8 pieces are exchanged by the row's number so that 8 rows read together lie in different banks.
// Rows side by side: [k][rows], turned by the LDS reads that do so: 16 lanes give the addresses of 4 numbers each, 16 rows of 4 k, and each gets the 4 k of
// one row.  A lane's k is 32 kk + 8 g + 4 h + r; kilobytes are numbered by r, g and kk, as far as that goes, and lie 1056 bytes apart: so
// the four k of a read lie in different banks, and what an instruction reads is at a distance from the lane's first address that does not depend on the lane.
template <typename T, bool TURN, int R, int THREADS> struct Straight {
    static constexpr int KS = 64, blocks = R / 8, waves = THREADS / 64, loads = blocks / waves, apart = TURN ? 1056 : 1024, bytes = blocks * apart;
    static_assert(blocks % waves == 0, "whole loads");
    uint32_t off[loads]; // bytes from the tile's first number
    const char *base;
    int64_t step;

    // k of a lane's piece in a block, and the row
    static __device__ __forceinline__ int k_of(int block, int lane)
    {
        if (!TURN) return ((lane & 7) ^ (lane >> 3)) * 8;
        const int in = lane / (R / 8), t = block + blocks * (in >> 1);
        return (t >> 4) * 32 + (t >> 2 & 3) * 8 + (in & 1) * 4 + (t & 3);
    }
    static __device__ __forceinline__ int row_of(int block, int lane) { return TURN ? lane % (R / 8) * 8 : block * 8 + (lane >> 3); }

    __device__ __forceinline__ void begin(const Side &s, int64_t row0, int64_t k0, int lane, int wave)
    {
        base = static_cast<const char *>(s.at) + (TURN ? k0 * s.ld + row0 : row0 * s.ld + k0) * 2;
        step = (TURN ? KS * s.ld : KS) * 2;
#pragma unroll
        for (int u = 0; u < loads; ++u) {
            const int block = u * waves + wave, k = k_of(block, lane), r = row_of(block, lane);
            const int64_t last = (TURN ? (s.n - 1) / 8 * 8 : s.n - 1) - row0, row = r < last ? r : last; // what comes of rows behind the last is not stored
            off[u] = (uint32_t)((TURN ? k * s.ld + row : row * s.ld + k) * 2);
        }
    }
    // loads of the stage that `base` is at; left: numbers of k that there are (WHOLE: a stage's)
    template <bool WHOLE> __device__ __forceinline__ void fetch(char *lds, int64_t left, int lane, int wave) const
    {
        typedef __attribute__((address_space(3))) void *Lds;
        typedef __attribute__((address_space(1))) const void *Global;
        if (WHOLE || left >= KS) {
#pragma unroll
            for (int u = 0; u < loads; ++u)
                __builtin_amdgcn_global_load_lds((Global)(base + off[u]), (Lds)(lds + (u * waves + wave) * apart), 16, 0, 0);
        } else {
#pragma unroll
            for (int u = 0; u < loads; ++u) {
                char *to = lds + (u * waves + wave) * apart;
                if (k_of(u * waves + wave, lane) < left) __builtin_amdgcn_global_load_lds((Global)(base + off[u]), (Lds)to, 16, 0, 0);
                else *reinterpret_cast<u4 *>(to + lane * 16) = u4{0, 0, 0, 0};
            }
        }
    }
    __device__ __forceinline__ void next() { base += step; }
    // numbers of k from 32 kk + 8 (lane / 16) on, of row 16 f + lane % 16
    static __device__ __forceinline__ u4 read(const char *lds, int f, int kk, int lane)
    {
        if constexpr (TURN) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4 *At;
            const int t = (lane >> 4) * 4 + (lane >> 2 & 3); // r + 4 g
            const char *p = lds + t % blocks * apart + t / blocks * (4 * R) + (lane & 3) * 8; // this lane's 4 of 16 rows
            p += kk * (blocks > 16 ? 16 * apart : 16 / blocks * 4 * R) + f * 32;
            const u2 lo = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)p));
            const u2 hi = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p + 2 * R)));
            return u4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            return *reinterpret_cast<const u4 *>(lds + (f * 16 + (lane & 15)) * 128 + ((kk * 4 + (lane >> 4)) ^ (lane & 7)) * 16);
        }
    }
};

template <bool TP, bool TQ, typename C> constexpr int straight_bytes()
{
    constexpr int stages = 2 * (Straight<half_t, TP, C::BI, C::threads>::bytes + Straight<half_t, TQ, C::BJ, C::threads>::bytes);
    constexpr int out = out_bytes<C, C::FI < 4 ? C::FI : 4>();
    return stages > out ? stages : out;
}
// Bound by the matrix units, which alone reach 2.4 PFLOP/s on zeros and 1.8 on random numbers here.  4096^3 in bf16: 115 us (1.2 PFLOP/s) where operands stay in caches, 126 to 135 where not,
// matrix units 51 to 54 % busy, 256 x 256 tiles (one to a compute unit: 512 numbers of operands from LDS for 65,536 products; 128 x 128 take 131 us).  32,768 x 768 -> 1000 in
// fp16 92 us, 40 of them what ends the tiles (gelu, dropout, slopes) with nothing beside it, and 113 in tiles of 128 x 128; its gradient of x 75 us in tiles of 128 x 128.
// The next numbers are read from LDS while those before are multiplied, and a stage's loads are given out when all wavefronts have read the one
// before it, which is half a stage before they multiply its last numbers.
template <typename T, bool TP, bool TQ, typename C> __global__ void __launch_bounds__(C::threads, C::per) straight_kernel(TileArgs a)
{
    extern __shared__ __align__(16) char lds[];
    typedef Straight<T, TP, C::BI, C::threads> P;
    typedef Straight<T, TQ, C::BJ, C::threads> Q;
    constexpr int FI = C::FI, FJ = C::FJ, stage = P::bytes + Q::bytes;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / C::WJ, wj = wave % C::WJ;
    int ti, tj, stretch;
    place_of(a, blockIdx.x, &ti, &tj, &stretch);
    const int64_t i0 = (int64_t)ti * C::BI, j0 = (int64_t)tj * C::BJ;
    const int64_t k0 = (int64_t)stretch * a.stretch, k1 = k0 + a.stretch < a.K ? k0 + a.stretch : a.K;
    P p;
    Q q;
    p.begin(a.p, i0, k0, lane, wave);
    q.begin(a.q, j0, k0, lane, wave);
    const int steps = (int)((k1 - k0 + 63) / 64);
    int64_t left = k1 - k0;
    const auto fetch = [&](int s, auto whole) {
        char *to = lds + (s & 1) * stage;
        p.template fetch<whole>(to, left, lane, wave);
        q.template fetch<whole>(to + P::bytes, left, lane, wave);
        p.next(), q.next(), left -= 64;
    };
    Sums<C> sum;
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) sum[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    // A stage in units of GI x FJ products of 16 x 16 x 32; the numbers of a unit are read while the one before is multiplied.
    constexpr int GI = FI < 4 ? FI : 4, per = FI / GI, units = 2 * per;
    u4 x[2][GI], y[2][FJ];
    const auto read = [&](int s, int u) {
        const char *from = lds + (s & 1) * stage;
        if (u % per == 0)
#pragma unroll
            for (int j = 0; j < FJ; ++j) y[u / per][j] = Q::read(from + P::bytes, wj * FJ + j, u / per, lane);
#pragma unroll
        for (int i = 0; i < GI; ++i) x[u & 1][i] = P::read(from, wi * FI + u % per * GI + i, u / per, lane);
    };
    const auto multiply = [&](int u, int first, int end) {
#pragma unroll
        for (int i = first; i < end; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) sum[u % per * GI + i][j] = mfma(T(), x[u & 1][i], y[u / per][j], sum[u % per * GI + i][j]);
    };
    const auto begin_of = [&](int s) { // units of stage s but the last two, and the first products of the last but one
#pragma unroll
        for (int u = 0; u < units - 1; ++u) {
            read(s, u + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(u, 0, u < units - 2 ? GI : 1);
        }
    };
    // From there to the same place of the next stage.  Wavefronts wait for one another where they have products left to do behind that, beside which loads and reads begin.
    // plain: the stage behind the next is there, a whole one.  That loop turns where everything is waited for anyway, and has no condition in it, or waits at
    // its joins are for everything.
    const auto go_on = [&](int s, auto plain) {
        wait_for_all<0>(); // stage s has been read, stage s + 1 is there
        multiply(units - 2, 1, GI);
        if (plain || s + 2 < steps) fetch(s + 2, plain);
        read(s + 1, 0);
        __builtin_amdgcn_sched_barrier(0);
        multiply(units - 1, 0, GI);
        begin_of(s + 1);
    };
    if (steps > 0) {
        fetch(0, std::false_type());
        wait_for_all<0>();
        if (steps > 1) fetch(1, std::false_type());
        read(0, 0);
        begin_of(0);
        int s = 0;
        for (const int whole = (int)((k1 - k0) / 64); s + 2 < whole; ++s) go_on(s, std::true_type());
        for (; s + 1 < steps; ++s) go_on(s, std::false_type());
        multiply(units - 2, 1, GI);
        multiply(units - 1, 0, GI);
    }
    __syncthreads(); // all of the last stage is read
    finish_tile<T, TP, TQ, C, FI < 4 ? FI : 4>(a, sum, lds, i0, j0, k0, k1, stretch, false, tid);
}

// ---------------------------------------------------------------------------------- large products of fp32 numbers
// Weights are split once, into planes [piece][k / 32][row][32] with zeros behind the ends, so that 16 rows of a stage are 1 KB for one load straight to LDS; the
// other operand, and both of a gradient of weights, are split on their way through registers.  Two stages of 32 numbers of k lie in LDS: while one is
// multiplied the next is split, and the numbers of the two after it are on their way.  96 instructions of 16 cycles to a wavefront's stage.
constexpr int kSplitBlocks = 256, kUnits = 256;
struct Planes {
    const bfloat_t *at;
    int64_t rows, plane; // padded rows, numbers of a plane
    const int *hot;      // [kSplitBlocks]: whether numbers are too large for pieces
};
struct SplitArgs {
    const float *w;
    int64_t ld, n, K, rows, chunks; // padded rows, chunks of 8 numbers of k (padded)
    bfloat_t *to;
    int *hot;
};
// Weights of 256 x 256: 5 to 7 us; 4096 x 4096: 30 us, of memory.
template <bool TURN> __global__ void __launch_bounds__(kT) split_kernel(SplitArgs a)
{
    float hot = 0.0f;
    const int64_t all = a.rows * a.chunks, plane = all * 8;
    for (int64_t id = (int64_t)blockIdx.x * kT + threadIdx.x; id < all; id += (int64_t)gridDim.x * kT) {
        // the order in which the weights lie, but for the four chunks that lie together in a plane
        const int64_t j = TURN ? id % a.rows : id / 4 % a.rows, c = TURN ? id / a.rows : id / 4 / a.rows * 4 + id % 4;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t k = c * 8 + i;
            x[i] = j < a.n && k < a.K ? a.w[TURN ? k * a.ld + j : j * a.ld + k] : 0.0f;
        }
        uint32_t p[4][3];
#pragma unroll
        for (int q = 0; q < 4; ++q) pieces(x[2 * q], x[2 * q + 1], hot, p[q]);
        bfloat_t *to = a.to + (c / 4 * a.rows + j) * 32 + c % 4 * 8;
#pragma unroll
        for (int o = 0; o < 3; ++o) *reinterpret_cast<u4 *>(to + o * plane) = u4{p[0][o], p[1][o], p[2][o], p[3][o]};
    }
    const int any = __syncthreads_or(hot >= kHot);
    if (threadIdx.x == 0) a.hot[blockIdx.x] = any;
}

template <typename C> constexpr int pieces_bytes()
{
    constexpr int stages = 2 * (C::BI + C::BJ) * 64 * 3, out = out_bytes<C, 2>();
    return stages > out ? stages : out;
}
struct Spot { // a tile and its stretch of k, which is taken in pairs of stages, two at least
    int64_t i0, j0;
    int k0, k1, end, stretch;
};
template <typename C> __device__ __forceinline__ Spot spot_of(const TileArgs &a, int tile)
{
    Spot s;
    int ti, tj;
    place_of(a, tile, &ti, &tj, &s.stretch);
    s.i0 = (int64_t)ti * C::BI, s.j0 = (int64_t)tj * C::BJ;
    s.k0 = (int)(s.stretch * a.stretch), s.k1 = (int)(s.k0 + a.stretch < a.K ? s.k0 + a.stretch : a.K);
    s.end = s.k0 + (s.k1 - s.k0 <= 128 ? 128 : (s.k1 - s.k0 + 63) / 64 * 64);
    return s;
}
// The thread's number, from which the compiler is to work out addresses where they are used: kept in registers for a whole loop they leave sums no room.
__device__ __forceinline__ int again_of(int tid)
{
    asm volatile("" : "+v"(tid));
    return tid;
}
// Products with weights.  A compute unit's workgroup takes its tiles one behind the other, and the first numbers of a tile are on their way, and in LDS, while
// what follows the one before it is done.  No load stands behind a condition, or waits behind it would be for all of them: places behind a row's end are read in front
// of it, and what lies there is put right on its way to LDS.
// 250,000 x 256 -> 256: 311 us (silu, dropout, a residual, slopes; 1.04 GB), gradient of x 220 (0.55 GB); a tile to a workgroup took 331 and 251.  Six products of 33 GFLOP would be 110 us
// at the rate of random numbers above; matrix units are 29 and 43 % busy, the rest is the ends of tiles and, in a stage, reads from LDS and the wait for numbers that were asked for one and a half
// stages before (loads return in order, so that the wait for a stage's planes is one for them too).  Halves of the wavefronts a stage apart, one moving while the other
// multiplies, took 1.04 of this for gradients.
template <bool TQ, typename C> __global__ void __launch_bounds__(C::threads, C::per) planes_kernel(TileArgs a, Planes w)
{
    typedef float T;
    typedef typename Pack<float, 4>::type Raw;
    constexpr int FI = C::FI, FJ = C::FJ, planeP = C::BI * 64, planeQ = C::BJ * 64, stage = 3 * (planeP + planeQ), waves = C::threads / 64, U = C::BI * 4 / C::threads;
    constexpr int loads = 3 * C::BJ / 16 / waves; // of planes, to a wavefront
    static_assert(3 * C::BJ / 16 % waves == 0 && C::BI * 4 % C::threads == 0 && out_bytes<C, 2>() <= stage, "whole loads, a tile's end in a stage");
    extern __shared__ __align__(16) char lds[];
    __shared__ int met[2]; // large numbers of weights, of a tile's rows
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / C::WJ, wj = wave % C::WJ;
    const int all = a.tiles_i * a.tiles_j * a.stretches, beside = all < kUnits ? all : kUnits, K = (int)a.K;
    if (tid < 2) met[tid] = 0;
    __syncthreads();
    if (tid < kSplitBlocks && w.hot[tid]) met[0] = 1;
    float hot = 0.0f;
    const char *first; // a tile's first row
    uint32_t rows[U];  // numbers from there to a thread's rows
    const auto rows_of = [&](int64_t i0) {
        first = static_cast<const char *>(a.p.at) + i0 * a.p.ld * 4;
        const int last = a.p.n - 1 - i0 < C::BI ? (int)(a.p.n - 1 - i0) : C::BI; // what comes of rows behind the last is not stored
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = (tid + u * C::threads) / 4;
            rows[u] = (uint32_t)(row < last ? row : last) * (uint32_t)a.p.ld;
        }
    };
    struct Numbers {
        Raw raw[U][2];
    } even, odd; // of stages
    const auto fetch = [&](Numbers &n, int k) {
        const int c = k + again_of(tid) % 4 * 8;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < 2; ++q) n.raw[u][q] = *reinterpret_cast<const Raw *>(first + (rows[u] + (c + q * 4 < K - 4 ? c + q * 4 : K - 4)) * 4u);
    };
    const auto load_planes = [&](char *to, int64_t j0, int k) {
        typedef __attribute__((address_space(3))) void *Lds;
        typedef __attribute__((address_space(1))) const void *Global;
        const int l = again_of(tid) & 63;
        const uint32_t off = (l >> 2) * 64 + ((l & 3) ^ turn_of(l >> 4)) * 16;
#pragma unroll
        for (int u = 0; u < loads; ++u) {
            const int b = u * waves + wave, o = b / (C::BJ / 16), row = b % (C::BJ / 16) * 16;
            const char *from = reinterpret_cast<const char *>(w.at + o * w.plane + (k / 32 * w.rows + j0 + row) * 32);
            __builtin_amdgcn_global_load_lds((Global)(from + off), (Lds)(to + 3 * planeP + o * planeQ + row * 64), 16, 0, 0);
        }
    };
    const auto put = [&](char *to, Numbers &n, int k, int k1) { // numbers of k from k on; those behind k1 are 0
        const int t = again_of(tid);
        if (k + 32 > k1) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int c = k + t % 4 * 8 + q * 4, by = c < K - 4 ? 0 : c - (K - 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) { // (upwards: those behind it are as they were)
                        float v = 0.0f;
#pragma unroll
                        for (int e = i; e < 4; ++e) v = by == e - i ? n.raw[u][q][e] : v;
                        n.raw[u][q][i] = c + i < k1 ? v : 0.0f;
                    }
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = t + u * C::threads;
            uint32_t h[4][3];
#pragma unroll
            for (int q = 0; q < 4; ++q) pieces(n.raw[u][q >> 1][(q & 1) * 2], n.raw[u][q >> 1][(q & 1) * 2 + 1], hot, h[q]);
#pragma unroll
            for (int o = 0; o < 3; ++o) *reinterpret_cast<u4 *>(to + o * planeP + place<32>(id / 4, id % 4)) = u4{h[0][o], h[1][o], h[2][o], h[3][o]};
        }
    };
    Sums<C> sum;
    // from: the stage that is multiplied, to: where the next one goes, planes of j0 and numbers of k from k to k1; n: those, then the ones two stages behind them, from `ahead` on
    const auto step = [&](char *from, char *to, Numbers &n, int64_t j0, int k, int k1, int ahead) {
        const int t = again_of(tid), at = t & 15, chunk = t >> 4 & 3;
        u4 x[FI][3], y[FJ][3];
#pragma unroll
        for (int o = 0; o < 3; ++o)
#pragma unroll
            for (int j = 0; j < FJ; ++j) y[j][o] = *reinterpret_cast<const u4 *>(from + 3 * planeP + o * planeQ + place<32>((wj * FJ + j) * 16 + at, chunk));
        const auto read = [&](int i) {
#pragma unroll
            for (int o = 0; o < 3; ++o) x[i][o] = *reinterpret_cast<const u4 *>(from + o * planeP + place<32>((wi * FI + i) * 16 + at, chunk));
        };
#pragma unroll
        for (int i = 0; i < FI / 2; ++i) read(i);
        __builtin_amdgcn_sched_barrier(0); // (reads and writes of LDS behind loads to it wait for them)
        load_planes(to, j0, k);
        const auto multiply = [&](int i) {
            f4 part[FJ];
            products32<FJ>(x[i], y, part);
#pragma unroll
            for (int j = 0; j < FJ; ++j) sum[i][j] += part[j];
        };
#pragma unroll
        for (int i = 0; i < FI / 2; ++i) multiply(i);
        __builtin_amdgcn_sched_barrier(0);
        put(to, n, k, k1);
#pragma unroll
        for (int i = FI / 2; i < FI; ++i) read(i);
        __builtin_amdgcn_sched_barrier(0); // the planes of the next stage are older than what is fetched here, which need not be there
        fetch(n, ahead);
#pragma unroll
        for (int i = FI / 2; i < FI; ++i) multiply(i);
        wait_for_all<U * 2>();
        __builtin_amdgcn_sched_barrier(0);
    };
    Spot here = spot_of<C>(a, blockIdx.x);
    rows_of(here.i0);
    fetch(even, here.k0);
    load_planes(lds, here.j0, here.k0);
    fetch(odd, here.k0 + 32);
    put(lds, even, here.k0, here.k1);
    fetch(even, here.k0 + 64);
    wait_for_all<0>();
    const bool large = met[0];
    for (int tile = blockIdx.x;; tile += beside) {
        const bool last = tile + beside >= all;
        const Spot next = last ? here : spot_of<C>(a, tile + beside); // (behind the last the last again)
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) sum[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = here.k0; k < here.end; k += 64) {
            const int left = here.end - k; // of k; what is behind is the next tile's
            step(lds, lds + stage, odd, here.j0, k + 32, here.k1, left > 64 ? k + 96 : next.k0 + 32);
            if (left == 128) rows_of(next.i0);
            step(lds + stage, lds, even, left > 64 ? here.j0 : next.j0, left > 64 ? k + 64 : next.k0, left > 64 ? here.k1 : next.k1,
                 left > 128 ? k + 128 : next.k0 + 128 - left);
        }
        if (hot >= kHot) met[1] = 1;
        wait_for_all<63>();
        const bool again = met[1];
        finish_tile<T, false, TQ, C, 2>(a, sum, lds + stage, here.i0, here.j0, here.k0, here.k1, here.stretch, again || large, again_of(tid));
        if (last) break;
        here = next;
        wait_for_all<63>();
        if (again) { // of the numbers met so far those of the next tile, in LDS, count on: a thread's own
            if (tid == 0) met[1] = 0;
            hot = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int id = tid + u * C::threads;
                const b8 v = *reinterpret_cast<const b8 *>(lds + place<32>(id / 4, id % 4));
#pragma unroll
                for (int i = 0; i < 8; ++i) hot = __builtin_fmaxf(hot, __builtin_fabsf((float)v[i]));
            }
            wait_for_all<63>();
        }
    }
}
// Gradients of weights: both operands are split on their way, and few tiles mean many stretches of k.  250,000 x 256 -> 256: 211 us in 254 workgroups (0.56 GB), matrix units 45 %
// busy (226 where writes that turn met in a bank); bound as planes_kernel is.
template <typename C> __global__ void __launch_bounds__(C::threads, C::per) pieces_kernel(TileArgs a)
{
    typedef float T;
    constexpr int KS = 32, FI = C::FI, FJ = C::FJ, planeP = C::BI * 64, planeQ = C::BJ * 64, stage = 3 * (planeP + planeQ);
    extern __shared__ __align__(16) char lds[];
    __shared__ int met;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave / C::WJ, wj = wave % C::WJ;
    int ti, tj, stretch;
    place_of(a, blockIdx.x, &ti, &tj, &stretch);
    const int64_t i0 = (int64_t)ti * C::BI, j0 = (int64_t)tj * C::BJ;
    const int64_t k0 = (int64_t)stretch * a.stretch, k1 = k0 + a.stretch < a.K ? k0 + a.stretch : a.K;
    const int steps = (int)((k1 - k0 + KS - 1) / KS);
    if (tid == 0) met = 0;
    float hot = 0.0f;
    Loader<T, true, C::BI, C::threads> p;
    Loader<T, true, C::BJ, C::threads> q;
    const auto fetch = [&](int s) {
        if (s >= steps) return;
        p.fetch(a.p, i0, k0 + s * KS, k1, tid);
        q.fetch(a.q, j0, k0 + s * KS, k1, tid);
    };
    const auto put = [&](int s) {
        if (s >= steps) return;
        char *to = lds + (s & 1) * stage;
        p.put(to, hot, tid);
        q.put(to + 3 * planeP, hot, tid);
    };
    Sums<C> sum;
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) sum[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    const int at = lane & 15, chunk = lane >> 4;
    fetch(0);
    put(0);
    fetch(1);
    wait_for_all<63>();
    for (int s = 0; s < steps; ++s) {
        const char *fromP = lds + (s & 1) * stage, *fromQ = fromP + 3 * planeP;
        u4 x[FI][3], y[FJ][3];
        const auto read = [&](int i) {
#pragma unroll
            for (int o = 0; o < 3; ++o) x[i][o] = *reinterpret_cast<const u4 *>(fromP + o * planeP + place<32, true>((wi * FI + i) * 16 + at, chunk));
        };
#pragma unroll
        for (int o = 0; o < 3; ++o)
#pragma unroll
            for (int j = 0; j < FJ; ++j) y[j][o] = *reinterpret_cast<const u4 *>(fromQ + o * planeQ + place<32, true>((wj * FJ + j) * 16 + at, chunk));
#pragma unroll
        for (int i = 0; i < FI / 2; ++i) read(i);
        const auto multiply = [&](int i) {
            f4 part[FJ];
            products32<FJ>(x[i], y, part);
#pragma unroll
            for (int j = 0; j < FJ; ++j) sum[i][j] += part[j];
        };
#pragma unroll
        for (int i = 0; i < FI / 2; ++i) multiply(i);
        put(s + 1);
        __builtin_amdgcn_sched_barrier(0);
        fetch(s + 2);
#pragma unroll
        for (int i = FI / 2; i < FI; ++i) {
            read(i);
            multiply(i);
        }
        wait_for_all<63>();
    }
    if (hot >= kHot) met = 1;
    __syncthreads();
    finish_tile<T, true, true, C, 2>(a, sum, lds, i0, j0, k0, k1, stretch, met, tid);
}

// ---------------------------------------------------------------------------------- many rows and few weights
// The weights lie in LDS for as long as the workgroup lives, in pieces, and wavefronts take 16 rows at a time, each for itself: a lane's numbers of the next rows
// are on their way to its registers while these are multiplied, nothing waits for other wavefronts, and x is read once.
// STEPS: of 32 numbers of k.  FJ tiles of 16 columns at a time.  WHOLE: all of k is there, and of columns 8 or none.  RES: a residual is there.
// 2,000,000 x 256 -> 64 in fp32 with a residual 614 to 624 us: 3.07 GB, 4.9 to 5.0 TB/s; matrix units are 35 % busy, vector units 43.  480,000 x 64 -> 256 in bf16 with gelu,
// dropout and slopes 157 us (141 where slopes were kept to 2^-16 alone): vector units are 98 % busy with what follows the product (memory would take 89).
// Loads come back in their order, and so do the waits: what a strip's end needs is asked for before the next strip's numbers, and the bias lies in LDS.
template <typename T, int STEPS> constexpr int weights_pitch() { return STEPS * 64; } // bytes of a row
// Chunks of 16 bytes are exchanged by these bits of a row's number, so that the 16 that are read at once (place) lie in different banks.
template <int STEPS> __device__ __forceinline__ int exchange(int row) { return STEPS >= 4 ? row & 15 : STEPS == 2 ? row >> 1 & 7 : turn_of(row >> 2 & 3); }
template <typename T, int STEPS> int64_t weights_bytes(int64_t cols) { return Num<T>::NP * up(cols, 64) * 64 * weights_pitch<T, STEPS>(); }

template <typename T, bool TQ, int STEPS, int FJ, bool WHOLE, bool RES> __global__ void __launch_bounds__(512) rows_kernel(TileArgs a, int groups)
{
    typedef typename Num<T>::E E;
    constexpr int NP = Num<T>::NP, N = kPer16<T>, parts = 8 / N, pitch = weights_pitch<T, STEPS>(), LD = FJ * 16 + 4, per = FJ * 2, passes = (16 * per + 63) / 64;
    typedef typename Pack<T, N>::type Raw;
    extern __shared__ __align__(16) char lds[];
    __shared__ int met;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), at = lane & 15, chunk = lane >> 4;
    const int cols = groups * FJ * 16, plane = cols * pitch;
    float *biases = reinterpret_cast<float *>(lds + NP * plane), *own = biases + cols + wave * 16 * LD;
    const int64_t rows = a.tail.rows, stride = (int64_t)gridDim.x * 8;
    const int K = (int)a.K;
    Raw raw[STEPS][parts];
    const auto row_at = [&](int64_t strip) {
        const int64_t r = strip * 16 + at, row = r < rows ? r : rows - 1; // what comes of rows behind the last is not stored
        return static_cast<const T *>(a.p.at) + row * a.p.ld + chunk * 8;
    };
    const auto fetch = [&](const T *p, int t) {
#pragma unroll
        for (int q = 0; q < parts; ++q) {
            const int k = t * 32 + chunk * 8 + q * N, o = t * 32 + q * N;
            if (WHOLE || k + N <= K) raw[t][q] = *reinterpret_cast<const Raw *>(p + o);
            else
#pragma unroll
                for (int i = 0; i < N; ++i) raw[t][q][i] = k + i < K ? p[o + i] : (T)0.0f;
        }
    };
    int64_t strip = (int64_t)blockIdx.x * 8 + wave;
    if (strip * 16 < rows) {
        const T *p = row_at(strip);
#pragma unroll
        for (int t = 0; t < STEPS; ++t) fetch(p, t);
    }
    if (tid == 0) met = 0;
    __syncthreads();
    { // weights: a thread takes two numbers of k of a row
        float hot = 0.0f;
        for (int id = tid; id < cols * STEPS * 16; id += 512) {
            const int j = TQ ? id % cols : id / (STEPS * 16), k = (TQ ? id / cols : id % (STEPS * 16)) * 2;
            T w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                w[e] = j < a.q.n && k + e < K ? static_cast<const T *>(a.q.at)[TQ ? (k + e) * a.q.ld + j : j * a.q.ld + k + e] : (T)0.0f;
            uint32_t *to = reinterpret_cast<uint32_t *>(lds + j * pitch + (k / 8 ^ exchange<STEPS>(j)) * 16 + k % 8 * 2);
            if constexpr (NP == 3) {
                uint32_t h[3];
                pieces(w[0], w[1], hot, h);
#pragma unroll
                for (int o = 0; o < 3; ++o) to[o * plane / 4] = h[o];
            } else {
                typedef T t2 __attribute__((ext_vector_type(2)));
                *to = __builtin_bit_cast(uint32_t, t2{w[0], w[1]});
            }
        }
        if (NP == 3 && hot >= kHot) met = 1;
        for (int j = tid; j < cols; j += 512) {
            float b = 0.0f;
            if (a.tail.bias && j < a.tail.cols) b = a.tail.bias_type == PCSR_F32 ? static_cast<const float *>(a.tail.bias)[j] : (float)static_cast<const T *>(a.tail.bias)[j];
            biases[j] = b;
        }
    }
    __syncthreads();
    const bool hot_weights = NP == 3 && met;
    DropKey key = {};
    if (a.tail.drop.threshold) {
        key = key_of(a.tail.drop);
        if (blockIdx.x == 0 && tid == 0) tell_key(a.tail.drop, key);
    }
    const int mine = at * pitch + (chunk ^ exchange<STEPS>(at)) * 16;
    const int c = lane % per * 8;
    float hot = 0.0f;
    for (; strip * 16 < rows; strip += stride) {
        const T *next = row_at(strip + stride); // (behind the last rows the last row again)
        const auto group = [&](int g, auto last) { // last: the next rows are fetched
            const int64_t col = g * FJ * 16 + c;
            const int m = a.tail.cols - col >= 8 ? 8 : a.tail.cols > col ? (int)(a.tail.cols - col) : 0;
            float res[passes][8]; // on its way while the products are taken
            if (RES)
#pragma unroll
                for (int h = 0; h < passes; ++h) {
                    const int64_t r = strip * 16 + lane / per + h * (64 / per), row = r < rows ? r : rows - 1;
                    const T *p = static_cast<const T *>(a.tail.residual) + row * a.tail.r_stride;
                    if (WHOLE) load<T, 8>(p + (m > 0 ? col : 0), res[h]);
                    else if (m > 0) load_upto<T, 8>(p + col, m, res[h]);
                }
            const char *w = lds + g * FJ * 16 * pitch;
            f4 sum[FJ];
#pragma unroll
            for (int j = 0; j < FJ; ++j) sum[j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                u4 x[NP];
                const int here = NP == 3 ? again_of(mine) : mine;
                if constexpr (NP == 3) {
                    // the compiler is kept from making the pieces of all steps once for all groups: registers do not hold them
#pragma unroll
                    for (int q = 0; q < parts; ++q) {
                        u4 same = __builtin_bit_cast(u4, raw[t][q]);
                        asm volatile("" : "+v"(same));
                        raw[t][q] = __builtin_bit_cast(Raw, same);
                    }
                    uint32_t h[4][3];
#pragma unroll
                    for (int q = 0; q < 4; ++q) pieces(raw[t][q >> 1][(q & 1) * 2], raw[t][q >> 1][(q & 1) * 2 + 1], hot, h[q]);
#pragma unroll
                    for (int o = 0; o < 3; ++o) x[o] = u4{h[0][o], h[1][o], h[2][o], h[3][o]};
                } else {
                    x[0] = __builtin_bit_cast(u4, raw[t][0]);
                }
                if (last) fetch(next, t);
                constexpr int B = NP == 3 ? 2 : FJ; // tiles at a time
#pragma unroll
                for (int b = 0; b < FJ; b += B) {
                    u4 y[B][NP];
#pragma unroll
                    for (int j = 0; j < B; ++j)
#pragma unroll
                        for (int o = 0; o < NP; ++o) y[j][o] = *reinterpret_cast<const u4 *>(w + o * plane + (b + j) * 16 * pitch + (t & ~3) * 64 + (here ^ (t & 3) * 64));
                    if constexpr (NP == 3) {
                        f4 part[B];
                        products32<B>(x, y, part);
#pragma unroll
                        for (int j = 0; j < B; ++j) sum[b + j] += part[j];
                    } else {
#pragma unroll
                        for (int j = 0; j < B; ++j) sum[b + j] = mfma(E(), x[0], y[j][0], sum[b + j]);
                    }
                }
                if (NP == 3) __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = 0; j < FJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) own[(chunk * 4 + e) * LD + j * 16 + at] = sum[j][e];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            float bias[8];
            load<float, 8>(biases + col, bias);
#pragma unroll
            for (int h = 0; h < passes; ++h) {
                const int r = lane / per + h * (64 / per);
                const int64_t row = strip * 16 + r;
                float v[8];
                const f4 lo = *reinterpret_cast<const f4 *>(own + r * LD + c), hi = *reinterpret_cast<const f4 *>(own + r * LD + c + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = NP == 3 ? lo[e] * kDown : lo[e];
                    v[e + 4] = NP == 3 ? hi[e] * kDown : hi[e];
                }
                if (TQ)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= a.tail.times;
                if (m > 0 && row < rows) put8<T, WHOLE, RES>(a.tail, key, row, col, m, v, bias, res[h]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
#pragma unroll 1
        for (int g = 0; g < groups - 1; ++g) group(g, std::false_type());
        group(groups - 1, std::true_type());
    }
    if (NP == 3 && (hot_weights || __any(hot >= kHot))) // the wavefront's rows with such numbers once more (a loop of its own: the addresses that it needs are kept nowhere else)
        for (strip = (int64_t)blockIdx.x * 8 + wave; strip * 16 < rows; strip += stride) {
            float most = 0.0f;
            for (int k = chunk; k < K; k += 4)
                if (strip * 16 + at < rows) most = __builtin_fmaxf(most, __builtin_fabsf(number<T, false>(a.p, strip * 16 + at, k)) * kUp);
            if (!hot_weights && !__any(most >= kHot)) continue;
            for (int64_t col = c; col < a.tail.cols; col += FJ * 16)
                for (int r = lane / per; r < 16 && strip * 16 + r < rows; r += 64 / per) {
                    const int m = a.tail.cols - col >= 8 ? 8 : (int)(a.tail.cols - col);
                    float v[8];
                    once_more<T, false, TQ>(a, strip * 16 + r, col, m, 0, a.K, v);
                    if (TQ)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= a.tail.times;
                    put_one<T>(a.tail, key, strip * 16 + r, col, m, v);
                }
        }
}

// ---------------------------------------------------------------------------------- few rows
// One to eight rows: bound by reading the weights.  `lanes` lanes take a row of them, 16 bytes each at a time, add up its products with all R rows of x in fp32,
// and put their sums together; of the lanes that then have them, lane r ends row r.
// One row, 4096 x 4096 in bf16: 9.7 us (33.6 MB; 64 x 64 take 2.8, so 4.9 TB/s of the rest).
template <typename T, int R> __global__ void __launch_bounds__(kT) few_kernel(TileArgs a, int lanes)
{
    constexpr int N = kPer16<T>, A = R == 1 ? 8 : R == 2 ? 4 : 2; // loads on their way
    const int lane = threadIdx.x % lanes, rows = (int)a.tail.rows;
    const int64_t col = (int64_t)blockIdx.x * (kT / lanes) + threadIdx.x / lanes;
    DropKey key = {};
    if (a.tail.drop.threshold) {
        key = key_of(a.tail.drop);
        if (blockIdx.x == 0 && threadIdx.x == 0) tell_key(a.tail.drop, key);
    }
    const bool there = col < a.tail.cols;
    const T *w = static_cast<const T *>(a.q.at) + (there ? col : 0) * a.q.ld, *x = static_cast<const T *>(a.p.at);
    float sum[R] = {};
    const int64_t step = (int64_t)lanes * N, whole = a.K / step * step;
    const auto take = [&](const float (&y)[N], int64_t k, int m) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v[N];
            load_upto<T, N>(x + (r < rows ? r : 0) * a.p.ld + k, m, v);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (m >= N || i < m) sum[r] = __builtin_fmaf(y[i], v[i], sum[r]);
        }
    };
    int64_t k = lane * N;
    for (; k + (A - 1) * step < whole; k += A * step) {
        float y[A][N];
#pragma unroll
        for (int u = 0; u < A; ++u) load<T, N>(w + k + u * step, y[u]);
#pragma unroll
        for (int u = 0; u < A; ++u) take(y[u], k + u * step, N);
    }
    for (; k < a.K; k += step) {
        const int m = a.K - k < N ? (int)(a.K - k) : N;
        float y[N];
        load_upto<T, N>(w + k, m, y);
        take(y, k, m);
    }
    for (int o = lanes / 2; o > 0; o /= 2)
#pragma unroll
        for (int r = 0; r < R; ++r) sum[r] += __shfl_xor(sum[r], o);
    if (lane >= rows || !there) return;
    float v[1] = {sum[0]}, f[1];
#pragma unroll
    for (int r = 1; r < R; ++r) v[0] = lane == r ? sum[r] : v[0];
    const Tail &t = a.tail;
    const int64_t at = lane * t.cols + col;
    if (t.bias) v[0] += t.bias_type == PCSR_F32 ? static_cast<const float *>(t.bias)[col] : (float)static_cast<const T *>(t.bias)[col];
    activate_for<sizeof(T) == 2, true>(v, f, t.act);
    if (t.slope) static_cast<typename Slope<T>::type *>(t.slope)[at] = Slope<T>::put(f[0]);
    if (t.drop.threshold) {
        uint32_t b[4];
        philox(key, (uint32_t)(col >> 3), (uint32_t)lane, b);
        const int e = col & 7;
        const uint32_t word = e < 4 ? (e < 2 ? b[0] : b[1]) : (e < 6 ? b[2] : b[3]), bits = e & 1 ? word >> 16 : word & 0xffffu;
        v[0] = bits >= t.drop.threshold ? v[0] * t.drop.keep : 0.0f;
    }
    if (t.residual) v[0] += (float)static_cast<const T *>(t.residual)[lane * t.r_stride + col];
    static_cast<T *>(t.y)[at] = (T)v[0];
}

// Sums of the stretches of k and what follows.  A workgroup takes `across` places of 8 columns; of its threads kT / across share a place and take
// every so-manieth stretch each, and their sums are added up in order.  127 stretches of 256 x 256: 9.6 us; three of 1000 x 768: 7.5.
struct FinishArgs {
    const float *part;
    int stretches, across;
    uint32_t groups;
    Tail tail;
};
template <typename T> __device__ __forceinline__ void finish_of(const FinishArgs &f, int64_t block, float (*sums)[9])
{
    const Tail &a = f.tail;
    const float *part = f.part;
    const int stretches = f.stretches, across = f.across;
    const uint32_t groups = f.groups;
    const int lane = threadIdx.x % across, q = threadIdx.x / across, beside = kT / across;
    const int64_t t = block * across + lane, row = t / groups, c = (t - row * groups) * 8;
    DropKey key = {};
    if (a.drop.threshold) {
        key = key_of(a.drop);
        if (t == 0 && q == 0) tell_key(a.drop, key);
    }
    const int m = a.cols - c < 8 ? (int)(a.cols - c) : 8;
    float v[8] = {};
    if (row < a.rows)
#pragma unroll 4
        for (int s = q; s < stretches; s += beside) {
            float x[8];
            load_upto<float, 8>(part + (s * a.rows + row) * a.cols + c, m, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += x[i];
        }
    if (beside > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = v[i];
        __syncthreads();
        if (q) return;
        for (int p = 1; p < beside; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += sums[p * across + lane][i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= a.times;
    if (row < a.rows) put_one<T>(a, key, row, c, m, v);
}
template <typename T> __global__ void __launch_bounds__(kT) finish_kernel(FinishArgs f)
{
    __shared__ float sums[kT][9];
    finish_of<T>(f, blockIdx.x, sums);
}

// ---------------------------------------------------------------------------------- gradient at z
struct SlopeArgs {
    const void *dy, *slope;
    int64_t dy_stride, rows, cols, ld; // ld: of dz
    void *dz;                          // null: sums alone
    float *sums;                       // [workgroup][cols], null: none
    int lanes;                         // to a row
    Drop drop;
};
constexpr int kSlopeT = 1024, kSlopeBlocks = 512; // two workgroups a compute unit: as many sums as sums_kernel adds up in 6 us

// dz = act'(z) dy or 0 where it was dropped, and c times the sums of its columns over a workgroup's rows.  A thread keeps its 8 columns and walks down the rows, the next row's numbers on their way.
// dz is rounded to T, as matrix instructions take it, which for 16-bit types makes gradients of X and W behind silu or gelu 1.41 times as inexact as their own rounding.  In two
// pieces it would not, with products over twice as many numbers: 32,768 x 768 -> 1000 in fp16 75.7 and 81.3 us for dx and dw, twice as many numbers 135 and 127; 4096^3 in bf16
// 123 and 127, 224 and 217.  That is 1.4 to 1.5 of a training pass, for gradients that are rounded once more anyway.
// Bound by memory: 250,000 x 256 in fp32 144 us (768 MB, 5.3 TB/s; 152 without the row ahead), 32,768 x 1000 in fp16 43, 4096 x 4096 in bf16 26 (100 MB).
template <typename T> __global__ void __launch_bounds__(kSlopeT) slope_kernel(SlopeArgs a)
{
    typedef typename Slope<T>::type S;
    __shared__ float part[kSlopeT][9];
    const int lane = threadIdx.x % a.lanes, r = threadIdx.x / a.lanes, per = kSlopeT / a.lanes;
    const int64_t c = ((int64_t)blockIdx.y * a.lanes + lane) * 8;
    const int m = a.cols - c >= 8 ? 8 : a.cols > c ? (int)(a.cols - c) : 0;
    DropKey key = {};
    if (a.drop.threshold) key = key_of(a.drop);
    float sum[8] = {};
    if (m > 0) {
        const int64_t step = (int64_t)gridDim.x * per; // workgroups side by side
        float next[8];
        typename Pack<S, 8>::type q, q_next;
        const auto fetch = [&](int64_t row) { // behind the last row the last again
            row = row < a.rows ? row : a.rows - 1;
            load_upto<T, 8>(static_cast<const T *>(a.dy) + row * a.dy_stride + c, m, next);
            if (a.slope) {
                const S *at = static_cast<const S *>(a.slope) + row * a.cols + c;
                if (m >= 8) {
                    q_next = *reinterpret_cast<const typename Pack<S, 8>::type *>(at);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) q_next[i] = i < m ? at[i] : (S)0;
                }
            }
        };
        int64_t row = (int64_t)blockIdx.x * per + r;
        fetch(row);
        for (; row < a.rows; row += step) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = next[i];
            q = q_next;
            fetch(row + step);
            if (a.slope)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= Slope<T>::take(q[i]);
            if (a.drop.threshold) drop8<false>(a.drop, key, (uint32_t)(c >> 3), (uint32_t)row, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += d[i]; // (behind the end 0 times something)
            if (a.dz) store_upto<T, 8>(static_cast<T *>(a.dz) + row * a.ld + c, m, d);
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[threadIdx.x][i] = sum[i];
    __syncthreads();
    for (int t = threadIdx.x; t < a.lanes * 8; t += kSlopeT) {
        float s = 0.0f;
        for (int q = 0; q < per; ++q) s += part[q * a.lanes + t / 8][t % 8];
        const int64_t col = (int64_t)blockIdx.y * a.lanes * 8 + t;
        if (col < a.cols) a.sums[blockIdx.x * a.cols + col] = s * a.drop.keep;
    }
}
// db: 16 columns to a workgroup of W threads
struct SumsArgs {
    const float *sums;
    int64_t blocks, cols;
    int type;
    void *db;
};
template <int W> __device__ __forceinline__ void sums_of(const SumsArgs &a, int64_t block, double (*part)[17])
{
    const int lane = threadIdx.x & 15, q = threadIdx.x >> 4;
    const int64_t c = block * 16 + lane;
    double s = 0.0;
    if (c < a.cols)
#pragma unroll 8
        for (int64_t b = q; b < a.blocks; b += W / 16) s += (double)a.sums[b * a.cols + c];
    part[q][lane] = s;
    __syncthreads();
    if (q || c >= a.cols) return;
    for (int p = 1; p < W / 16; ++p) s += part[p][lane];
    const float v = (float)s;
    if (a.type == PCSR_F32) static_cast<float *>(a.db)[c] = v;
    else if (a.type == PCSR_BF16) static_cast<bfloat_t *>(a.db)[c] = (bfloat_t)v;
    else static_cast<half_t *>(a.db)[c] = (half_t)v;
}
__global__ void __launch_bounds__(1024) sums_kernel(SumsArgs a)
{
    __shared__ double part[64][17];
    sums_of<1024>(a, blockIdx.x, part);
}
// What is left of a backward pass of pair_kernel, in one launch: stretches of dx, those of dw, db.
template <typename T> __global__ void __launch_bounds__(kT) last_kernel(FinishArgs x, FinishArgs w, SumsArgs b, int blocks_x, int blocks_w)
{
    __shared__ __align__(8) char memory[kT * 9 * 4];
    const int block = blockIdx.x;
    if (block < blocks_x) finish_of<T>(x, block, reinterpret_cast<float (*)[9]>(memory));
    else if (block < blocks_x + blocks_w) finish_of<T>(w, block - blocks_x, reinterpret_cast<float (*)[9]>(memory));
    else sums_of<kT>(b, block - blocks_x - blocks_w, reinterpret_cast<double (*)[17]>(memory));
}

// ---------------------------------------------------------------------------------- gradients of many rows and few weights
// dz, dx, dw and db of 16-bit numbers from one read of dy, the slopes and x, where dw fits a workgroup's registers: up to 256 columns of dy and 64 of x.
// A workgroup takes 64 or 128 rows at a time: dz and x go to LDS as they are, [row][column], the weights lie there turned, and dx = dz w reads dz by rows,
// dw += dz^T x both by columns (turned by the LDS reads).  A thread keeps its 8 columns of dy, so that db is a sum of its own; when it has used a row's numbers
// it asks for those that come next.  480,000 x 64 -> 256 in bf16, dropout: 162 to 169 us (630 MB: memory would take 102), vector units 68 % busy with the
// generator and the slopes, LDS 34 %; all wavefronts at the same of both took 1.06 of it, with one buffer too; slope_kernel and both products 285.
struct NarrowArgs {
    const void *dy, *slope, *x, *w; // slope: null for none
    int64_t dy_stride, x_stride, w_stride, rows;
    int in, out;
    void *dx;           // null: not needed, nor w
    float *part, *sums; // [workgroup][out][in] (null: not needed, nor x), [workgroup][out]
    Drop drop;
};
constexpr int kNarrowT = 1024, kNarrowBlocks = 256;
constexpr int narrow_rows(int lanes) { return lanes == 32 ? 64 : 128; } // (of 32 lanes to a row registers hold two rows' numbers beside the rest)
constexpr int64_t narrow_lds(int lanes, int64_t out, int64_t in) // dz and x, of two tiles, weights
{
    const int64_t pitch = up(out, 32) * 64 + 16, rows = narrow_rows(lanes);
    return 2 * rows * (pitch + up(in, 16) * 32 + 16) + up(in, 16) * 16 * pitch;
}

// L: lanes to a row of dy
template <typename T, int L> __global__ void __launch_bounds__(kNarrowT) narrow_kernel(NarrowArgs a)
{
    typedef typename Slope<T>::type S;
    typedef typename Pack<T, 8>::type Raw;
    typedef typename Pack<S, 8>::type RawS;
    constexpr int per = kNarrowT / L, ROWS = narrow_rows(L), passes = ROWS / per, J = ROWS / 64; // J: tiles of dx to a wavefront
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), at = lane & 15, chunk = lane >> 4;
    const int in = a.in, out = a.out, steps = (int)up(out, 32), tiles_k = (int)up(in, 16), pitch = steps * 64 + 16, pitch_x = tiles_k * 32 + 16;
    const int buffer = ROWS * (pitch + pitch_x);
    char *const ldsW = lds + 2 * buffer;
    const int64_t all = (a.rows + ROWS - 1) / ROWS;
    const int c = tid % L * 8, r0 = tid / L, xc = tid % 8 * 8, xr = tid / 8;
    const bool mine = c < out, mine_x = a.x && xc < in && xr < ROWS;
    Raw dy[passes], x;
    RawS slope[passes];
    const auto row_of = [&](int64_t tile, int r) { const int64_t row = tile * ROWS + r; return row < a.rows ? row : a.rows - 1; };
    const auto fetch = [&](int64_t tile, int u) {
        if (!mine) return;
        const int64_t row = row_of(tile, r0 + u * per);
        dy[u] = *reinterpret_cast<const Raw *>(static_cast<const T *>(a.dy) + row * a.dy_stride + c);
        if (a.slope) slope[u] = *reinterpret_cast<const RawS *>(static_cast<const S *>(a.slope) + row * out + c);
    };
    const auto fetch_x = [&](int64_t tile) {
        if (mine_x) x = *reinterpret_cast<const Raw *>(static_cast<const T *>(a.x) + row_of(tile, xr) * a.x_stride + xc);
    };
    int64_t tile = blockIdx.x;
#pragma unroll
    for (int u = 0; u < passes; ++u) fetch(tile, u);
    fetch_x(tile);
    // what is behind the ends stays 0
    for (int id = tid; id < (int)(narrow_lds(L, out, in) / 16); id += kNarrowT) *reinterpret_cast<u4 *>(lds + id * 16) = u4{0, 0, 0, 0};
    __syncthreads();
    for (int id = a.w ? tid : out * in; id < out * in; id += kNarrowT) {
        const int n = id / in, k = id - n * in;
        *reinterpret_cast<T *>(ldsW + k * pitch + n * 2) = static_cast<const T *>(a.w)[n * a.w_stride + k];
    }
    DropKey key = {};
    if (a.drop.threshold) key = key_of(a.drop);
    float sum[8] = {};
    f4 dw[4]; // 16 rows of dw, up to 64 columns
#pragma unroll
    for (int t = 0; t < 4; ++t) dw[t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    // a number of 16 rows x 16 columns that lie at 4 k a lane, turned
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4 *At;
    const auto turned = [&](const char *from, int p) {
        const char *q = from + (chunk * 8 + (lane >> 2 & 3)) * p + (lane & 3) * 8;
        const u2 lo = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)q));
        const u2 hi = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(q + 4 * p)));
        return u4{lo[0], lo[1], hi[0], hi[1]};
    };
    const auto fill = [&](int64_t tile, char *ldsZ, char *ldsX) { // with what is there of this tile; the one behind it is asked for
        const int64_t next = tile + gridDim.x;
        const auto pass = [&](auto u) {
            const int r = r0 + u * per;
            const int64_t row = tile * ROWS + r;
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = (float)dy[u][i];
            if (a.slope)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= Slope<T>::take(slope[u][i]);
            fetch(next, u);
            if (a.drop.threshold) drop8<false>(a.drop, key, (uint32_t)(c >> 3), (uint32_t)row, d);
            const bool there = row < a.rows;
            Raw g;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = there ? d[i] : 0.0f;
                sum[i] += d[i];
                g[i] = (T)d[i];
            }
            *reinterpret_cast<Raw *>(ldsZ + r * pitch + c * 2) = g;
            __builtin_amdgcn_sched_barrier(0); // one after the other: side by side registers do not hold them
        };
        if (mine) {
            pass(std::integral_constant<int, 0>());
            if constexpr (passes > 1) pass(std::integral_constant<int, 1>());
            static_assert(passes <= 2, "two passes at most");
        }
        if (mine_x) {
            Raw g = x;
            if (tile * ROWS + xr >= a.rows)
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = (T)0.0f;
            *reinterpret_cast<Raw *>(ldsX + xr * pitch_x + xc * 2) = g;
        }
        fetch_x(next);
    };
    const auto multiply = [&](int64_t tile, const char *ldsZ, const char *ldsX) {
        if (a.dx) { // 16 rows and J tiles of 16 columns to a wavefront
            const int rt = wave * J / 4, ct = wave * J % 4;
            f4 s[J];
#pragma unroll
            for (int j = 0; j < J; ++j) s[j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
            if (ct < tiles_k)
                for (int t = 0; t < steps; ++t) {
                    const u4 p = *reinterpret_cast<const u4 *>(ldsZ + (rt * 16 + at) * pitch + t * 64 + chunk * 16);
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        if (ct + j < tiles_k) s[j] = mfma(T(), p, *reinterpret_cast<const u4 *>(ldsW + ((ct + j) * 16 + at) * pitch + t * 64 + chunk * 16), s[j]);
                }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int col = (ct + j) * 16 + at;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t row = tile * ROWS + rt * 16 + chunk * 4 + e;
                    if (ct + j < tiles_k && col < in && row < a.rows) static_cast<T *>(a.dx)[row * in + col] = (T)(s[j][e] * a.drop.keep);
                }
            }
        }
        if (a.part && wave * 16 < out) // dw: 16 of its rows to a wavefront
#pragma unroll
            for (int t = 0; t < ROWS / 32; ++t) {
                const u4 p = turned(ldsZ + t * 32 * pitch + wave * 32, pitch);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < tiles_k) dw[j] = mfma(T(), p, turned(ldsX + t * 32 * pitch_x + j * 32, pitch_x), dw[j]);
            }
    };
    // Half of the wavefronts of a SIMD multiply a tile before they fill the other buffer with the next one, half afterwards, so that the one's reads from LDS
    // and the other's arithmetic share the time.
    fill(tile, lds, lds + ROWS * pitch);
    for (int cur = 0;; cur ^= buffer) {
        char *const z = lds + cur, *const z_next = lds + (cur ^ buffer);
        const bool more = tile + gridDim.x < all, first = wave >> 2 & 1;
        __syncthreads(); // the tile is whole, and all have multiplied the one before
        if (first) multiply(tile, z, z + ROWS * pitch);
        if (more) fill(tile + gridDim.x, z_next, z_next + ROWS * pitch);
        if (!first) multiply(tile, z, z + ROWS * pitch);
        if (!more) break;
        tile += gridDim.x;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = wave * 16 + chunk * 4 + e, k = j * 16 + at;
            if (a.part && n < out && k < in) a.part[((int64_t)blockIdx.x * out + n) * in + k] = dw[j][e] * a.drop.keep;
        }
    float(*const sums)[9] = reinterpret_cast<float(*)[9]>(lds); // what lay there has been read
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[tid][i] = sum[i];
    __syncthreads();
    for (int t = tid; t < out; t += kNarrowT) {
        float s = 0.0f;
        for (int q = 0; q < per; ++q) s += sums[q * L + t / 8][t % 8];
        a.sums[(int64_t)blockIdx.x * out + t] = s * a.drop.keep;
    }
}

// ---------------------------------------------------------------------------------- launches
int64_t round16(int64_t n) { return up(n, 16) * 16; }

// Whether an operand's pieces can go straight to LDS: 16-byte rows, or, with its rows side by side, runs of rows; of places that 32 bits reach.
// padded: rows behind the last one can be read up to a whole piece.
template <typename T> bool straight(const Side &s, bool turned, bool padded)
{
    return sizeof(T) == 2 && s.ld % 8 == 0 && (uintptr_t)s.at % 16 == 0 && s.ld < (1 << 22) && (!turned || s.n % 8 == 0 || padded);
}
// Whether a product with weights w can go straight to LDS, or, of fp32 numbers, to planes_kernel.
template <typename T> bool straight_with(const Side &x, const Side &w, bool turned, int64_t K)
{
    if (sizeof(T) == 4) return x.ld < (1 << 21); // places of a tile that 32 bits reach
    return K % 8 == 0 && straight<T>(x, false, false) && straight<T>(w, turned, false);
}

// How a product of I x J numbers over K is cut: into tiles, and k into stretches, whose sums go through memory, where tiles are too few for the chip.  By what each
// way's loops would take beside the other ways' (`us`): a workgroup `fixed` and, for a stage, `stage` alone on a compute unit and `beside` more for each of up to `most` that run there side by
// side; sums of stretches a launch and their bytes, twice.  Operands that come from memory and what ends a tile are left out, so that these are no times of
// large products: 47 and 60 for the gradients of 32,768 x 768 -> 1000 in fp16, which take 75 and 77 us.  The numbers are fitted to 64 products of 16 to 4096 columns over 64 to 250,000 numbers of k, in every
// way they can be cut, each table to products of its own (so that tiles of 64 x 64, one kernel for 16 bits, have two prices); what is picked takes 1.05 (16 bits, straight), 1.02 (16 bits) and 1.01 (fp32) of the best of them, at most 1.27, where
// the widest tiles that fill the chip, in as many stretches as that takes, took up to 2.8 (1024^3 in bf16: 20.8 us, now 9.4; 2048^3 39.6 and 23).
struct Plan {
    int which; // tiling
    int64_t tiles_i, tiles_j, stretch;
    int stretches;
    float us;
};
enum { WIDE, TALL, FLAT, SMALL, LARGE, PIECES_FLAT, PIECES_TALL, TILINGS };
constexpr int kTileI[] = {Wide::BI, Tall::BI, Flat::BI, Small::BI, Large::BI, PiecesFlat::BI, PiecesTall::BI};
constexpr int kTileJ[] = {Wide::BJ, Tall::BJ, Flat::BJ, Small::BJ, Large::BJ, PiecesFlat::BJ, PiecesTall::BJ};
struct Cost {
    float fixed, stage, beside;
    int most; // 0: no such way
};
struct Costs {
    float launch, bytes; // of sums of stretches; bytes in a us
    Cost of[TILINGS];
};
constexpr Costs kStraight16 = {2.8f, 5.3e6f, {{2.4f, 0.55f, 0.28f, 2}, {2.0f, 0.48f, 0.13f, 3}, {2.2f, 0.47f, 0.14f, 3}, {1.8f, 0.50f, 0.085f, 4}, {8.0f, 1.07f, 0.4f, 1}, {}, {}}};
constexpr Costs kAny16 = {3.1f, 7.7e6f, {{4.3f, 1.08f, 0.51f, 2}, {2.5f, 0.84f, 0.30f, 3}, {2.6f, 0.85f, 0.26f, 3}, {2.1f, 0.51f, 0.24f, 5}, {}, {}, {}}};
constexpr Costs kAny32 = {3.9f, 6.9e6f, {{2.3f, 2.10f, 0.99f, 2}, {0.8f, 1.47f, 0.62f, 3}, {0.7f, 1.53f, 0.62f, 2}, {0.0f, 1.02f, 0.38f, 4}, {}, {7.4f, 2.34f, 0.4f, 1}, {7.1f, 2.56f, 0.4f, 1}}};

// weights: q is W, whose planes PIECES_* write first; only: one tiling, or -1
template <typename T> Plan plan(int64_t I, int64_t J, int64_t K, bool direct, bool weights, int only = -1)
{
    const Costs &costs = sizeof(T) == 4 ? kAny32 : direct ? kStraight16 : kAny16;
    const int64_t stages = up(K, Num<T>::KS), most = stages / 2 < 1 ? 1 : stages / 2;
    Plan best = {};
    best.us = -1.0f;
    for (int which = 0; which < TILINGS; ++which) {
        const Cost &c = costs.of[which];
        if (c.most == 0 || (only >= 0 && which != only) || (which >= PIECES_FLAT && K < 64) || (weights && (which == PIECES_TALL || (which == PIECES_FLAT && !direct)))) continue;
        const int64_t ti = up(I, kTileI[which]), tj = up(J, kTileJ[which]), tiles = ti * tj;
        const int64_t fill = tiles < kUnits ? kUnits / (tiles ? tiles : 1) : 1;
        int64_t before = 0;
        for (const int64_t want : {int64_t(1), fill, 2 * fill, c.most * fill}) {
            int64_t s = want < most ? want : most;
            if (tiles >= 2 * kUnits || 4 * I * J * s > int64_t(1) << 30) s = 1;
            if (s <= before) continue;
            before = s;
            const int64_t each = up(stages, s);
            s = stages ? up(stages, each) : 1;
            if (which >= PIECES_FLAT && each * Num<T>::KS >= int64_t(1) << 31) continue; // (which count k of a stretch in 32 bits)
            const int64_t all = tiles * s, full = all / (kUnits * c.most), rest = all - full * kUnits * c.most;
            float us = (float)full * (c.fixed + (float)each * (c.stage + c.beside * (float)(c.most - 1)));
            if (rest) us += c.fixed + (float)each * (c.stage + c.beside * (float)(up(rest, kUnits) - 1));
            if (s > 1) us += costs.launch + (float)(8 * I * J * s) / costs.bytes;
            if (which >= PIECES_FLAT && weights) us += (float)(10 * J * K) / 5e6f;
            if (best.us < 0.0f || us < best.us) best = {which, ti, tj, each * Num<T>::KS, (int)s, us};
        }
    }
    return best;
}
int64_t part_bytes(const Plan &p, int64_t I, int64_t J) { return p.stretches > 1 ? round16(4 * I * J * p.stretches) : 0; }
// planes of weights, and whether numbers in them are too large
int64_t plane_rows(const Plan &p) { return p.tiles_j * PiecesFlat::BJ; }
int64_t plane_depth(int64_t K) { return up(K, 64) * 64 + 128; } // a stretch begins below K and is read to four stages of 32 from there, or to the end of its last pair
int64_t plane_bytes(const Plan &p, int64_t K) { return p.which >= PIECES_FLAT ? 3 * 2 * plane_rows(p) * plane_depth(K) + 4 * kSplitBlocks : 0; }
// workspace of a product; weights: of rows with weights
int64_t product_bytes(const Plan &p, int64_t I, int64_t J, int64_t K, bool weights) { return part_bytes(p, I, J) + (weights ? plane_bytes(p, K) : 0); }

template <typename T, bool TP, bool TQ, typename C> int launch_straight(const TileArgs &a, unsigned grid, hipStream_t stream)
{
    constexpr int bytes = straight_bytes<TP, TQ, C>();
    if (!allow_lds(&straight_kernel<T, TP, TQ, C>, bytes)) return PCSR_E_HIP;
    hipLaunchKernelGGL((straight_kernel<T, TP, TQ, C>), dim3(grid), dim3(C::threads), bytes, stream, a);
    return PCSR_OK;
}
// Many rows and few weights: what rows_kernel takes.  Weights of up to 104 KB, so that two workgroups or one of eight wavefronts fit with their own rows' room, and
// rows enough to give every wavefront some.
template <typename T> int64_t rows_lds(int64_t J, int64_t K)
{
    const int64_t w = K <= 32 ? weights_bytes<T, 1>(J) : K <= 64 ? weights_bytes<T, 2>(J) : K <= 128 ? weights_bytes<T, 4>(J) : weights_bytes<T, 8>(J);
    return w + up(J, 64) * 64 * 4 + 8 * 16 * 68 * 4;
}
// (Registers do not hold eight steps of fp32 numbers and what ends of rows take.)
template <typename T> constexpr bool ends_fit(int steps) { return sizeof(T) == 2 || steps < 8; }
// direct: tiles whose pieces go straight to LDS are as fast for more than 128 numbers of k (480,000 x 256 -> 64 in bf16: 63 us for 72).
template <typename T> bool many_rows(int64_t I, int64_t J, int64_t K, bool direct)
{
    return (K <= 128 || (K <= 256 && !(direct && sizeof(T) == 2))) && I >= 32768 && rows_lds<T>(J, K) <= 140 * 1024 && (K <= 128 || (K == 256 && J % 8 == 0) || J <= 32 || ends_fit<T>(8));
}

template <typename T, bool TQ, int STEPS> int launch_rows(const TileArgs &a, hipStream_t stream)
{
    const int64_t J = a.tail.cols, lds = rows_lds<T>(J, a.K);
    const unsigned blocks = lds <= 78 * 1024 ? 512 : 256;
    const auto go = [&](auto *kernel, int width) {
        if (!allow_lds(kernel, (size_t)lds)) return (int)PCSR_E_HIP;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(512), (size_t)lds, stream, a, (int)up(J, width));
        return (int)PCSR_OK;
    };
    const bool whole = a.K == STEPS * 32 && J % 8 == 0;
    if constexpr (TQ) { // gradients of x: nothing follows
        if (J <= 32) return go(&rows_kernel<T, TQ, STEPS, 2, false, false>, 32);
        if constexpr (ends_fit<T>(STEPS))
            if (!whole) return go(&rows_kernel<T, TQ, STEPS, 4, false, false>, 64);
        return go(&rows_kernel<T, TQ, STEPS, 4, true, false>, 64);
    } else {
        const bool res = a.tail.residual;
        if (J <= 32) return res ? go(&rows_kernel<T, TQ, STEPS, 2, false, true>, 32) : go(&rows_kernel<T, TQ, STEPS, 2, false, false>, 32);
        if constexpr (ends_fit<T>(STEPS))
            if (!whole) return res ? go(&rows_kernel<T, TQ, STEPS, 4, false, true>, 64) : go(&rows_kernel<T, TQ, STEPS, 4, false, false>, 64);
        return res ? go(&rows_kernel<T, TQ, STEPS, 4, true, true>, 64) : go(&rows_kernel<T, TQ, STEPS, 4, true, false>, 64);
    }
}

FinishArgs finish_args(const Plan &c, const float *part, const Tail &tail, unsigned *blocks)
{
    const uint32_t groups = (uint32_t)up(tail.cols, 8);
    const int64_t places = tail.rows * groups;
    int across = kT;
    while (across > 8 && places / across < 512 && kT / across * 4 < c.stretches) across /= 2;
    *blocks = (unsigned)up(places, across);
    return {part, c.stretches, across, groups, tail};
}

// direct: both operands' pieces can go straight to LDS
template <typename T, bool TP, bool TQ> int product(const Side &p, const Side &q, int64_t K, bool direct, const Plan &c, const Tail &tail, void *ws, hipStream_t stream)
{
    if constexpr (!TP) {
        if (many_rows<T>(p.n, q.n, K, direct)) {
            const TileArgs a = {p, q, K, K, 1, 1, 1, nullptr, tail};
            const int rc = K <= 32 ? launch_rows<T, TQ, 1>(a, stream) : K <= 64 ? launch_rows<T, TQ, 2>(a, stream) : K <= 128 ? launch_rows<T, TQ, 4>(a, stream) : launch_rows<T, TQ, 8>(a, stream);
            return rc == PCSR_OK ? launched() : rc;
        }
    }
    TileArgs a = {p, q, K, c.stretch, (int)c.tiles_i, (int)c.tiles_j, c.stretches, c.stretches > 1 ? static_cast<float *>(ws) : nullptr, tail};
    const unsigned grid = (unsigned)(c.tiles_i * c.tiles_j * c.stretches);
    int rc = PCSR_OK;
    bool done = false;
    if constexpr (sizeof(T) == 2) {
        if (direct && c.which != SMALL) {
            done = true;
            switch (c.which) {
            case WIDE: rc = launch_straight<T, TP, TQ, StraightWide>(a, grid, stream); break;
            case TALL: rc = launch_straight<T, TP, TQ, StraightTall>(a, grid, stream); break;
            case FLAT: rc = launch_straight<T, TP, TQ, StraightFlat>(a, grid, stream); break;
            default: rc = launch_straight<T, TP, TQ, Large>(a, grid, stream);
            }
        }
    }
    if constexpr (sizeof(T) == 4) {
        if (c.which >= PIECES_FLAT) {
            done = true;
            const auto go = [&](auto *kernel, unsigned blocks, int bytes, int threads, auto... more) {
                if (!allow_lds(kernel, (size_t)bytes)) return (int)PCSR_E_HIP;
                hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), (size_t)bytes, stream, a, more...);
                return (int)PCSR_OK;
            };
            if constexpr (TP) {
                rc = c.which == PIECES_FLAT ? go(&pieces_kernel<PiecesFlat>, grid, pieces_bytes<PiecesFlat>(), PiecesFlat::threads)
                                            : go(&pieces_kernel<PiecesTall>, grid, pieces_bytes<PiecesTall>(), PiecesTall::threads);
            } else {
                char *at = static_cast<char *>(ws) + part_bytes(c, tail.rows, tail.cols);
                const int64_t rows = plane_rows(c), chunks = plane_depth(K) / 8;
                const Planes w = {reinterpret_cast<bfloat_t *>(at + 4 * kSplitBlocks), rows, rows * chunks * 8, reinterpret_cast<int *>(at)};
                const SplitArgs s = {static_cast<const float *>(q.at), q.ld, q.n, K, rows, chunks, const_cast<bfloat_t *>(w.at), reinterpret_cast<int *>(at)};
                hipLaunchKernelGGL(split_kernel<TQ>, dim3(kSplitBlocks), dim3(kT), 0, stream, s);
                const unsigned blocks = grid < kUnits ? grid : kUnits;
                rc = go(&planes_kernel<TQ, PiecesFlat>, blocks, pieces_bytes<PiecesFlat>(), PiecesFlat::threads, w);
            }
        }
    }
    if (rc != PCSR_OK) return rc;
    if (!done) switch (c.which) {
        case WIDE: hipLaunchKernelGGL((tile_kernel<T, TP, TQ, Wide>), dim3(grid), dim3(Wide::threads), 0, stream, a); break;
        case TALL: hipLaunchKernelGGL((tile_kernel<T, TP, TQ, Tall>), dim3(grid), dim3(Tall::threads), 0, stream, a); break;
        case FLAT: hipLaunchKernelGGL((tile_kernel<T, TP, TQ, Flat>), dim3(grid), dim3(Flat::threads), 0, stream, a); break;
        default: hipLaunchKernelGGL((tile_kernel<T, TP, TQ, Small>), dim3(grid), dim3(Small::threads), 0, stream, a);
        }
    if (c.stretches > 1) {
        unsigned blocks;
        const FinishArgs f = finish_args(c, a.part, tail, &blocks);
        hipLaunchKernelGGL(finish_kernel<T>, dim3(blocks), dim3(kT), 0, stream, f);
    }
    return launched();
}

// Whether narrow_kernel takes a backward pass: rows enough to give every workgroup a few times 128.
template <typename T> bool narrow(const pcsr_linear_t &a)
{
    return sizeof(T) == 2 && a.rows >= 512 * kNarrowBlocks && a.out <= 256 && a.in <= 64 && a.out > 0 && a.in > 0 && a.out % 8 == 0 && a.in % 8 == 0;
}

// The products of a backward pass, dx = dz w and dw = dz^T x: one choice, for what runs and for what is asked for to hold its sums.
struct Ways {
    Plan best, small; // the cheapest, and in tiles of 64 x 64
};
template <typename T> Ways ways(int64_t I, int64_t J, int64_t K, bool direct, bool weights)
{
    return {plan<T>(I, J, K, direct, weights), plan<T>(I, J, K, direct, weights, SMALL)};
}
template <typename T> Ways ways_x(const pcsr_linear_t &a, bool direct) { return ways<T>(a.rows, a.in, a.out, direct, true); }
template <typename T> Ways ways_w(const pcsr_linear_t &a, bool direct) { return ways<T>(a.out, a.in, a.rows, direct, false); }
struct Products {
    Plan x, w;
    bool rows, pair;          // rows_kernel takes dx; both side by side in tiles of 64 x 64
    int64_t bytes_x, bytes_w; // of workspace that they write
    template <typename T> static Products of(const pcsr_linear_t &a, const Ways &x, const Ways &w, bool direct_x)
    {
        Products p = {x.best, w.best, many_rows<T>(a.rows, a.in, a.out, direct_x), false, 0, 0};
        // tiles of 64 x 64 for both, where side by side they take less; whatever is asked for, so that the bits do not depend on that
        const Plan &sx = x.small, &sw = w.small;
        const bool fit = sx.tiles_i * sx.tiles_j * sx.stretches + sw.tiles_i * sw.tiles_j * sw.stretches <= 1024;
        if (!p.rows && fit && 1.1f * (sx.us > sw.us ? sx.us : sw.us) < p.x.us + p.w.us + 4.0f) p.x = sx, p.w = sw;
        p.pair = !p.rows && a.in > 0 && p.x.which == SMALL && p.w.which == SMALL;
        p.bytes_x = p.rows ? 0 : round16(product_bytes(p.x, a.rows, a.in, a.out, true));
        p.bytes_w = round16(product_bytes(p.w, a.out, a.in, a.rows, false));
        return p;
    }
};

// the parts of the workspace of a backward call
struct Space {
    int64_t ld, dz, sums, x, w, bytes; // bytes of dz (rows ld numbers apart), of sums of its columns, of what the products write
    int64_t blocks; // workgroups of slope_kernel along the rows
    int lanes;
    int64_t at_sums() const { return dz; }
    int64_t at_x() const { return dz + sums; }
    int64_t at_w() const { return dz + sums + x; }
    template <typename T> static Space of(const pcsr_linear_t &a, bool own)
    {
        Space s = {};
        if (narrow<T>(a)) { // sums alone: it keeps dz to itself
            s.sums = round16(4 * kNarrowBlocks * a.out), s.w = round16(4 * kNarrowBlocks * a.out * a.in);
            s.bytes = s.sums + s.w;
            return s;
        }
        s.ld = up(a.out, 8) * 8;
        s.lanes = 1;
        while (s.lanes < 64 && s.lanes * 8 < a.out) s.lanes *= 2;
        const int64_t beside = up(a.out, s.lanes * 8), per = kSlopeT / s.lanes;
        const int64_t most = beside < kSlopeBlocks ? kSlopeBlocks / beside : 1;
        s.blocks = up(a.rows, per) < most ? up(a.rows, per) : most;
        s.dz = own ? round16(a.rows * s.ld * (int64_t)sizeof(T)) : 0;
        s.sums = round16(4 * s.blocks * a.out);
        // however the operands lie, dy's place is not known here
        const Ways x[2] = {ways_x<T>(a, false), ways_x<T>(a, true)}, w[2] = {ways_w<T>(a, false), ways_w<T>(a, true)};
        for (int d = 0; d < 4; ++d) {
            const Products p = Products::of<T>(a, x[d & 1], w[d >> 1], d & 1);
            s.x = p.bytes_x > s.x ? p.bytes_x : s.x, s.w = p.bytes_w > s.w ? p.bytes_w : s.w;
        }
        s.bytes = s.dz + s.sums + s.x + s.w;
        return s;
    }
};
template <typename T> bool forward_direct(const pcsr_linear_t &a)
{
    return straight_with<T>({a.x, a.x_stride, a.rows}, {a.w, a.w_stride, a.out}, false, a.in);
}
template <typename T> Plan forward_plan(const pcsr_linear_t &a) { return plan<T>(a.rows, a.out, a.in, forward_direct<T>(a), true); }
bool has_slope(const pcsr_linear_t &a) { return a.act != PCSR_ACT_NONE || drop_of(&a.drop).threshold; }

// Rows that few_kernel takes: more of them are read again by every group of lanes.
constexpr int64_t kFew = 8;
template <typename T> int few_rows(const TileArgs &a, hipStream_t stream)
{
    int lanes = 8; // as many as rows at least
    while (lanes < 64 && lanes * kPer16<T> < a.K) lanes *= 2;
    const dim3 grid((unsigned)up(a.tail.cols, kT / lanes));
    const int64_t rows = a.tail.rows;
    if (rows == 1) hipLaunchKernelGGL((few_kernel<T, 1>), grid, dim3(kT), 0, stream, a, lanes);
    else if (rows == 2) hipLaunchKernelGGL((few_kernel<T, 2>), grid, dim3(kT), 0, stream, a, lanes);
    else if (rows <= 4) hipLaunchKernelGGL((few_kernel<T, 4>), grid, dim3(kT), 0, stream, a, lanes);
    else hipLaunchKernelGGL((few_kernel<T, 8>), grid, dim3(kT), 0, stream, a, lanes);
    return launched();
}

// A backward call as it runs, from arguments that are checked.  at: its workspace.
struct Pass {
    bool one; // narrow_kernel takes it: what is below space is not used
    bool own; // dz is written; it is dy otherwise
    Space space;
    Side dz;
    bool direct_x, direct_w;
    Products products;
    template <typename T> static Pass of(const pcsr_linear_t &a, const void *dy, int64_t dy_stride, const void *at)
    {
        Pass p = {};
        p.own = has_slope(a);
        p.space = Space::of<T>(a, p.own);
        if ((p.one = narrow<T>(a))) return p;
        p.dz = p.own ? Side{at, p.space.ld, a.rows} : Side{dy, dy_stride, a.rows};
        p.direct_x = straight_with<T>(p.dz, {a.w, a.w_stride, a.in}, true, a.out);
        p.direct_w = straight<T>({p.dz.at, p.dz.ld, a.out}, true, p.own) && straight<T>({a.x, a.x_stride, a.in}, true, false);
        p.products = Products::of<T>(a, ways_x<T>(a, p.direct_x), ways_w<T>(a, p.direct_w), p.direct_x);
        return p;
    }
};

} // namespace

template <typename T> int64_t LinearOf<T>::workspace(const pcsr_linear_t &a, bool backward)
{
    return backward ? Space::of<T>(a, has_slope(a)).bytes : a.rows <= kFew ? 0 : product_bytes(forward_plan<T>(a), a.rows, a.out, a.in, true);
}

template <typename T> int LinearOf<T>::forward(const pcsr_linear_t &a, void *y, void *slope, void *ws, hipStream_t stream)
{
    const Tail tail = {a.bias, a.residual, y, a.act == PCSR_ACT_NONE ? nullptr : slope, a.r_stride, a.rows, a.out, a.act, a.bias_type, drop_of(&a.drop), 1.0f};
    const Side x = {a.x, a.x_stride, a.rows}, w = {a.w, a.w_stride, a.out};
    if (a.rows <= kFew) return few_rows<T>({x, w, a.in, a.in, 1, 1, 1, nullptr, tail}, stream);
    const bool direct = forward_direct<T>(a);
    return product<T, false, false>(x, w, a.in, direct, plan<T>(a.rows, a.out, a.in, direct, true), tail, ws, stream);
}

template <typename T>
int LinearOf<T>::backward(const pcsr_linear_t &a, const void *slope, const void *dy, int64_t dy_stride, void *dx, void *dw, void *db, void *ws, hipStream_t stream)
{
    char *at = static_cast<char *>(ws);
    const Pass pass = Pass::of<T>(a, dy, dy_stride, at);
    const Space &sp = pass.space;
    const bool own = pass.own;
    float *sums = reinterpret_cast<float *>(at + sp.at_sums()), *part_w = reinterpret_cast<float *>(at + sp.at_w());
    if (pass.one) { // whatever is asked for, so that the bits do not depend on that
        if constexpr (sizeof(T) == 2) {
            const NarrowArgs n = {dy, a.act == PCSR_ACT_NONE ? nullptr : slope, dw ? a.x : nullptr, dx ? a.w : nullptr, dy_stride, a.x_stride, a.w_stride, a.rows, (int)a.in, (int)a.out, dx,
                                  dw ? part_w : nullptr, sums, drop_of(&a.drop)};
            const auto go = [&](auto *kernel, int lanes) {
                const size_t lds = (size_t)narrow_lds(lanes, a.out, a.in), bytes = lds > kNarrowT * 36 ? lds : kNarrowT * 36;
                if (!allow_lds(kernel, bytes)) return (int)PCSR_E_HIP;
                hipLaunchKernelGGL(kernel, dim3(kNarrowBlocks), dim3(kNarrowT), bytes, stream, n);
                return (int)PCSR_OK;
            };
            if (const int rc = a.out <= 64 ? go(&narrow_kernel<T, 8>, 8) : a.out <= 128 ? go(&narrow_kernel<T, 16>, 16) : go(&narrow_kernel<T, 32>, 32)) return rc;
            Plan p = {};
            p.stretches = kNarrowBlocks;
            unsigned blocks = 0;
            FinishArgs f = {};
            if (dw) f = finish_args(p, n.part, {nullptr, nullptr, dw, nullptr, 0, a.out, a.in, PCSR_ACT_NONE, PCSR_F32, drop_of(nullptr), 1.0f}, &blocks);
            const SumsArgs b = {sums, kNarrowBlocks, a.out, a.bias_type, db};
            if (dw || db) hipLaunchKernelGGL(last_kernel<T>, dim3(blocks + (db ? (unsigned)up(a.out, 16) : 0)), dim3(kT), 0, stream, FinishArgs{}, f, b, 0, (int)blocks);
            return launched();
        }
    }
    if (own || db) {
        SlopeArgs s = {dy, a.act == PCSR_ACT_NONE ? nullptr : slope, dy_stride, a.rows, a.out, sp.ld, own && (dx || dw) ? at : nullptr,
                       db ? sums : nullptr, sp.lanes, drop_of(&a.drop)};
        hipLaunchKernelGGL(slope_kernel<T>, dim3((unsigned)sp.blocks, (unsigned)up(a.out, sp.lanes * 8)), dim3(kSlopeT), 0, stream, s);
    }
    const SumsArgs b = {sums, sp.blocks, a.out, a.bias_type, db};
    const float times = drop_of(&a.drop).keep;
    const Tail tail_x = {nullptr, nullptr, dx, nullptr, 0, a.rows, a.in, PCSR_ACT_NONE, PCSR_F32, drop_of(nullptr), times};
    const Tail tail_w = {nullptr, nullptr, dw, nullptr, 0, a.out, a.in, PCSR_ACT_NONE, PCSR_F32, drop_of(nullptr), times};
    const Side &dz = pass.dz, w = {a.w, a.w_stride, a.in}, g = {dz.at, dz.ld, a.out}, x = {a.x, a.x_stride, a.in};
    int rc = launched();
    if (rc != PCSR_OK) return rc;
    const Plan &px = pass.products.x, &pw = pass.products.w;
    if (dx && dw && pass.products.pair) {
        float *part_x = px.stretches > 1 ? reinterpret_cast<float *>(at + sp.at_x()) : nullptr;
        if (pw.stretches == 1) part_w = nullptr;
        const TileArgs ax = {dz, w, a.out, px.stretch, (int)px.tiles_i, (int)px.tiles_j, px.stretches, part_x, tail_x};
        const TileArgs aw = {g, x, a.rows, pw.stretch, (int)pw.tiles_i, (int)pw.tiles_j, pw.stretches, part_w, tail_w};
        const unsigned first = (unsigned)(px.tiles_i * px.tiles_j * px.stretches), second = (unsigned)(pw.tiles_i * pw.tiles_j * pw.stretches);
        hipLaunchKernelGGL(pair_kernel<T>, dim3(first + second), dim3(Small::threads), 0, stream, ax, aw, (int)first);
        unsigned blocks_x = 0, blocks_w = 0;
        FinishArgs fx = {}, fw = {};
        if (part_x) fx = finish_args(px, part_x, tail_x, &blocks_x);
        if (part_w) fw = finish_args(pw, part_w, tail_w, &blocks_w);
        const unsigned blocks = blocks_x + blocks_w + (db ? (unsigned)up(a.out, 16) : 0);
        if (blocks) hipLaunchKernelGGL(last_kernel<T>, dim3(blocks), dim3(kT), 0, stream, fx, fw, b, (int)blocks_x, (int)blocks_w);
        return launched();
    }
    if (db) {
        hipLaunchKernelGGL(sums_kernel, dim3((unsigned)up(a.out, 16)), dim3(1024), 0, stream, b);
        rc = launched();
    }
    if (dx && a.in > 0 && rc == PCSR_OK) rc = product<T, false, true>(dz, w, a.out, pass.direct_x, px, tail_x, at + sp.at_x(), stream);
    if (dw && a.in > 0 && rc == PCSR_OK) rc = product<T, true, true>(g, x, a.rows, pass.direct_w, pw, tail_w, part_w, stream);
    return rc;
}

template <typename T> void LinearOf<T>::uses(const pcsr_linear_t &a, const void *dy, int64_t dy_stride, int64_t (&ends)[4][2])
{
    const Pass pass = Pass::of<T>(a, dy, dy_stride, nullptr);
    const Space &sp = pass.space;
    const bool one = pass.one;
    const int64_t in[4][2] = {{0, pass.own && !one ? a.rows * sp.ld * (int64_t)sizeof(T) : 0},
                              {sp.at_sums(), 4 * (one ? kNarrowBlocks : sp.blocks) * a.out},
                              {sp.at_x(), one ? 0 : pass.products.bytes_x},
                              {sp.at_w(), one ? 4 * kNarrowBlocks * a.out * a.in : pass.products.bytes_w}};
    for (int k = 0; k < 4; ++k) ends[k][0] = in[k][0], ends[k][1] = in[k][0] + in[k][1];
}

} // namespace pcsr
