// Updates of weight matrices orthogonalised by Newton-Schulz products (see pcsr_train.h).
//
// X <- a X + (b A + c A A) X with A = X X^T, X the update over its Frobenius norm, turned so that it is m x n with m <= n.  Every singular
// value s of X becomes a s + b s^3 + c s^5; singular vectors stay.
//
// Products run on the fp16 matrix instructions, 16 times the rate of the fp32 ones, summed in fp32.  Operands are two fp16 numbers each,
// h + l = x to 2^-23 of it, and a product is h h + h l + l h (the last, l l, is below 2^-22): three instructions, 5 times the fp32 rate.  So it is for
// bf16 matrices as well: one fp16 number, 2^-12 of rounding, is an eighth of what their result is rounded by, but where a matrix has few directions the
// roundings do not average out, and the polynomial's terms, which cancel, make them many times as large (520 x 700 of 1 and -1 in one direction was
// off by 0.010, where the result's own rounding is 0.004 at most).  X itself is held in fp32 from step to step (a X and the sum are fp32), so that what is rounded are the
// operands of the products alone: directions of small singular values, which a step makes 3.4 times as large, keep their bits.
// fp16 ends at 65504 and loses bits below 2^-14: the planes hold numbers times a power of two that the host finds from how
// large singular values can be in that step (X0 has norm 1, then the polynomial's maximum over the range).
#include <hip/hip_runtime.h>

#include <cmath>
#include <memory>
#include <new>
#include <type_traits>

#include "pcsr_num.h"

namespace pcsr {
namespace {

typedef half_t h8 __attribute__((ext_vector_type(8)));
typedef half_t h4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kItems = 24;  // matrices of a launch
constexpr int kSteps = PCSR_ORTHO_STEPS;
constexpr int kSmall = 128; // widest side of a matrix that one workgroup takes whole
constexpr int kT = 256;
constexpr int kP = 2;       // pieces of an operand

struct Item {
    const void *grad;
    float *buf;
    void *out;
    int rows, cols;
    int64_t grad_ld, buf_ld, out_ld;
    float rate;
    int flip; // X is the transpose
};
struct Items {
    Item item[kItems];
    int update, nesterov;
    float momentum, keep;
};

// the update's number at (r, c) of the matrix; buf is written
template <typename T> __device__ __forceinline__ float take(const Items &q, const Item &it, int r, int c, bool write)
{
    const float g = (float)static_cast<const T *>(it.grad)[r * it.grad_ld + c];
    if (!it.buf) return g;
    float *at = it.buf + r * it.buf_ld + c;
    float b = *at;
    if (write) {
        b = q.momentum * b + g;
        *at = b;
    }
    return q.nesterov ? g + q.momentum * b : b;
}
template <typename T> __device__ __forceinline__ void give(const Items &q, const Item &it, int r, int c, float v)
{
    T *at = static_cast<T *>(it.out) + r * it.out_ld + c;
    *at = (T)(q.update ? q.keep * (float)*at - it.rate * v : v);
}

// what one step multiplies with, and the powers of two in the planes it reads and writes
struct Step {
    float a, b, c;
    float x, over_xx, A, over_AA, B, over_Bx, next; // of X, 1 / (of X X), of A, 1 / (A A), of B, 1 / (B X), of the X that comes out
};

// ---------------------------------------------------------------------------------- small matrices
// One workgroup of 16 wavefronts to a matrix, everything in LDS: bound by the latency
// of fifteen dependent products, so no wavefront has more than Q x Q tiles of 16 x 16.  X's planes make room for A's and B's, X transposed stays beside them, X in fp32 is in registers.
struct SmallArgs {
    Items q;
    Step step[kSteps];
    int steps;
};

// 16x16x32: lane l holds A[i = l % 16][k = 8 (l / 16) ..] and B[k][j = l % 16] likewise; D[i = 4 (l / 16) + r][j = l % 16]
template <int Q> struct Tiles {
    f4 v[Q][Q];
    __device__ void zero()
    {
#pragma unroll
        for (int i = 0; i < Q; ++i)
#pragma unroll
            for (int j = 0; j < Q; ++j) v[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
};
template <int S> struct SmallPlanes {
    static constexpr int LD = S + 8; // rows 16 bytes apart in the banks
    half_t p[kP][S][LD];
};

// sums over k of p[i][k] q[j][k]
template <int Q, int S, bool SYMMETRIC>
__device__ __forceinline__ void small_product(const SmallPlanes<S> &p, const SmallPlanes<S> &q, int K, int wr, int wc, int lane,
                                              int rows, int cols, Tiles<Q> &out)
{
    Tiles<Q> low;
    out.zero();
    low.zero();
    if (wr * Q * 16 >= rows || wc * Q * 16 >= cols || (SYMMETRIC && wc > wr)) return;
    const int i = lane & 15, k0 = (lane >> 4) * 8;
    for (int k = 0; k < K; k += 32) {
        h8 a[Q][kP], b[Q][kP];
#pragma unroll
        for (int t = 0; t < Q; ++t)
#pragma unroll
            for (int o = 0; o < kP; ++o) {
                a[t][o] = *reinterpret_cast<const h8 *>(&p.p[o][(wr * Q + t) * 16 + i][k + k0]);
                b[t][o] = *reinterpret_cast<const h8 *>(&q.p[o][(wc * Q + t) * 16 + i][k + k0]);
            }
#pragma unroll
        for (int r = 0; r < Q; ++r)
#pragma unroll
            for (int c = 0; c < Q; ++c) {
                low.v[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[r][1], b[c][0], low.v[r][c], 0, 0, 0);
                low.v[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[r][0], b[c][1], low.v[r][c], 0, 0, 0);
                out.v[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[r][0], b[c][0], out.v[r][c], 0, 0, 0);
            }
    }
#pragma unroll
    for (int r = 0; r < Q; ++r)
#pragma unroll
        for (int c = 0; c < Q; ++c) out.v[r][c] += low.v[r][c];
}

// a number times the plane's power of two, in pieces
__device__ __forceinline__ void pieces(float x, half_t (&h)[kP])
{
    h[0] = (half_t)x;
    h[1] = (half_t)(x - (float)h[0]);
}

// A lane holds four rows of its column; four lanes side by side exchange them, and each ends up with four columns of a row of its own (its
// number in the four): 8 bytes of a row in one store.
__device__ __forceinline__ h4 quad_turn(const h4 &v, int lane)
{
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    const u2 d = __builtin_bit_cast(u2, v);
    const bool odd = lane & 1, high = lane & 2;
    const unsigned keep = high ? d[1] : d[0], send = high ? d[0] : d[1];
    const unsigned got = __builtin_amdgcn_mov_dpp((int)send, 0x4e, 0xf, 0xf, true); // from the lane two further
    const unsigned even_rows = (keep & 0xffffu) | got << 16, odd_rows = keep >> 16 | (got & 0xffff0000u); // columns j and j ^ 2
    const unsigned own = odd ? odd_rows : even_rows, other = odd ? even_rows : odd_rows;
    const unsigned next = __builtin_amdgcn_mov_dpp((int)other, 0xb1, 0xf, 0xf, true); // columns j ^ 1 and j ^ 3, from the lane beside
    const unsigned x = odd ? next : own, y = odd ? own : next; // columns 0 and 1 of their pairs
    const unsigned lo = (x & 0xffffu) | y << 16, hi = x >> 16 | (y & 0xffff0000u);
    const u2 out = {high ? hi : lo, high ? lo : hi};
    return __builtin_bit_cast(h4, out);
}

// tiles into planes, as they are and transposed (where TURN)
template <int Q, int S, bool ROWS, bool TURN>
__device__ __forceinline__ void small_put(const Tiles<Q> &v, float scale, int wr, int wc, int lane, SmallPlanes<S> *rows, SmallPlanes<S> *turned)
{
#pragma unroll
    for (int r = 0; r < Q; ++r)
#pragma unroll
        for (int c = 0; c < Q; ++c) {
            const int i = (wr * Q + r) * 16 + (lane >> 4) * 4, j = (wc * Q + c) * 16 + (lane & 15);
            h4 h[kP];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                half_t t[kP];
                pieces(v.v[r][c][e] * scale, t);
#pragma unroll
                for (int o = 0; o < kP; ++o) h[o][e] = t[o];
            }
#pragma unroll
            for (int o = 0; o < kP; ++o) {
                if (ROWS) *reinterpret_cast<h4 *>(&rows->p[o][i + (lane & 3)][j & ~3]) = quad_turn(h[o], lane);
                if (TURN) *reinterpret_cast<h4 *>(&turned->p[o][j][i]) = h[o];
            }
        }
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// Ten matrices of 16 x 64 to 64 x 64 in fp32, five steps, with momentum and update: 20 us.  Q = 2: for sides above 64.
template <typename T, int Q> __global__ void __launch_bounds__(1024) small_kernel(SmallArgs a)
{
    constexpr int S = 64 * Q;
    extern __shared__ char memory[];
    __shared__ double part[16];
    typedef SmallPlanes<S> Planes;
    Planes &first = *reinterpret_cast<Planes *>(memory), &turned = *reinterpret_cast<Planes *>(memory + sizeof(Planes));
    const Item &it = a.q.item[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave >> 2, wc = wave & 3;
    const int m = it.flip ? it.cols : it.rows, n = it.flip ? it.rows : it.cols;
    Tiles<Q> X, A;
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < Q; ++r)
#pragma unroll
        for (int c = 0; c < Q; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = (wr * Q + r) * 16 + (lane >> 4) * 4 + e, j = (wc * Q + c) * 16 + (lane & 15);
                float v = 0.0f;
                if (i < m && j < n) v = it.flip ? take<T>(a.q, it, j, i, true) : take<T>(a.q, it, i, j, true);
                X.v[r][c][e] = v;
                sum += (double)v * (double)v;
            }
    sum = wave_sum(sum);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += part[w];
    const double over = sum == 0.0 ? 0.0 : 1.0 / sqrt(sum); // in 64 bits: squares of fp32 neither overflow nor vanish
#pragma unroll
    for (int r = 0; r < Q; ++r)
#pragma unroll
        for (int c = 0; c < Q; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) X.v[r][c][e] = (float)((double)X.v[r][c][e] * over);
    // of a symmetric product wavefronts on and below the diagonal have their tiles, and put them at both places
    const auto put_symmetric = [&](const Tiles<Q> &v, float scale) {
        if (wr == wc) small_put<Q, S, false, true>(v, scale, wr, wc, lane, nullptr, &first);
        if (wr > wc) small_put<Q, S, true, true>(v, scale, wr, wc, lane, &first, &first);
    };
    for (int s = 0; s < a.steps; ++s) {
        const Step &st = a.step[s];
        small_put<Q, S, true, true>(X, st.x, wr, wc, lane, &first, &turned);
        __syncthreads();
        small_product<Q, S, true>(first, first, n, wr, wc, lane, m, m, A);
#pragma unroll
        for (int r = 0; r < Q; ++r)
#pragma unroll
            for (int c = 0; c < Q; ++c) A.v[r][c] *= st.over_xx;
        __syncthreads();
        put_symmetric(A, st.A);
        __syncthreads();
        Tiles<Q> B;
        small_product<Q, S, true>(first, first, m, wr, wc, lane, m, m, B);
#pragma unroll
        for (int r = 0; r < Q; ++r)
#pragma unroll
            for (int c = 0; c < Q; ++c) B.v[r][c] = st.b * A.v[r][c] + st.c * st.over_AA * B.v[r][c];
        __syncthreads();
        put_symmetric(B, st.B);
        __syncthreads();
        small_product<Q, S, false>(first, turned, m, wr, wc, lane, m, n, A);
#pragma unroll
        for (int r = 0; r < Q; ++r)
#pragma unroll
            for (int c = 0; c < Q; ++c) X.v[r][c] = st.a * X.v[r][c] + st.over_Bx * A.v[r][c];
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < Q; ++r)
#pragma unroll
        for (int c = 0; c < Q; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = (wr * Q + r) * 16 + (lane >> 4) * 4 + e, j = (wc * Q + c) * 16 + (lane & 15);
                if (i < m && j < n) {
                    if (it.flip) give<T>(a.q, it, j, i, X.v[r][c][e]);
                    else give<T>(a.q, it, i, j, X.v[r][c][e]);
                }
            }
}

// ---------------------------------------------------------------------------------- large matrices
// Sides padded with zeros to whole tiles.  Planes of a matrix, one after the other (kP of each): X, its transpose twice (one is read while the
// other is written), A, B; then X and A in fp32.  A plane of R rows of K numbers lies as [K / 32][R][32]: what a product reads at a time,
// 32 numbers of k of a tile's rows, is one stretch of whole lines from all channels of L2.
struct Space {
    int64_t Mp, Np, x, t[2], A, B, xf, Af, bytes; // bytes of a matrix
    Space(int64_t m, int64_t n, int tile)
    {
        Mp = (m + tile - 1) / tile * tile, Np = (n + tile - 1) / tile * tile;
        int64_t at = 0;
        auto room = [&](int64_t b) { const int64_t o = at; at += b; return o; };
        x = room(2 * kP * Mp * Np), t[0] = room(2 * kP * Mp * Np), t[1] = room(2 * kP * Mp * Np), A = room(2 * kP * Mp * Mp), B = room(2 * kP * Mp * Mp);
        xf = room(4 * Mp * Np), Af = room(4 * Mp * Mp);
        bytes = at;
    }
};
__device__ __forceinline__ int64_t plane_at(int64_t R, int64_t row, int64_t k) { return (k / 32 * R + row) * 32 + k % 32; }
constexpr int kNormBlocks = 256; // partial sums of a matrix's squares

// sums of squares; buf is written.  A thread takes 16 bytes of a row, as many threads to a row as it has of them.  4096 x 4096 in bf16: 20 us.
template <typename T> __global__ void __launch_bounds__(kT) measure_kernel(Items q, double *sums)
{
    constexpr int N = kPer16<T>;
    __shared__ double part[kT / 64];
    const Item &it = q.item[blockIdx.y];
    int lanes = 1;
    while (lanes < kT && lanes * N < it.cols) lanes *= 2;
    const int lane = threadIdx.x % lanes, per = kT / lanes;
    double sum = 0.0;
    for (int64_t r = (int64_t)blockIdx.x * per + threadIdx.x / lanes; r < it.rows; r += (int64_t)gridDim.x * per)
#pragma unroll 4
        for (int c = lane * N; c < it.cols; c += lanes * N) {
            const int m = it.cols - c < N ? it.cols - c : N;
            float v[N];
            load_upto<T, N>(static_cast<const T *>(it.grad) + r * it.grad_ld + c, m, v);
            if (it.buf) {
                float b[N];
                load_upto<float, N>(it.buf + r * it.buf_ld + c, m, b);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    b[i] = q.momentum * b[i] + v[i];
                    v[i] = q.nesterov ? v[i] + q.momentum * b[i] : b[i];
                }
                store_upto<float, N>(it.buf + r * it.buf_ld + c, m, b);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) sum += (double)v[i] * (double)v[i]; // zeros behind the end
        }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) sums[blockIdx.y * kNormBlocks + blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// Products D[i][j] = sum over k of p[i][k] q[j][k], rows of both contiguous in k.
enum { MAKE_A, MAKE_B, MAKE_X, LAST_X }; // A = X X^T; B = b A + c A A; X <- a X + B X; the last one
struct ProductArgs {
    char *ws;
    Space sp;
    Step st;
    int tiles_i; // of D; symmetric: the tiles with i >= j
    int turn;    // which of the transposes is read
};

// WI x WJ wavefronts of FI x FJ tiles of 32 x 32.  Stages of 32 numbers of k go from memory straight to a ring of S places in LDS, S - 1 of
// them on their way or there while one is multiplied: a round trip to memory is some 2,000 cycles, a stage's products 500 to 1,000.  64 bytes of a row
// and piece lie together; 16-byte chunks of a row are exchanged by bits 2 and 3 of its number, so that the 16 rows that a
// quarter of a wavefront reads lie in different banks.
// 32x32x16: lane l holds A[i = l % 32][k = 8 (l / 32) ..], B[k][j = l % 32] likewise; D[i = 8 (r / 4) + 4 (l / 32) + r % 4][j = l % 32].
// A stage's products have a sum of their own, which is then added to the rest: the matrix instructions cut off what
// does not reach a sum's last bit, always downwards, and over 1,000 numbers that was 1.5 times the error of fp32 products.
template <int TI_, int TJ_, int WI_, int WJ_, int S_, int G_ = 1> struct Tiling {
    static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, S = S_, G = G_; // G: teams of WI x WJ wavefronts, each with a stretch of k
    static constexpr int threads = 64 * WI * WJ * G, FI = TI / 32 / WI, FJ = TJ / 32 / WJ, blocks = (TI + TJ) / 16 * kP; // 16 rows, 1 KB
    static constexpr int loads = blocks / (WI * WJ), stage = blocks * 1024, lds = G * S * stage;
    static_assert(blocks % (WI * WJ) == 0 && lds <= 160 * 1024 && G <= 2, "whole loads, in LDS");
};
typedef Tiling<64, 64, 2, 2, 3, 2> Few;
typedef Tiling<64, 64, 2, 2, 3> Small;
typedef Tiling<128, 128, 2, 4, 4> Large;

template <int N> __device__ __forceinline__ void wait_loads() // until N of the wavefront's loads are on their way, for all wavefronts
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <typename C> struct Sums {
    f16v v[C::FI][C::FJ];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int r = 0; r < C::FI; ++r)
#pragma unroll
            for (int c = 0; c < C::FJ; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) v[r][c][e] = 0.0f;
    }
};

struct Operand {
    const half_t *at; // the tile's rows, k = 0
    int64_t R, plane; // rows of the plane, numbers of it
};
template <typename C> __device__ __forceinline__ void product(const Operand &p, const Operand &q, int64_t Kp, char *lds, int lane, int wave, int team, Sums<C> &sum)
{
    typedef __attribute__((address_space(3))) void *Lds;
    typedef __attribute__((address_space(1))) const void *Global;
    const half_t *from[C::loads];
    int64_t step[C::loads];
#pragma unroll
    for (int u = 0; u < C::loads; ++u) {
        const int block = wave + u * C::WI * C::WJ;
        constexpr int PI = C::TI / 16, PJ = C::TJ / 16;
        const bool second = block >= kP * PI;
        const Operand &o = second ? q : p;
        const int rest = second ? block - kP * PI : block, per = second ? PJ : PI, plane = rest / per, row = (rest - plane * per) * 16 + (lane >> 2);
        step[u] = o.R * 32;
        from[u] = o.at + plane * o.plane + row * 32 + (((lane & 3) ^ (lane >> 4)) << 3) + team * (Kp / 32 / C::G) * step[u];
    }
    const auto fetch = [&](int s, int u) { // a wavefront's load of a stage
        __builtin_amdgcn_global_load_lds((Global)(from[u] + s * step[u]), (Lds)(lds + s % C::S * C::stage + (wave + u * C::WI * C::WJ) * 1024), 16, 0, 0);
    };
    const int i = lane & 31, half = lane >> 5, wr = wave / C::WJ, wc = wave % C::WJ, turn = (i >> 2) & 3;
    const int at0 = (wr * C::FI * 32 + i) * 64, at1 = (kP * C::TI + wc * C::FJ * 32 + i) * 64;
    const int steps = (int)(Kp / 32 / C::G); // sides are whole tiles of 64 at least: an even number of stages
    lds += team * C::S * C::stage;
    sum.zero();
    // The operands of 16 numbers of k are read while the 16 before are multiplied.
    struct Half {
        h8 x[C::FI][kP], y[C::FJ][kP];
    };
    const auto read = [&](int s, int kk, Half &h) {
        const char *here = lds + s % C::S * C::stage;
        const int chunk = ((kk * 2 + half) ^ turn) * 16;
#pragma unroll
        for (int o = 0; o < kP; ++o) {
#pragma unroll
            for (int f = 0; f < C::FI; ++f) h.x[f][o] = *reinterpret_cast<const h8 *>(here + at0 + (o * C::TI + f * 32) * 64 + chunk);
#pragma unroll
            for (int f = 0; f < C::FJ; ++f) h.y[f][o] = *reinterpret_cast<const h8 *>(here + at1 + (o * C::TJ + f * 32) * 64 + chunk);
        }
    };
    const auto multiply = [&](const Half &h, Sums<C> &to, auto between) {
#pragma unroll
        for (int r = 0; r < C::FI; ++r) {
#pragma unroll
            for (int c = 0; c < C::FJ; ++c) {
                to.v[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h.x[r][1], h.y[c][0], to.v[r][c], 0, 0, 0);
                to.v[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h.x[r][0], h.y[c][1], to.v[r][c], 0, 0, 0);
                to.v[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h.x[r][0], h.y[c][0], to.v[r][c], 0, 0, 0);
            }
            between(r);
        }
    };
    const auto nothing = [](int) {};
    const auto take_part = [&](Sums<C> &part) {
#pragma unroll
        for (int r = 0; r < C::FI; ++r)
#pragma unroll
            for (int c = 0; c < C::FJ; ++c) sum.v[r][c] += part.v[r][c];
    };
#pragma unroll
    for (int s = 0; s < C::S - 1; ++s)
        if (s < steps)
#pragma unroll
            for (int u = 0; u < C::loads; ++u) fetch(s, u);
    if (steps >= C::S - 1) wait_loads<C::loads * (C::S - 2)>();
    else wait_loads<0>();
    Half h0, h1;
    read(0, 0, h0);
    int s = 0;
    // Reads are issued before the products that they are to run beside: left to the compiler they come behind them, and matrix units are
    // busy 57 % of a lone tile's time.  Loads are issued between products, into the place that the barrier of the stage before has freed: all at once they
    // keep the wavefronts from their products while the memory unit takes one after the other.  No condition in the loop, or the waits at its
    // joins are for everything.
    for (; s + C::S - 1 < steps; ++s) {
        Sums<C> part;
        part.zero();
        read(s, 1, h1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(h0, part, [&](int r) {
#pragma unroll
            for (int u = r * C::loads / C::FI; u < (r + 1) * C::loads / C::FI; ++u) fetch(s + C::S - 1, u);
            __builtin_amdgcn_sched_barrier(0);
        });
        wait_loads<C::loads * (C::S - 2)>(); // all of stage s has been read by all wavefronts when they pass; stage s + 1 is there
        read(s + 1, 0, h0);
        __builtin_amdgcn_sched_barrier(0);
        multiply(h1, part, nothing);
        take_part(part);
    }
    for (; s < steps; ++s) { // the last stages: nothing is left to fetch
        Sums<C> part;
        part.zero();
        read(s, 1, h1);
        multiply(h0, part, nothing);
        wait_loads<0>();
        if (s + 1 < steps) read(s + 1, 0, h0);
        multiply(h1, part, nothing);
        take_part(part);
    }
    if (C::G == 2) { // the second team's sums
        f4 *to = reinterpret_cast<f4 *>(lds - team * C::S * C::stage) + (wave * 64 + lane);
        __syncthreads(); // the last stages are read
#pragma unroll
        for (int r = 0; r < C::FI; ++r)
#pragma unroll
            for (int c = 0; c < C::FJ; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f4 &at = to[((r * C::FJ + c) * 4 + e) * 64 * C::WI * C::WJ];
                    if (team) at = f4{sum.v[r][c][e * 4], sum.v[r][c][e * 4 + 1], sum.v[r][c][e * 4 + 2], sum.v[r][c][e * 4 + 3]};
                }
        __syncthreads();
        if (team) return;
#pragma unroll
        for (int r = 0; r < C::FI; ++r)
#pragma unroll
            for (int c = 0; c < C::FJ; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum.v[r][c][e] += to[((r * C::FJ + c) * 4 + e / 4) * 64 * C::WI * C::WJ][e % 4];
    }
}

// X and A in fp32 lie as the products' sums do, so that both are read and written 16 bytes a lane: [tile][wavefront][r][c][e][lane] of four rows
template <typename C> __device__ __forceinline__ int64_t own_place(int64_t tile, int wave, int r, int c, int e, int lane)
{
    return ((((tile * C::WI * C::WJ + wave) * C::FI + r) * C::FJ + c) * 4 + e) * 64 + lane;
}

// X0 = U / ||U|| as planes, transposed planes and fp32; 32 x 32 numbers to a workgroup.  4096 x 4096 in bf16: 63 us, 268 MB.
template <typename T, typename C> __global__ void __launch_bounds__(kT) pack_kernel(Items q, const double *sums, int blocks, char *ws, Space sp, float scale)
{
    __shared__ float tile[32][33];
    const Item &it = q.item[blockIdx.z];
    char *base = ws + blockIdx.z * sp.bytes;
    double sum = 0.0;
    for (int k = threadIdx.x & 63; k < blocks; k += 64) sum += sums[blockIdx.z * kNormBlocks + k];
    sum = wave_sum(sum);
    const double over = sum == 0.0 ? 0.0 : 1.0 / sqrt(sum);
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t i0 = (int64_t)blockIdx.y * 32, j0 = (int64_t)blockIdx.x * 32; // of X
    for (int k = ty; k < 32; k += 8) { // rows of the matrix, as they lie
        const int64_t r = (it.flip ? j0 : i0) + k, c = (it.flip ? i0 : j0) + tx;
        float v = 0.0f;
        if (r < it.rows && c < it.cols) v = (float)((double)take<T>(q, it, (int)r, (int)c, false) * over);
        tile[k][tx] = v;
    }
    __syncthreads();
    half_t *x = reinterpret_cast<half_t *>(base + sp.x), *t = reinterpret_cast<half_t *>(base + sp.t[0]);
    for (int k = ty; k < 32; k += 8) {
        const float v = it.flip ? tile[tx][k] : tile[k][tx], w = it.flip ? tile[k][tx] : tile[tx][k]; // X[i0 + k][j0 + tx], X[i0 + tx][j0 + k]
        half_t hv[kP], hw[kP];
        pieces(v * scale, hv);
        pieces(w * scale, hw);
#pragma unroll
        for (int o = 0; o < kP; ++o) {
            x[o * sp.Mp * sp.Np + plane_at(sp.Mp, i0 + k, j0 + tx)] = hv[o];
            t[o * sp.Mp * sp.Np + plane_at(sp.Np, j0 + k, i0 + tx)] = hw[o];
        }
    }
    { // as the products' sums lie: a 32 x 32 tile is 256 times four rows
        const int e = threadIdx.x >> 6, lane = threadIdx.x & 63, i = e * 8 + (lane >> 5) * 4, j = lane & 31;
        const int64_t ti = i0 / C::TI, tj = j0 / C::TJ;
        const int wr = (int)(i0 % C::TI) / (C::FI * 32), wc = (int)(j0 % C::TJ) / (C::FJ * 32), r = (int)(i0 / 32) % C::FI, c = (int)(j0 / 32) % C::FJ;
        f4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = it.flip ? tile[j][i + k] : tile[i + k][j];
        reinterpret_cast<f4 *>(base + sp.xf)[own_place<C>(tj * (sp.Mp / C::TI) + ti, wr * C::WJ + wc, r, c, e, lane)] = v;
    }
}

// Tile of a workgroup.  Workgroups are dealt to the 8 dies one by one, each with an L2 of its own: a die takes a stretch of tiles that are in
// blocks of four columns (of four rows, SYMMETRIC), so that 32 of them read 12 strips of operands where 16 x 2 of them read 18.
template <bool SYMMETRIC> __device__ __forceinline__ void place_of(int bid, int all, int tiles_i, int *ti, int *tj)
{
    constexpr int B = 4;
    const int per = all / 8, t = bid < per * 8 ? (bid & 7) * per + (bid >> 3) : bid;
    if (SYMMETRIC) {
        int g = 0, r = t; // block of rows from g on, tile in it
        for (;;) {
            const int n = tiles_i - g < B ? tiles_i - g : B, have = n * g + n * (n + 1) / 2;
            if (r < have) {
                if (r < n * g) {
                    *tj = r / n, *ti = g + r % n;
                } else {
                    r -= n * g;
                    int c = 0;
                    while (r >= n - c) r -= n - c, ++c;
                    *tj = g + c, *ti = g + c + r;
                }
                return;
            }
            r -= have, g += B;
        }
    } else {
        const int tiles_j = all / tiles_i, g = t / (tiles_i * B) * B, n = tiles_j - g < B ? tiles_j - g : B, r = t - g * tiles_i;
        *ti = r / n, *tj = g + r % n;
    }
}

// A product and what follows it: pieces of the result as the next product reads them, by rows and by columns, fp32 where it is needed again.
// 4096 x 4096: A and B 280 us each (the half with i >= j: 528 tiles of 128, 0.76 PFLOP/s of fp16 products), X 444 us (0.93 PFLOP/s; a library product of
// this size in fp16 alone 1.05 to 1.3).
// 4 of 1000 x 333 in fp32: A 11 us, B 8, X 14: a stage of two teams is 32 KB for a compute unit and takes 0.3 us, 45 bytes a cycle; the rest is the
// launch, the first round trip and what follows. Deeper rings (4 and 5 stages) and tiles of 16 x 16 side by side, which wait less for one
// another, changed nothing.
template <typename T, typename C, int MODE> __global__ void __launch_bounds__(C::threads) product_kernel(ProductArgs a, Items items)
{
    extern __shared__ char memory[];
    const Space &sp = a.sp;
    char *base = a.ws + blockIdx.y * sp.bytes;
    int ti, tj;
    place_of<MODE == MAKE_A || MODE == MAKE_B>(blockIdx.x, gridDim.x, a.tiles_i, &ti, &tj);
    const int64_t Kp = MODE == MAKE_A ? sp.Np : sp.Mp;
    const auto plane = [&](int64_t at) { return reinterpret_cast<const half_t *>(base + at); };
    Operand p, q;
    if (MODE == MAKE_A) p = q = {plane(sp.x), sp.Mp, sp.Mp * sp.Np};
    else if (MODE == MAKE_B) p = q = {plane(sp.A), sp.Mp, sp.Mp * sp.Mp};
    else p = {plane(sp.B), sp.Mp, sp.Mp * sp.Mp}, q = {plane(sp.t[a.turn]), sp.Np, sp.Mp * sp.Np};
    p.at += (int64_t)ti * C::TI * 32;
    q.at += (int64_t)tj * C::TJ * 32;
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = all / (C::WI * C::WJ), wave = all % (C::WI * C::WJ);
    Sums<C> acc;
    product<C>(p, q, Kp, memory, lane, wave, team, acc);
    if (team) return;
    const Step &st = a.st;
    const int64_t i0 = (int64_t)ti * C::TI + wave / C::WJ * C::FI * 32 + (lane >> 5) * 4, j0 = (int64_t)tj * C::TJ + wave % C::WJ * C::FJ * 32 + (lane & 31);
#pragma unroll
    for (int r = 0; r < C::FI; ++r)
#pragma unroll
        for (int c = 0; c < C::FJ; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) { // four rows in a row
                const int64_t ii = i0 + r * 32 + e * 8, jj = j0 + c * 32;
                f4 v = {acc.v[r][c][e * 4], acc.v[r][c][e * 4 + 1], acc.v[r][c][e * 4 + 2], acc.v[r][c][e * 4 + 3]};
                if (MODE == MAKE_A || MODE == MAKE_B) {
                    f4 &Af = reinterpret_cast<f4 *>(base + sp.Af)[own_place<C>(ti * (ti + 1) / 2 + tj, wave, r, c, e, lane)];
                    half_t *out = reinterpret_cast<half_t *>(base + (MODE == MAKE_A ? sp.A : sp.B));
                    if (MODE == MAKE_A) {
                        v *= st.over_xx;
                        Af = v;
                    } else {
                        v = st.b * Af + st.c * st.over_AA * v;
                    }
                    h4 h[kP];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        half_t t[kP];
                        pieces(v[k] * (MODE == MAKE_A ? st.A : st.B), t);
#pragma unroll
                        for (int o = 0; o < kP; ++o) h[o][k] = t[o];
                    }
#pragma unroll
                    for (int o = 0; o < kP; ++o) {
                        *reinterpret_cast<h4 *>(out + o * sp.Mp * sp.Mp + plane_at(sp.Mp, jj, ii)) = h[o];
                        if (ti != tj) *reinterpret_cast<h4 *>(out + o * sp.Mp * sp.Mp + plane_at(sp.Mp, ii + (lane & 3), jj & ~3)) = quad_turn(h[o], lane);
                    }
                } else {
                    f4 &xf = reinterpret_cast<f4 *>(base + sp.xf)[own_place<C>((int64_t)tj * a.tiles_i + ti, wave, r, c, e, lane)];
                    v = st.a * xf + st.over_Bx * v;
                    if (MODE == LAST_X) {
                        const Item &it = items.item[blockIdx.y];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int row = (int)(it.flip ? jj : ii + k), col = (int)(it.flip ? ii + k : jj);
                            if (row < it.rows && col < it.cols) give<T>(items, it, row, col, v[k]);
                        }
                    } else {
                        half_t *x = reinterpret_cast<half_t *>(base + sp.x), *t = reinterpret_cast<half_t *>(base + sp.t[1 - a.turn]);
                        h4 h[kP];
                        xf = v;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            half_t s[kP];
                            pieces(v[k] * st.next, s);
#pragma unroll
                            for (int o = 0; o < kP; ++o) h[o][k] = s[o];
                        }
#pragma unroll
                        for (int o = 0; o < kP; ++o) {
                            *reinterpret_cast<h4 *>(x + o * sp.Mp * sp.Np + plane_at(sp.Mp, ii + (lane & 3), jj & ~3)) = quad_turn(h[o], lane);
                            *reinterpret_cast<h4 *>(t + o * sp.Mp * sp.Np + plane_at(sp.Np, jj, ii)) = h[o];
                        }
                    }
                }
            }
}

// ---------------------------------------------------------------------------------- host
// The power of two that takes numbers up to `bound` to 32768 at most; 2^60 at most, so that 1 over its square is an fp32 number.
float power_below(double bound)
{
    int e = 60;
    if (bound > 0.0) {
        const int up = 15 - (int)std::ceil(std::log2(bound));
        e = up < e ? up : e;
    }
    return (float)std::ldexp(1.0, e);
}

// Largest magnitudes of b w + c w^2 and of v (a + b w + c w^2), w = v^2, for v in [0, s]: at the end or where the slope is 0.
void largest(double a, double b, double c, double s, double *of_B, double *of_x)
{
    const double end = s * s;
    const auto B = [&](double w) { return std::fabs(w * (b + c * w)); };
    const auto x = [&](double w) { return std::fabs(std::sqrt(w) * (a + w * (b + c * w))); };
    *of_B = B(end), *of_x = x(end);
    const auto look = [&](double w) { // (a NaN is nowhere)
        if (w > 0.0 && w < end) *of_B = std::fmax(*of_B, B(w)), *of_x = std::fmax(*of_x, x(w));
    };
    look(-b / (2.0 * c));
    const double d = 9.0 * b * b - 20.0 * a * c, r = std::sqrt(d); // a + 3 b w + 5 c w^2 = 0
    look((-3.0 * b + r) / (10.0 * c));
    look((-3.0 * b - r) / (10.0 * c));
    look(-a / (3.0 * b)); // c = 0
}

// Powers of two of every step, from the largest singular value that can occur: X0's is 1 at most.  false: they leave fp32's range.
bool plan_steps(const pcsr_ortho_t &how, Step *out)
{
    double s = 1.0;
    float x = power_below(s * 1.01);
    for (int k = 0; k < how.steps; ++k) {
        const double a = how.coefficients[3 * k], b = how.coefficients[3 * k + 1], c = how.coefficients[3 * k + 2];
        double most_B = 0.0, most_x = 0.0;
        largest(a, b, c, s, &most_B, &most_x);
        if (!(std::isfinite(a) && std::isfinite(b) && std::isfinite(c)) || !(most_x < 0x1p24) || !(most_B < 0x1p100)) return false;
        Step &st = out[k];
        st.a = (float)a, st.b = (float)b, st.c = (float)c;
        st.x = x;
        st.A = power_below(s * s * 1.01), st.B = power_below(most_B * 1.01);
        s = most_x * 1.001;
        st.next = x = power_below(s * 1.01);
        st.over_xx = 1.0f / st.x / st.x, st.over_AA = 1.0f / st.A / st.A, st.over_Bx = 1.0f / st.B / st.x;
    }
    return true;
}

bool is_small(const pcsr_matrix_t &m) { return m.rows <= kSmall && m.cols <= kSmall; }

// The tiling of a group of matrices: tiles of 128 where the symmetric products have half as many as there are compute units; tiles of 64
// otherwise, with two teams to a tile where a product has fewer tiles than compute units.  Five steps, us:
//                    64 (a team / two)   128
//   512 x 512            153 /  135      241
//   1024 x 1024          251 /  207      387
//   1024 x 4096          554 /  562      700
//   2048 x 2048         1029 / 1087      894
//   3000 x 3000         2464            2477
//   4096 x 4096         5593 / 6208     5073
//   8 of 512             238 /  277      293
//   16 of 300            179 /  200      264
//   4 of 1000            622 /  676      527
constexpr int64_t kUnits = 256; // compute units
bool large_tiles(int64_t m, int64_t count)
{
    const int64_t a = (m + Large::TI - 1) / Large::TI;
    return a * (a + 1) / 2 * count >= kUnits / 2;
}

// the matrices from `first` on that go with it in one launch
int64_t group_of(const pcsr_matrix_t *m, int64_t count, int64_t first, const char *done, int64_t *members)
{
    int64_t n = 0;
    const bool small = is_small(m[first]); // all small ones together: a compute unit each, side by side
    for (int64_t k = first; k < count && n < kItems; ++k) {
        if (done && done[k]) continue;
        if (small ? is_small(m[k]) : m[k].rows == m[first].rows && m[k].cols == m[first].cols) members[n++] = k;
    }
    return n;
}

int64_t group_bytes(const pcsr_matrix_t &x, int64_t n)
{
    if (is_small(x)) return 0;
    const int64_t m = x.rows < x.cols ? x.rows : x.cols, w = x.rows < x.cols ? x.cols : x.rows;
    return kItems * kNormBlocks * (int64_t)sizeof(double) + n * Space(m, w, large_tiles(m, n) ? Large::TI : Small::TI).bytes;
}

int ortho_check(const pcsr_matrix_t *m, int64_t count, const pcsr_ortho_t *how)
{
    if (count < 0 || (count && !m) || !how || !how->coefficients || how->steps < 1 || how->steps > kSteps) return PCSR_E_INVALID_ARG;
    if (how->type < PCSR_F32 || how->type > PCSR_F16) return PCSR_E_UNSUPPORTED;
    for (int64_t k = 0; k < count; ++k) {
        const pcsr_matrix_t &x = m[k];
        if (x.rows < 0 || x.cols < 0) return PCSR_E_INVALID_ARG;
        if (x.rows == 0 || x.cols == 0) continue;
        if (!x.grad || !x.out || x.grad_ld < x.cols || x.out_ld < x.cols || (x.buf && x.buf_ld < x.cols)) return PCSR_E_INVALID_ARG;
        if (x.rows > (1 << 17) || x.cols > (1 << 17) || x.rows * x.cols > int64_t(1) << 32) return PCSR_E_TOO_LARGE;
    }
    return PCSR_OK;
}

template <typename T, int Q> int run_small(const SmallArgs &a, int n, hipStream_t s)
{
    const size_t lds = 2 * sizeof(SmallPlanes<64 * Q>);
    if (!allow_lds(&small_kernel<T, Q>, lds)) return PCSR_E_HIP;
    hipLaunchKernelGGL((small_kernel<T, Q>), dim3(n), dim3(1024), lds, s, a);
    return PCSR_OK;
}

template <typename T, typename C, int MODE> bool run_product(const ProductArgs &a, const Items &q, unsigned tiles, int n, hipStream_t s)
{
    if (!allow_lds(&product_kernel<T, C, MODE>, C::lds)) return false;
    hipLaunchKernelGGL((product_kernel<T, C, MODE>), dim3(tiles, n), dim3(C::threads), C::lds, s, a, q);
    return true;
}
template <typename T, typename C> int run_large(const Items &q, int n, const Step *step, int steps, char *ws, hipStream_t s)
{
    static_assert(C::TI == C::TJ, "square tiles");
    const Item &it = q.item[0];
    const int64_t m = it.flip ? it.cols : it.rows, w = it.flip ? it.rows : it.cols;
    const Space sp(m, w, C::TI);
    double *sums = reinterpret_cast<double *>(ws);
    ws += kItems * kNormBlocks * sizeof(double);
    const int64_t want = (m * w + kT * 4 - 1) / (kT * 4);
    const int blocks = (int)(want < kNormBlocks ? want : kNormBlocks);
    hipLaunchKernelGGL((measure_kernel<T>), dim3(blocks, n), dim3(kT), 0, s, q, sums);
    hipLaunchKernelGGL((pack_kernel<T, C>), dim3((unsigned)(sp.Np / 32), (unsigned)(sp.Mp / 32), n), dim3(kT), 0, s, q, sums, blocks, ws, sp, step[0].x);
    const unsigned ti = (unsigned)(sp.Mp / C::TI), tj = (unsigned)(sp.Np / C::TJ), sym = ti * (ti + 1) / 2;
    bool ok = true;
    for (int k = 0; k < steps && ok; ++k) {
        const ProductArgs a = {ws, sp, step[k], (int)ti, k & 1};
        const auto run = [&](auto type, auto mode, unsigned tiles) {
            typedef decltype(type) U;
            constexpr int MODE = decltype(mode)::value;
            if constexpr (std::is_same<C, Small>::value) // the same tiles and places
                if ((int64_t)tiles * n <= kUnits) return run_product<U, Few, MODE>(a, q, tiles, n, s);
            return run_product<U, C, MODE>(a, q, tiles, n, s);
        };
        ok = run(float{}, std::integral_constant<int, MAKE_A>{}, sym); // (the type matters to the last alone)
        ok = ok && run(float{}, std::integral_constant<int, MAKE_B>{}, sym);
        ok = ok && (k + 1 < steps ? run(float{}, std::integral_constant<int, MAKE_X>{}, ti * tj) : run(T{}, std::integral_constant<int, LAST_X>{}, ti * tj));
    }
    return ok ? PCSR_OK : PCSR_E_HIP;
}

} // namespace
} // namespace pcsr

using namespace pcsr;

extern "C" {

int64_t pcsr_ortho_workspace(const pcsr_matrix_t *m, int64_t count, const pcsr_ortho_t *how)
{
    if (ortho_check(m, count, how) != PCSR_OK) return 0;
    int64_t most = 0, members[kItems];
    for (int64_t k = 0; k < count; ++k) {
        if (m[k].rows == 0 || m[k].cols == 0 || is_small(m[k])) continue; // they need none
        // a group that starts at any of them is no larger than all that are like it
        const int64_t n = group_of(m, count, k, nullptr, members);
        for (int64_t c = 1; c <= n; ++c) { // fewer matrices can mean smaller tiles, but never more memory than counted here
            const int64_t b = group_bytes(m[k], c);
            most = b > most ? b : most;
        }
    }
    return most;
}

int pcsr_orthogonalize(const pcsr_matrix_t *m, int64_t count, const pcsr_ortho_t *how, void *ws, void *stream)
{
    const int rc = ortho_check(m, count, how);
    if (rc != PCSR_OK) return rc;
    SmallArgs a;
    a.steps = how->steps;
    if (!plan_steps(*how, a.step)) return PCSR_E_UNSUPPORTED;
    if (!ws && pcsr_ortho_workspace(m, count, how)) return PCSR_E_INVALID_ARG;
    a.q.update = how->update, a.q.nesterov = how->nesterov, a.q.momentum = how->momentum, a.q.keep = how->keep;
    hipStream_t s = static_cast<hipStream_t>(stream);
    int64_t members[kItems];
    bool any = false;
    // matrices are taken in the order they come, each with those behind it that are like it
    const std::unique_ptr<char[]> done(new (std::nothrow) char[(size_t)count]());
    if (!done) return PCSR_E_OOM;
    for (int64_t k = 0; k < count; ++k) {
        if (done[k]) continue;
        if (m[k].rows == 0 || m[k].cols == 0) continue;
        const int64_t n = group_of(m, count, k, done.get(), members);
        int used = 0;
        bool wide = false;
        for (int64_t i = 0; i < n; ++i) {
            const pcsr_matrix_t &x = m[members[i]];
            done[members[i]] = 1;
            if (x.rows == 0 || x.cols == 0) continue;
            wide = wide || x.rows > 64 || x.cols > 64;
            a.q.item[used++] = {x.grad, x.buf, x.out, (int)x.rows, (int)x.cols, x.grad_ld, x.buf_ld, x.out_ld, x.rate, x.rows > x.cols};
        }
        const int r = for_type(how->type, [&](auto t) {
            typedef decltype(t) T;
            if (is_small(m[k])) return wide ? run_small<T, 2>(a, used, s) : run_small<T, 1>(a, used, s);
            char *at = static_cast<char *>(ws);
            const bool large = large_tiles(m[k].rows < m[k].cols ? m[k].rows : m[k].cols, used);
            return large ? run_large<T, Large>(a.q, used, a.step, a.steps, at, s) : run_large<T, Small>(a.q, used, a.step, a.steps, at, s);
        });
        if (r != PCSR_OK) return r;
        any = true;
    }
    return any ? launched() : PCSR_OK;
}

} // extern "C"
