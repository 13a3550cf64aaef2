// What a training step needs around the graph layers (internal to the package: embedding.py, norm.py, muon.py, dropout.py and
// linear.py call these through ctypes): a table of node features and its gradient, group norm with an activation over rows of
// channels, updates of weight matrices orthogonalised by Newton-Schulz products, dropout, linear layers of any width with what follows them.
//
// All arrays are device memory unless a host array is named; nothing is allocated here and the stream is not waited for.
// Kernels go to the device that is current, which has to be that of the stream and the arrays.
#pragma once
#include <cstdint>

#include "../../include/pcsr.h"

extern "C" {

// type of the numbers of an array; sums are 32 bits at least whatever it is
enum { PCSR_F32 = 0, PCSR_BF16 = 1, PCSR_F16 = 2 };

// ---------------------------------------------------------------------------------- embedding (pcsr_embed.hip)
// out[n x d] = scale * table[ids[i]], rounded once.  ids int32 (wide 0) or int64 (wide 1); an id outside [0, rows) stands
// for no row and gives zeros.  Rows of the table are `stride` numbers apart, those of out d.
int pcsr_embed(int64_t n, int64_t rows, int64_t d, int32_t type, const void *ids, int32_t wide, const void *table,
               int64_t stride, float scale, void *out, void *stream);
// grad[rows x d] = scale * the sum of dout[i] over the i with ids[i] = row, in 32 bits in an order that the ids, n, rows, d and the
// type alone decide, rounded once; zeros for rows without an id.  Rows of dout are `stride` numbers apart.
// TOO_LARGE: n of 2^31 - 1024 and more, rows of 2^31, d above 2^23, stride above 2^31.
// ws: pcsr_embed_workspace bytes (0 for few ids), 16-byte aligned.
int64_t pcsr_embed_workspace(int64_t n, int64_t rows, int64_t d);
int pcsr_embed_backward(int64_t n, int64_t rows, int64_t d, int32_t type, const void *ids, int32_t wide,
                        const void *dout, int64_t stride, float scale, void *grad, void *ws, void *stream);

// ---------------------------------------------------------------------------------- group norm (pcsr_norm.hip)
enum { PCSR_ACT_NONE = 0, PCSR_ACT_RELU = 1, PCSR_ACT_SILU = 2, PCSR_ACT_GELU = 3 };

// Rows of channels, channels last, in graphs: graph s has the rows from offsets[s] to offsets[s + 1].  In a group of
// channels / groups channels over the rows of its graph: xhat = (x - mean) / sqrt(variance + eps), y = act(xhat * weight +
// bias).
typedef struct {
    int64_t rows, channels, groups;
    int64_t graphs;
    const void *offsets; // device, int32 or int64[graphs + 1], ascending from 0 to rows; null: graphs of rows / graphs each
    int32_t wide;        // 1: offsets are int64
    int32_t type;        // of x, y and their gradients
    int32_t param_type;  // of weight and bias and their gradients
    int32_t act;
    const void *x;       // [rows x channels], rows x_stride numbers apart
    int64_t x_stride;
    const void *weight, *bias; // [channels], null: 1 and 0
    float eps;
    float *mean, *rstd;  // [graphs x groups]: written by the forward call, read by the backward one
} pcsr_norm_t;

// bytes of workspace (16-byte aligned) of the calls below
int64_t pcsr_norm_workspace(const pcsr_norm_t *a, int32_t backward);
// y: [rows x channels].  UNSUPPORTED for groups of more than 2048 (fp32) or 4096 channels.  TOO_LARGE: channels above 2^22, strides above 2^31,
// and more graphs than a launch has teams for: 2^26, but where a graph takes a workgroup (more than 8 KB a graph on the average, or groups of
// more than 64 pieces of 16 bytes) 2^24, and of groups above 256 pieces 2^23.
int pcsr_norm(const pcsr_norm_t *a, void *y, void *ws, void *stream);
// From dy (rows dy_stride numbers apart): dx [rows x channels], dweight and dbias [channels]; each may be null.
int pcsr_norm_backward(const pcsr_norm_t *a, const void *dy, int64_t dy_stride, void *dx, void *dweight, void *dbias, void *ws,
                       void *stream);

// ---------------------------------------------------------------------------------- orthogonalised updates (pcsr_ortho.hip)
// One matrix.  Update U = grad, or with momentum: buf = momentum * buf + grad, U = grad + momentum * buf (nesterov) or buf.
// O = `steps` times X <- a X + (b A + c A A) X, A = X X^T, from X = U / ||U|| (Frobenius; zeros stay zeros).
// out = O, or with `update`: out = keep * out - rate * O.  grad and out have `type`, buf is fp32.
typedef struct {
    const void *grad;
    float *buf;         // null: no momentum
    void *out;
    int64_t rows, cols;
    int64_t grad_ld, buf_ld, out_ld; // distance of rows
    float rate;
    int32_t reserved;
} pcsr_matrix_t;
typedef struct {
    int32_t type, steps; // steps 1 to PCSR_ORTHO_STEPS
    const double *coefficients; // host, [steps][3]
    int32_t update, nesterov;
    float momentum, keep;
} pcsr_ortho_t;
#define PCSR_ORTHO_STEPS 16
// matrices: host, [count], which may overlap with no other's buf or out.  Products of fp16 numbers added up in fp32: operands are two fp16
// numbers each (22 bits).
// ws: 16-byte aligned, pcsr_ortho_workspace bytes.  UNSUPPORTED where the coefficients let the numbers grow out of fp32's range; TOO_LARGE: sides
// above 2^17, matrices of more than 2^32 numbers.
int64_t pcsr_ortho_workspace(const pcsr_matrix_t *matrices, int64_t count, const pcsr_ortho_t *how);
int pcsr_orthogonalize(const pcsr_matrix_t *matrices, int64_t count, const pcsr_ortho_t *how, void *ws, void *stream);

// ---------------------------------------------------------------------------------- dropout (pcsr_drop.hip)
// What is dropped is a function of seed, offset, row and column (pcsr_drop.h).  p: in [0, 1], rounded to a multiple of 2^-16.
typedef struct {
    double p;
    uint64_t seed, offset;
    const int64_t *state; // device, null or {seed, offset}: read by the kernels when they run, in place of the two above
    int64_t *used;        // device, null or [2]: seed and offset that were used (p > 0)
} pcsr_drop_t;
// out[rows x cols] = residual + x with numbers dropped and the others multiplied by 1 / (1 - p), in fp32, rounded once.  residual: null for
// none.  Rows of x are x_stride, of residual r_stride numbers apart, those of out cols.  out may be x or residual where their rows lie as its own do.
// TOO_LARGE: rows of 2^32 and more, columns of 2^31.
int pcsr_dropout(int64_t rows, int64_t cols, int32_t type, const void *x, int64_t x_stride, const void *residual, int64_t r_stride,
                 const pcsr_drop_t *how, void *out, void *stream);

// ---------------------------------------------------------------------------------- linear layers (pcsr_linear.hip)
// y = residual + dropout(act(x w^T + bias)): x [rows x in], w [out x in], y and residual [rows x out], one type; bias [out] of
// that type or fp32, null for none; residual null for none.  Products of 16-bit numbers are exact and summed in fp32; those of
// fp32 numbers are taken of three bf16 numbers each (24 bits).  Everything behind the product is fp32, rounded once.
typedef struct {
    int64_t rows, in, out;
    int32_t type, bias_type, act, reserved;
    const void *x, *w, *bias, *residual;
    int64_t x_stride, w_stride, r_stride;
    pcsr_drop_t drop;
} pcsr_linear_t;
// bytes of workspace (16-byte aligned) of the calls below with the same a; backward: those for all of its results
int64_t pcsr_linear_workspace(const pcsr_linear_t *a, int32_t backward);
// slope: null, or [rows x out] for the backward call where act is not none: the activation's slopes, fp32 for fp32 and otherwise
// 16 bits, 2^15 (slope + 1/4) (0: not a number), or, from 45312 on, of slopes between -2^-6 and -2^-45 (their bits as fp32 - 0xA9000000) / 2^14 + 45312, each rounded.
// TOO_LARGE: rows of 2^32 and more, in or out of 2^24 and more, and more than 2^23 tiles of 64 x 64 of y, of dx or of dw.
int pcsr_linear(const pcsr_linear_t *a, void *y, void *slope, void *ws, void *stream);
// From dy (rows dy_stride numbers apart): dx [rows x in], dw [out x in], db [out] of bias_type; each may be null (rows of 0: nothing is written).  a->bias and a->residual are not read; a->x is for
// dw alone, a->w for dx.
int pcsr_linear_backward(const pcsr_linear_t *a, const void *slope, const void *dy, int64_t dy_stride, void *dx, void *dw, void *db, void *ws,
                         void *stream);
// Where a backward call that is asked for all of its results writes its workspace, the host's arithmetic alone: first and last byte (exclusive) of dz, of sums of its columns, of
// what the products of dx and of dw write: ends[4][2].  dy: its address, which is not read.
int pcsr_linear_uses(const pcsr_linear_t *a, const void *dy, int64_t dy_stride, int64_t *ends);
}
