// What a training step needs around the graph layers (internal to the package: embedding.py, norm.py and muon.py call
// these through ctypes): a table of node features and its gradient, group norm with an activation over rows of
// channels, updates of weight matrices orthogonalised by Newton-Schulz products.
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
}
