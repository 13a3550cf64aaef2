// Linear layers of any width with what follows them: the entry points (see pcsr_train.h; pcsr_linear_kernels.h has the kernels).
#include "pcsr_linear.h"

namespace pcsr {
namespace {

constexpr int64_t up(int64_t n, int64_t by) { return (n + by - 1) / by; }
constexpr int64_t kMostTiles = int64_t(1) << 23;

int check(const pcsr_linear_t *a)
{
    if (!a || a->rows < 0 || a->in < 0 || a->out < 1 || !(a->drop.p >= 0.0 && a->drop.p <= 1.0)) return PCSR_E_INVALID_ARG;
    if (a->type < PCSR_F32 || a->type > PCSR_F16 || a->act < PCSR_ACT_NONE || a->act > PCSR_ACT_GELU) return PCSR_E_UNSUPPORTED;
    if (a->bias_type != PCSR_F32 && a->bias_type != a->type) return PCSR_E_UNSUPPORTED;
    const int64_t wide = int64_t(1) << 24;
    if (a->rows >= int64_t(1) << 32 || a->in >= wide || a->out >= wide) return PCSR_E_TOO_LARGE;
    for (const int64_t t : {up(a->rows, 64) * up(a->out, 64), up(a->rows, 64) * up(a->in, 64), up(a->out, 64) * up(a->in, 64)})
        if (t > kMostTiles) return PCSR_E_TOO_LARGE;
    if (a->rows > 0 && a->in > 0 && (a->x_stride < a->in || a->w_stride < a->in)) return PCSR_E_INVALID_ARG;
    return PCSR_OK;
}

} // namespace
} // namespace pcsr

using namespace pcsr;

extern "C" {

int64_t pcsr_linear_workspace(const pcsr_linear_t *a, int32_t backward)
{
    if (check(a) != PCSR_OK || a->rows == 0) return 0;
    int64_t need = 0;
    for_type(a->type, [&](auto t) {
        need = LinearOf<decltype(t)>::workspace(*a, backward != 0);
        return 0;
    });
    return need;
}

int pcsr_linear(const pcsr_linear_t *a, void *y, void *slope, void *ws, void *stream)
{
    if (const int rc = check(a)) return rc;
    if (a->rows == 0) return PCSR_OK;
    if (!y || (a->in > 0 && (!a->x || !a->w)) || (a->residual && a->r_stride < a->out)) return PCSR_E_INVALID_ARG;
    if (!ws && pcsr_linear_workspace(a, 0)) return PCSR_E_INVALID_ARG;
    return for_type(a->type, [&](auto t) { return LinearOf<decltype(t)>::forward(*a, y, slope, ws, (hipStream_t)stream); });
}

int pcsr_linear_backward(const pcsr_linear_t *a, const void *slope, const void *dy, int64_t dy_stride, void *dx, void *dw, void *db, void *ws,
                         void *stream)
{
    if (const int rc = check(a)) return rc;
    if (a->rows == 0 || (!dx && !dw && !db)) return PCSR_OK;
    if (!dy || dy_stride < a->out || (a->act != PCSR_ACT_NONE && !slope) || (dx && !a->w) || (dw && !a->x) || !ws) return PCSR_E_INVALID_ARG;
    return for_type(a->type, [&](auto t) { return LinearOf<decltype(t)>::backward(*a, slope, dy, dy_stride, dx, dw, db, ws, (hipStream_t)stream); });
}

int pcsr_linear_uses(const pcsr_linear_t *a, const void *dy, int64_t dy_stride, int64_t *ends)
{
    if (const int rc = check(a)) return rc;
    if (a->rows == 0 || dy_stride < a->out || !ends) return PCSR_E_INVALID_ARG;
    return for_type(a->type, [&](auto t) {
        LinearOf<decltype(t)>::uses(*a, dy, dy_stride, *reinterpret_cast<int64_t (*)[4][2]>(ends));
        return (int)PCSR_OK;
    });
}
}
