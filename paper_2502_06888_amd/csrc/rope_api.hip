// C ABI of rotary positions (include/moe_rope.h): argument checks, then the launch.
#include "rope.h"

using namespace krope;
using namespace kcall;

namespace {

thread_local CallError g_error;

#define fail g_error.fail  // the text goes to this thread's buffer

moe_status check_rows(const moe_rope_rows* x, const char* name, int n_rows, int head_dim, unsigned size, Where* w) {
    if (x->reserved != 0) return fail(MOE_ERR_INVALID_ARG, "%s.reserved must be 0", name);
    if (x->n_heads < 0 || x->n_heads > 1024) return fail(MOE_ERR_SHAPE, "%s.n_heads %d outside 0..1024", name, x->n_heads);
    if (x->n_heads == 0 || n_rows == 0) return MOE_OK;
    if (x->in_row < 0 || x->in_head < 0 || x->out_row < 0 || x->out_head < 0) return fail(MOE_ERR_INVALID_ARG, "strides of %s are negative", name);
    if (pieces_overlap(n_rows, x->n_heads, x->out_row, x->out_head, head_dim)) return fail(MOE_ERR_INVALID_ARG, "rows or heads of %s.out overlap", name);
    if (x->in == x->out && (x->in_row != x->out_row || x->in_head != x->out_head))
        return fail(MOE_ERR_INVALID_ARG, "%s.out may be in only with the same strides", name);
    TRY(w->on(x->in, name, size));
    return w->on(x->out, name, size);
}

Rows rows_of(const moe_rope_rows* x) {
    if (!x) return Rows{};
    return Rows{x->in, x->out, x->n_heads, x->in_row, x->in_head, x->out_row, x->out_head};
}

}  // namespace

extern "C" {

const char* moe_rope_last_error(void) { return g_error.text; }

moe_status moe_rope_rotate(void* stream, const moe_rope_config* cfg, int32_t dtype, int32_t n_rows, int32_t head_dim,
                           const int32_t* positions, const moe_rope_rows* q, const moe_rope_rows* k) {
    TRY(check_config(cfg, g_error));
    if (dtype != MOE_F32 && dtype != MOE_BF16) return fail(MOE_ERR_INVALID_ARG, "dtype %d", dtype);
    if (n_rows < 0 || n_rows > (1 << 24)) return fail(MOE_ERR_SHAPE, "n_rows %d outside 0..2^24", n_rows);
    if (head_dim < 2 || head_dim > 1024) return fail(MOE_ERR_SHAPE, "head_dim %d outside 2..1024", head_dim);
    if (cfg->first > head_dim - cfg->rot_dim) return fail(MOE_ERR_SHAPE, "first + rot_dim is over head_dim");
    if (!q) return fail(MOE_ERR_INVALID_ARG, "q is null");
    const unsigned size = dtype == MOE_F32 ? 4 : 2;
    Where w{&g_error};
    if (k && k->n_heads > 0 && q->n_heads > 0 && n_rows > 0 && (q->out == k->out || q->out == k->in || k->out == q->in))
        return fail(MOE_ERR_INVALID_ARG, "q and k are written to the same memory, or one over the other's input");
    TRY(check_rows(q, "q", n_rows, head_dim, size, &w));
    if (k) TRY(check_rows(k, "k", n_rows, head_dim, size, &w));
    if (n_rows == 0 || (q->n_heads == 0 && (!k || k->n_heads == 0))) return MOE_OK;
    TRY(w.on(positions, "positions", 4));
    OnDevice on(w.device);
    if (on.failed()) return fail(MOE_ERR_HIP, "device %d cannot be made current", w.device);
    Rotate r{turns_of(*cfg), {rows_of(q), rows_of(k)}, n_rows, head_dim, cfg->rot_dim, cfg->first, cfg->interleaved, positions};
    launch_rotate((hipStream_t)stream, r, dtype == MOE_F32);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MOE_OK : fail(MOE_ERR_HIP, "launch failed: %s", hipGetErrorString(e));
}

}  // extern "C"
