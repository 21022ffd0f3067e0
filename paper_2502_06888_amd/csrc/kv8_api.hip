// C ABI of the 8-bit key-value cache (include/moe_kv8.h): argument checks, then the launches.  No state but the
// error text of each thread.
#include <cmath>

#include "call_checks.h"
#include "kv8_kernels.h"

using namespace kkv8;
using namespace kcall;

namespace {

thread_local CallError g_error;
constexpr double kLog2e = 1.4426950408889634;

#define fail g_error.fail  // the text goes to this thread's buffer

moe_status check_sizes(const moe_kv8_cache* c) {
    if (!c) return fail(MOE_ERR_INVALID_ARG, "cache is null");
    if (c->n_seq < 1 || c->n_seq > 65536) return fail(MOE_ERR_SHAPE, "n_seq %d outside 1..65536", c->n_seq);
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return fail(MOE_ERR_SHAPE, "n_kv_heads %d outside 1..1024", c->n_kv_heads);
    if ((int64_t)c->n_seq * c->n_kv_heads > (1 << 20)) return fail(MOE_ERR_SHAPE, "n_seq * n_kv_heads is over 2^20");
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return fail(MOE_ERR_SHAPE, "head_dim must be 32, 64 or 128");
    if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return fail(MOE_ERR_SHAPE, "block must be 16, 32, 64 or 128");
    if (c->max_len < 1 || c->max_len > (1 << 20) || c->max_len % c->block != 0) return fail(MOE_ERR_SHAPE, "max_len must be a multiple of block in 1..2^20");
    if (c->reserved != 0) return fail(MOE_ERR_INVALID_ARG, "cache.reserved must be 0");
    return MOE_OK;
}

moe_status check_step_sizes(const moe_kv8_cache* c, const moe_kv8_step* s) {
    if (!s) return fail(MOE_ERR_INVALID_ARG, "step is null");
    if (s->reserved != 0) return fail(MOE_ERR_INVALID_ARG, "step.reserved must be 0");
    if (s->n_rows < 0 || s->n_rows > (1 << 20)) return fail(MOE_ERR_SHAPE, "n_rows %d outside 0..2^20", s->n_rows);
    if (s->max_new < 0 || s->max_new > c->max_len) return fail(MOE_ERR_INVALID_ARG, "max_new %d outside 0..max_len", s->max_new);
    if (s->max_cached < 0 || s->max_cached > c->max_len) return fail(MOE_ERR_INVALID_ARG, "max_cached %d outside 0..max_len", s->max_cached);
    if (s->row_offsets == nullptr && (int64_t)c->n_seq * s->max_new != s->n_rows)
        return fail(MOE_ERR_INVALID_ARG, "without row_offsets n_rows must be n_seq * max_new");
    if ((s->max_new == 0) != (s->n_rows == 0)) return fail(MOE_ERR_INVALID_ARG, "n_rows %d with max_new %d", s->n_rows, s->max_new);
    return MOE_OK;
}

moe_status check_heads(const moe_kv8_cache* c, int n_q_heads) {
    if (n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0 || n_q_heads / c->n_kv_heads > 8)
        return fail(MOE_ERR_SHAPE, "n_q_heads must be a multiple of n_kv_heads, at most 8 times it");
    return MOE_OK;
}

moe_status check_cache(const moe_kv8_cache* c, Where* w) {
    TRY(w->on(c->k, "cache.k", 16));
    TRY(w->on(c->v, "cache.v", 16));
    TRY(w->on(c->k_scale, "cache.k_scale", 4));
    TRY(w->on(c->v_scale, "cache.v_scale", 4));
    if (c->position) TRY(w->on(c->position, "cache.position", 4));
    return MOE_OK;
}

moe_status check_step(const moe_kv8_step* s, Where* w) {
    if (s->row_offsets) TRY(w->on(s->row_offsets, "step.row_offsets", 4));
    TRY(w->on(s->cached, "step.cached", 4));
    if (s->next_position) TRY(w->on(s->next_position, "step.next_position", 4));
    return MOE_OK;
}

moe_status check_rows(const void* p, const char* name, int64_t row, int64_t head, Where* w) {
    TRY(w->on(p, name, 16));
    if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0) return fail(MOE_ERR_INVALID_ARG, "strides of %s must be multiples of 8", name);
    return MOE_OK;
}

moe_status check_workspace(const void* ws, int64_t bytes, int64_t need, Where* w) {
    if (need == 0) return MOE_OK;
    if (bytes < need) return fail(MOE_ERR_OOM, "workspace of %lld bytes, need %lld", (long long)bytes, (long long)need);
    return w->on(ws, "workspace", 256);
}

Cache cache_of(const moe_kv8_cache* c) {
    Cache k{};
    k.n_seq = c->n_seq;
    k.Hkv = c->n_kv_heads;
    k.hd = c->head_dim;
    k.max_len = c->max_len;
    k.logb = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
    k.codes[0] = (uint8_t*)c->k;
    k.codes[1] = (uint8_t*)c->v;
    k.scale[0] = c->k_scale;
    k.scale[1] = c->v_scale;
    k.position = c->position;
    return k;
}

// No sequence brings more than all rows there are: a bound beyond that sizes no launch.
Step step_of(const moe_kv8_step* s) {
    return Step{s->n_rows, s->max_new < s->n_rows ? s->max_new : s->n_rows, s->max_cached, s->row_offsets, s->cached, s->next_position};
}

// Everything that moe_kv8_append refuses; *device: where the tensors are.
moe_status check_append(const moe_kv8_cache* cache, const moe_kv8_step* step, const void* k_new, const void* v_new,
                        int64_t row_stride, int64_t head_stride, int* device) {
    TRY(check_sizes(cache));
    TRY(check_step_sizes(cache, step));
    Where w{&g_error};
    TRY(check_cache(cache, &w));
    TRY(check_step(step, &w));
    *device = w.device;
    if (step->n_rows == 0) return MOE_OK;
    TRY(check_rows(k_new, "k_new", row_stride, head_stride, &w));
    TRY(check_rows(v_new, "v_new", row_stride, head_stride, &w));
    if (!append_fits(cache_of(cache), step_of(step))) return fail(MOE_ERR_SHAPE, "too many workgroups: bring fewer sequences or tokens at once");
    return MOE_OK;
}

moe_status check_attend(const moe_kv8_cache* cache, const moe_kv8_step* step, int32_t n_q_heads, const void* q,
                        int64_t q_row_stride, int64_t q_head_stride, float softmax_scale, const void* out,
                        int64_t out_row_stride, int64_t out_head_stride, const float* weight_in, const float* weight_out,
                        const void* workspace, int64_t workspace_bytes, int* device) {
    TRY(check_sizes(cache));
    TRY(check_step_sizes(cache, step));
    TRY(check_heads(cache, n_q_heads));
    if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale * (float)kLog2e))
        return fail(MOE_ERR_INVALID_ARG, "softmax_scale must be finite, times log2(e) too, and not negative");
    if (step->n_rows > 0 && pieces_overlap(step->n_rows, n_q_heads, out_row_stride, out_head_stride, cache->head_dim))
        return fail(MOE_ERR_INVALID_ARG, "rows or heads of out overlap");
    Where w{&g_error};
    TRY(check_cache(cache, &w));
    TRY(check_step(step, &w));
    *device = w.device;
    if (step->n_rows > 0) {
        TRY(check_rows(q, "q", q_row_stride, q_head_stride, &w));
        TRY(check_rows(out, "out", out_row_stride, out_head_stride, &w));
        if (q == out && (weight_out || q_row_stride != out_row_stride || q_head_stride != out_head_stride))
            return fail(MOE_ERR_INVALID_ARG, "out may be q only without weight_out and with the same strides");
    }
    if (weight_in && !weight_out) return fail(MOE_ERR_INVALID_ARG, "weight_in without weight_out");
    if (weight_out) TRY(w.on(weight_out, "weight_out", 4));
    if (weight_in && weight_in != weight_out) TRY(w.on(weight_in, "weight_in", 4));
    const Cache c = cache_of(cache);
    const Step s = step_of(step);
    if (!attend_fits(c, s, n_q_heads, weight_out != nullptr)) return fail(MOE_ERR_SHAPE, "too many workgroups: bring fewer sequences or tokens at once");
    return check_workspace(workspace, workspace_bytes, attend_workspace(c, s, n_q_heads, weight_out != nullptr), &w);
}

moe_status launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MOE_OK : fail(MOE_ERR_HIP, "launch failed: %s", hipGetErrorString(e));
}

}  // namespace

namespace kkv8 {

moe_status check_layer_call(const moe_kv8_cache* cache, const moe_kv8_step* step, int n_q_heads, const void* rows,
                            const float* weight_in, const float* weight_out, const void* workspace, int64_t workspace_bytes) {
    int device = 0;
    TRY(check_append(cache, step, rows, rows, 8, 8, &device));
    return check_attend(cache, step, n_q_heads, rows, 8, 8, 0.f, (const uint8_t*)rows + 16, (int64_t)n_q_heads * cache->head_dim,
                        cache->head_dim, weight_in, weight_out, workspace, workspace_bytes, &device);
}

Cache cache_of_call(const moe_kv8_cache* c) { return cache_of(c); }
Step step_of_call(const moe_kv8_step* s) { return step_of(s); }

}  // namespace kkv8

extern "C" {

const char* moe_kv8_last_error(void) { return g_error.text; }

moe_status moe_kv8_append(void* stream, const moe_kv8_cache* cache, const moe_kv8_step* step, const void* k_new,
                          const void* v_new, int64_t row_stride, int64_t head_stride) {
    int device = 0;
    TRY(check_append(cache, step, k_new, v_new, row_stride, head_stride, &device));
    if (step->n_rows == 0) return MOE_OK;
    OnDevice on(device);
    if (on.failed()) return fail(MOE_ERR_HIP, "device %d cannot be made current", device);
    launch_append((hipStream_t)stream, cache_of(cache), step_of(step), Rows{(const uint16_t*)k_new, row_stride, head_stride},
                  Rows{(const uint16_t*)v_new, row_stride, head_stride});
    return launched();
}

moe_status moe_kv8_attend_workspace_bytes(const moe_kv8_cache* cache, const moe_kv8_step* step, int32_t n_q_heads,
                                          int32_t with_weights, int64_t* bytes_out) {
    if (!bytes_out) return fail(MOE_ERR_INVALID_ARG, "bytes_out is null");
    TRY(check_sizes(cache));
    TRY(check_step_sizes(cache, step));
    TRY(check_heads(cache, n_q_heads));
    if (!attend_fits(cache_of(cache), step_of(step), n_q_heads, with_weights != 0)) return fail(MOE_ERR_SHAPE, "too many workgroups: bring fewer sequences or tokens at once");
    *bytes_out = attend_workspace(cache_of(cache), step_of(step), n_q_heads, with_weights != 0);
    return MOE_OK;
}

moe_status moe_kv8_attend(void* stream, const moe_kv8_cache* cache, const moe_kv8_step* step, int32_t n_q_heads,
                          const void* q, int64_t q_row_stride, int64_t q_head_stride, float softmax_scale, void* out,
                          int64_t out_row_stride, int64_t out_head_stride, const float* weight_in,
                          float* weight_out, void* workspace, int64_t workspace_bytes) {
    int device = 0;
    TRY(check_attend(cache, step, n_q_heads, q, q_row_stride, q_head_stride, softmax_scale, out, out_row_stride,
                     out_head_stride, weight_in, weight_out, workspace, workspace_bytes, &device));
    if (step->n_rows == 0 && !weight_out) return MOE_OK;
    OnDevice on(device);
    if (on.failed()) return fail(MOE_ERR_HIP, "device %d cannot be made current", device);
    const Cache c = cache_of(cache);
    const Step s = step_of(step);
    Attend a{};
    a.Hq = n_q_heads;
    a.qscale = (float)(kLog2e * (softmax_scale == 0.f ? 1.0 / std::sqrt((double)c.hd) : (double)softmax_scale));
    a.q = Rows{(const uint16_t*)q, q_row_stride, q_head_stride};
    a.out = RowsOut{(uint16_t*)out, out_row_stride, out_head_stride};
    a.weight_in = weight_in;
    a.weight_out = weight_out;
    a.ws = (uint8_t*)workspace;
    launch_attend((hipStream_t)stream, c, s, a);
    return launched();
}

static moe_status check_keep(const moe_kv8_cache* c, int keep) {
    if (keep < 1 || keep > c->max_len || keep % c->block != 0) return fail(MOE_ERR_INVALID_ARG, "keep must be a multiple of block in 1..max_len");
    return MOE_OK;
}

moe_status moe_kv8_evict_workspace_bytes(const moe_kv8_cache* cache, int32_t keep, int64_t* bytes_out) {
    if (!bytes_out) return fail(MOE_ERR_INVALID_ARG, "bytes_out is null");
    TRY(check_sizes(cache));
    TRY(check_keep(cache, keep));
    if (!evict_fits(cache_of(cache), keep)) return fail(MOE_ERR_SHAPE, "too many workgroups: evict from fewer sequences at once");
    *bytes_out = evict_workspace(cache_of(cache), keep);
    return MOE_OK;
}

moe_status moe_kv8_evict(void* stream, const moe_kv8_cache* cache, const int32_t* held, int32_t max_held, int32_t keep,
                         int32_t recent, const int32_t* next_position, const float* weight_in, float* weight_out,
                         int32_t* position_out, int32_t* kept, void* workspace, int64_t workspace_bytes) {
    TRY(check_sizes(cache));
    TRY(check_keep(cache, keep));
    if (recent < 0 || recent > keep) return fail(MOE_ERR_INVALID_ARG, "recent %d outside 0..keep", recent);
    if (max_held < 0 || max_held > cache->max_len) return fail(MOE_ERR_INVALID_ARG, "max_held %d outside 0..max_len", max_held);
    if (!cache->position) return fail(MOE_ERR_INVALID_ARG, "eviction needs cache.position");
    Where w{&g_error};
    TRY(check_cache(cache, &w));
    TRY(w.on(held, "held", 4));
    if (next_position) TRY(w.on(next_position, "next_position", 4));
    TRY(w.on(weight_in, "weight_in", 4));
    TRY(w.on(weight_out, "weight_out", 4));
    if (position_out) TRY(w.on(position_out, "position_out", 4));
    if (kept) TRY(w.on(kept, "kept", 4));
    const Cache c = cache_of(cache);
    if (!evict_fits(c, keep)) return fail(MOE_ERR_SHAPE, "too many workgroups: evict from fewer sequences at once");
    TRY(check_workspace(workspace, workspace_bytes, evict_workspace(c, keep), &w));
    OnDevice on(w.device);
    if (on.failed()) return fail(MOE_ERR_HIP, "device %d cannot be made current", w.device);
    launch_evict((hipStream_t)stream, c, held, max_held, keep, recent, next_position, weight_in, weight_out,
                 position_out ? position_out : c.position, kept, (uint8_t*)workspace);
    return launched();
}

}  // extern "C"
