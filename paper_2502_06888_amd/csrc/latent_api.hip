// C ABI of the latent cache (include/moe_latent.h): argument checks, then the launches.  No state but the error text of each
// thread.
#include <cmath>

#include "call_checks.h"
#include "latent_kernels.h"

using namespace klat;
using namespace kcall;

namespace {

thread_local CallError g_error;
constexpr double kLog2e = 1.4426950408889634;

#define fail g_error.fail  // the text goes to this thread's buffer

moe_status check_sizes(const moe_latent_cache* c) {
    if (!c) return fail(MOE_ERR_INVALID_ARG, "cache is null");
    if (c->n_seq < 1 || c->n_seq > 65536) return fail(MOE_ERR_SHAPE, "n_seq %d outside 1..65536", c->n_seq);
    if (c->latent_dim != 128 && c->latent_dim != 256 && c->latent_dim != 512) return fail(MOE_ERR_SHAPE, "latent_dim must be 128, 256 or 512");
    if (c->rope_dim != 32 && c->rope_dim != 64) return fail(MOE_ERR_SHAPE, "rope_dim must be 32 or 64");
    if (c->max_len < 1 || c->max_len > (1 << 20)) return fail(MOE_ERR_SHAPE, "max_len %d outside 1..2^20", c->max_len);
    if (c->prefix_len < 0 || c->prefix_len > (1 << 20)) return fail(MOE_ERR_SHAPE, "prefix_len %d outside 0..2^20", c->prefix_len);
    if (c->reserved != 0) return fail(MOE_ERR_INVALID_ARG, "cache.reserved must be 0");
    return MOE_OK;
}

moe_status check_step_sizes(const moe_latent_cache* c, const moe_kv8_step* s) {
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

bool part_of_head(int n) { return n == 32 || n == 64 || n == 128; }

moe_status check_head_sizes(const moe_latent_cache* c, const moe_latent_heads* h) {
    if (!h) return fail(MOE_ERR_INVALID_ARG, "heads is null");
    if (h->reserved != 0) return fail(MOE_ERR_INVALID_ARG, "heads.reserved must be 0");
    if (h->n_heads < 1 || h->n_heads > 256) return fail(MOE_ERR_SHAPE, "n_heads %d outside 1..256", h->n_heads);
    if (!part_of_head(h->nope_dim)) return fail(MOE_ERR_SHAPE, "nope_dim must be 32, 64 or 128");
    if (!part_of_head(h->v_dim)) return fail(MOE_ERR_SHAPE, "v_dim must be 32, 64 or 128");
    for (int64_t stride : {h->w_k_head, h->w_v_head})
        if (stride < 0 || stride % 8 != 0) return fail(MOE_ERR_INVALID_ARG, "strides of w_k and w_v must be multiples of 8, not negative");
    return MOE_OK;
}

moe_status check_form(int32_t form) {
    if (form < MOE_LATENT_AUTO || form > MOE_LATENT_EXPANDED) return fail(MOE_ERR_INVALID_ARG, "form %d", form);
    return MOE_OK;
}

moe_status check_cache(const moe_latent_cache* c, Where* w) {
    TRY(w->on(c->rows, "cache.rows", 16));
    if (c->prefix_len > 0) TRY(w->on(c->prefix, "cache.prefix", 16));
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
    if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0) return fail(MOE_ERR_INVALID_ARG, "strides of %s must be multiples of 8, not negative", name);
    return MOE_OK;
}

Cache cache_of(const moe_latent_cache* c) {
    return Cache{c->n_seq, c->latent_dim, c->rope_dim, c->max_len, c->prefix_len, (uint16_t*)c->rows, (const uint16_t*)c->prefix};
}

// No sequence brings more than all rows there are: a bound beyond that sizes no launch.
Step step_of(const moe_kv8_step* s) {
    return Step{s->n_rows, s->max_new < s->n_rows ? s->max_new : s->n_rows, s->max_cached, s->row_offsets, s->cached, s->next_position};
}

Heads heads_of(const moe_latent_cache* c, const moe_latent_heads* h) {
    return Heads{h->n_heads, h->nope_dim, h->v_dim, (const uint16_t*)h->w_k, (const uint16_t*)h->w_v,
                 h->w_k_head ? h->w_k_head : (int64_t)h->nope_dim * c->latent_dim, h->w_v_head ? h->w_v_head : (int64_t)h->v_dim * c->latent_dim};
}

// Whether a step is better run expanded: by what either form takes in microseconds, from the step's bounds.  Both: launches, and steps over
// slots that one wavefront takes one after the other; about half as long at the smallest sizes of a head.  Expanded: keys and values of every
// slot (of 128 at a time) at 550 TFLOP/s, attention at 500.  Absorbed: attention at 800, and each row's way into the latent space and out of it, with its share of
// a workgroup's start and end, at 3 TB/s.  Measured, absorbed / expanded, 32 heads: 1 token behind 700 slots 26 / 46 us; 8 prompts of 128 tokens 102 / 35; 64 tokens behind
// 4000 slots 67 / 79, 128 tokens 94 / 90; 64 sequences of 64 tokens behind 500 slots 595 / 612, of 128 1211 / 769; behind a prefix of 4000
// slots and 100 of their own 64 sequences of 4 tokens 149 / 196, of 16 474 / 272.  Of 354 steps between, 9 took a form that is more than
// 10 % slower than the other, by 40 % at most.
bool expands(const Cache& c, const Step& s, const Heads& h, int form) {
    if (form != MOE_LATENT_AUTO) return form == MOE_LATENT_EXPANDED;
    if (s.n_rows == 0) return false;
    const double most = (double)(s.max_cached + s.max_new < c.max_len ? s.max_cached + s.max_new : c.max_len), heads = h.n, rows = s.n_rows;
    const double pairs = rows * (c.prefix_len + most - 0.5 * s.max_new) * heads, slots = c.prefix_len + c.n_seq * std::ceil(most / 128) * 128;
    const double sizes = 0.5 + c.latent / 1024., in_turn = most + c.prefix_len;
    const double expanded = sizes * (20 + 0.028 * std::fmin(in_turn, 600)) + slots * heads * 2 * c.latent * (h.nope + h.v) / 550e6 +
                            pairs * 2 * (h.nope + c.rope + h.v) / 500e6;
    const double absorbed = sizes * (std::fmin(14 + 2 * std::log2(rows * heads), 36) + 0.004 * std::fmin(in_turn, 1024)) +
                            pairs * 2 * (2 * c.latent + c.rope) / 800e6 + rows * heads * (16. * c.latent + 4 * c.rope) / 3e6;
    return expanded < absorbed;
}

bool fits(const Cache& c, const Step& s, const Heads& h, bool expanded) { return expanded ? expanded_fits(c, s, h) : absorbed_fits(c, s, h); }

// The form of a step: what was asked for, else what should be faster, or the other one where that has more workgroups than a launch can.
moe_status choose(const Cache& c, const Step& s, const Heads& h, int form, bool* expanded) {
    *expanded = expands(c, s, h, form);
    if (fits(c, s, h, *expanded)) return MOE_OK;
    *expanded = !*expanded;
    if (form == MOE_LATENT_AUTO && fits(c, s, h, *expanded)) return MOE_OK;
    return fail(MOE_ERR_SHAPE, "too many workgroups: bring fewer sequences or tokens at once");
}

int64_t workspace_of(const Cache& c, const Step& s, const Heads& h, bool expanded) { return expanded ? expanded_workspace(c, s, h) : absorbed_workspace(c, s, h); }

moe_status launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MOE_OK : fail(MOE_ERR_HIP, "launch failed: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" {

const char* moe_latent_last_error(void) { return g_error.text; }

moe_status moe_latent_append(void* stream, const moe_latent_cache* cache, const moe_kv8_step* step, const void* x,
                             int64_t x_row_stride, const void* norm, float eps, const moe_rope_config* rope) {
    TRY(check_sizes(cache));
    TRY(check_step_sizes(cache, step));
    if (rope) {
        TRY(krope::check_config(rope, g_error));
        if (rope->first > cache->rope_dim - rope->rot_dim) return fail(MOE_ERR_SHAPE, "first + rot_dim is over rope_dim");
    }
    if (norm && (!(eps >= 0.f) || std::isinf(eps))) return fail(MOE_ERR_INVALID_ARG, "eps must be finite and not negative");
    Where w{&g_error};
    TRY(w.on(cache->rows, "cache.rows", 16));
    TRY(check_step(step, &w));
    if (step->n_rows == 0) return MOE_OK;
    TRY(check_rows(x, "x", x_row_stride, 0, &w));
    if (norm) TRY(w.on(norm, "norm", 16));
    OnDevice on(w.device);
    if (on.failed()) return fail(MOE_ERR_HIP, "device %d cannot be made current", w.device);
    Append a{};
    a.x = (const uint16_t*)x;
    a.x_row = x_row_stride;
    a.norm = (const uint16_t*)norm;
    a.eps = eps;
    if (rope) {
        a.turns = krope::turns_of(*rope);
        a.rot = rope->rot_dim;
        a.first = rope->first;
        a.interleaved = rope->interleaved;
    }
    launch_append((hipStream_t)stream, cache_of(cache), step_of(step), a);
    return launched();
}

moe_status moe_latent_attend_workspace_bytes(const moe_latent_cache* cache, const moe_kv8_step* step, const moe_latent_heads* heads,
                                             int32_t form, int64_t* bytes_out) {
    if (!bytes_out) return fail(MOE_ERR_INVALID_ARG, "bytes_out is null");
    TRY(check_sizes(cache));
    TRY(check_step_sizes(cache, step));
    TRY(check_head_sizes(cache, heads));
    TRY(check_form(form));
    const Cache c = cache_of(cache);
    const Step s = step_of(step);
    const Heads h = heads_of(cache, heads);
    bool expanded;
    TRY(choose(c, s, h, form, &expanded));
    *bytes_out = workspace_of(c, s, h, expanded);
    return MOE_OK;
}

moe_status moe_latent_attend(void* stream, const moe_latent_cache* cache, const moe_kv8_step* step, const moe_latent_heads* heads,
                             const void* q, int64_t q_row_stride, int64_t q_head_stride, float softmax_scale, int32_t form, void* out,
                             int64_t out_row_stride, int64_t out_head_stride, void* workspace, int64_t workspace_bytes) {
    TRY(check_sizes(cache));
    TRY(check_step_sizes(cache, step));
    TRY(check_head_sizes(cache, heads));
    TRY(check_form(form));
    if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale * (float)kLog2e))
        return fail(MOE_ERR_INVALID_ARG, "softmax_scale must be finite, times log2(e) too, and not negative");
    const Cache c = cache_of(cache);
    const Step s = step_of(step);
    const Heads h = heads_of(cache, heads);
    Where w{&g_error};
    TRY(check_cache(cache, &w));
    TRY(check_step(step, &w));
    if (s.n_rows == 0) return MOE_OK;
    TRY(w.on(heads->w_k, "heads.w_k", 16));
    TRY(w.on(heads->w_v, "heads.w_v", 16));
    TRY(check_rows(q, "q", q_row_stride, q_head_stride, &w));
    TRY(check_rows(out, "out", out_row_stride, out_head_stride, &w));
    if (pieces_overlap(s.n_rows, h.n, out_row_stride, out_head_stride, h.v)) return fail(MOE_ERR_INVALID_ARG, "rows or heads of out overlap");
    if (q == out) return fail(MOE_ERR_INVALID_ARG, "out must not be q");
    bool expanded;
    TRY(choose(c, s, h, form, &expanded));
    const int64_t need = workspace_of(c, s, h, expanded);
    if (workspace_bytes < need) return fail(MOE_ERR_OOM, "workspace of %lld bytes, need %lld", (long long)workspace_bytes, (long long)need);
    TRY(w.on(workspace, "workspace", 256));
    OnDevice on(w.device);
    if (on.failed()) return fail(MOE_ERR_HIP, "device %d cannot be made current", w.device);
    Attend a{};
    a.qscale = (float)(kLog2e * (softmax_scale == 0.f ? 1.0 / std::sqrt((double)(h.nope + c.rope)) : (double)softmax_scale));
    a.q = Rows{(const uint16_t*)q, q_row_stride, q_head_stride};
    a.out = RowsOut{(uint16_t*)out, out_row_stride, out_head_stride};
    a.ws = (uint8_t*)workspace;
    if (expanded) launch_expanded((hipStream_t)stream, c, s, h, a);
    else launch_absorbed((hipStream_t)stream, c, s, h, a);
    return launched();
}

}  // extern "C"
