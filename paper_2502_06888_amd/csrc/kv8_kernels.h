// Internal interface between the host code of the 8-bit key-value cache and its HIP kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/moe_kv8.h"
#include "attn_device.h"

namespace kkv8 {

// A cache as the kernels see it; logb = log2(block).
struct Cache {
    int32_t n_seq, Hkv, hd, max_len, logb;
    uint8_t* codes[2];  // K, V
    float* scale[2];
    int32_t* position;
};

// The new rows of a step (moe_kv8_step).
struct Step {
    int32_t n_rows, max_new, max_cached;
    const int32_t* row_offsets;
    const int32_t* cached;
    const int32_t* next_position;
};

struct Rows {  // bf16 rows in the caller's layout, strides in elements
    const uint16_t* p;
    int64_t row, head;
};
struct RowsOut {
    uint16_t* p;
    int64_t row, head;
};

struct Attend {
    int32_t Hq;
    float qscale;  // softmax scale times log2(e): the kernels work with base-2 exponentials
    Rows q;
    RowsOut out;
    const float* weight_in;
    float* weight_out;
    uint8_t* ws;
};

// Workgroups of 256 threads of a launch, at most: it counts its threads in 32 bits.
constexpr int64_t kMostGroups = (1 << 24) - 1;

// Whether the grids of the launches stay within that.
bool append_fits(const Cache& c, const Step& s);
bool evict_fits(const Cache& c, int keep);
bool attend_fits(const Cache& c, const Step& s, int Hq, bool weights);

void launch_append(hipStream_t st, const Cache& c, const Step& s, const Rows& k, const Rows& v);
int64_t attend_workspace(const Cache& c, const Step& s, int Hq, bool weights);
void launch_attend(hipStream_t st, const Cache& c, const Step& s, const Attend& a);
int64_t evict_workspace(const Cache& c, int keep);
void launch_evict(hipStream_t st, const Cache& c, const int32_t* held, int max_held, int keep, int recent,
                  const int32_t* next_position, const float* weight_in, float* weight_out, int32_t* position_out,
                  int32_t* kept, uint8_t* ws);

// For the attention layer, whose rows lie in its own workspace: what moe_kv8_append and moe_kv8_attend would refuse (with
// the text in moe_kv8_last_error), and the kernels' views of the caller's structs.
moe_status check_layer_call(const moe_kv8_cache* cache, const moe_kv8_step* step, int n_q_heads, const void* rows,
                            const float* weight_in, const float* weight_out, const void* workspace, int64_t workspace_bytes);
Cache cache_of_call(const moe_kv8_cache* c);
Step step_of_call(const moe_kv8_step* s);

// ---- device helpers shared by the kernels -------------------------------------------------------

using namespace kattn;

// What a sequence brings and holds, every number brought into its bounds.
struct Seq {
    int row0, n_new, cached;
};
__device__ __forceinline__ Seq sequence(int max_len, const Step& s, int seq) {
    Seq q;
    if (s.row_offsets != nullptr) {
        q.row0 = clampi(s.row_offsets[seq], 0, s.n_rows);
        q.n_new = min(clampi(s.row_offsets[seq + 1], q.row0, s.n_rows) - q.row0, s.max_new);
    } else {
        q.row0 = seq * s.max_new;
        q.n_new = s.max_new;
    }
    q.cached = clampi(s.cached[seq], 0, s.max_cached);
    q.n_new = min(q.n_new, max_len - q.cached);
    return q;
}
__device__ __forceinline__ Seq sequence(const Cache& c, const Step& s, int seq) { return sequence(c.max_len, s, seq); }

// Sequence whose rows include `row`, and the token's place in it; -1 where there is none.
__device__ __forceinline__ int seq_of_row(const Cache& c, const Step& s, int row, int* token, Seq* q) {
    int lo = 0;
    if (s.row_offsets == nullptr) {
        lo = row / s.max_new;
    } else {
        int hi = c.n_seq - 1;  // last sequence whose rows begin at or before `row`
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (s.row_offsets[mid] <= row) lo = mid;
            else hi = mid - 1;
        }
    }
    *q = sequence(c, s, lo);
    *token = row - q->row0;
    return *token >= 0 && *token < q->n_new ? lo : -1;
}

// Two codes (bytes 0, 1 or 2, 3 of w) as bf16 times a power of two: exact.
template <bool HI>
__device__ __forceinline__ uint32_t widen2(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// Four floats as e4m3 codes, to nearest even; magnitudes beyond 448 become 448, NaN stays NaN.
__device__ __forceinline__ float fit(float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(fit(a), fit(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fit(c), fit(d), w, true);
}
// Four codes rounded again to another scale: `by` = old scale / new scale, a power of two of at most 1.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float by) {
    const uint32_t a = widen2<false>(w, 1.f), b = widen2<true>(w, 1.f);
    return codes4(bf_lo(a) * by, bf_hi(a) * by, bf_lo(b) * by, bf_hi(b) * by);
}
// Least power of two s with largest <= 448 s; `largest`: the magnitude bits of a finite bf16 value.
constexpr int kLeastExp = -100, kMostExp = 119;
__device__ __forceinline__ float least_scale(uint32_t largest_bf16) {
    const uint32_t f = largest_bf16 << 16;
    const int e = (int)(f >> 23) - 127 - ((f & 0x7fffffu) <= 0x600000u ? 8 : 7);  // 448 = 1.75 * 2^8
    return __uint_as_float((uint32_t)(clampi(e, kLeastExp, kMostExp) + 127) << 23);
}

}  // namespace kkv8
