// Internal interface between the host code of the latent cache and its HIP kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/moe_latent.h"
#include "attn_device.h"
#include "kv8_kernels.h"
#include "rope.h"

namespace klat {

using namespace kattn;
using kkv8::Rows;
using kkv8::RowsOut;
using kkv8::Seq;
using kkv8::Step;

// A cache as the kernels see it: rows of latent + rope elements.
struct Cache {
    int32_t n_seq, latent, rope, max_len, prefix_len;
    uint16_t* rows;
    const uint16_t* prefix;
};

struct Heads {
    int32_t n, nope, v;
    const uint16_t *w_k, *w_v;
    int64_t w_k_head, w_v_head;
};

struct Append {
    const uint16_t* x;
    int64_t x_row;
    const uint16_t* norm;
    float eps;
    krope::Turns turns;
    int32_t rot, first, interleaved;  // rot 0: nothing turns
};

struct Attend {
    float qscale;  // softmax scale times log2(e): the kernels work with base-2 exponentials
    Rows q;
    RowsOut out;
    uint8_t* ws;
};

// Whether a launch of `groups` workgroups of `threads` each counts its threads in 32 bits.
constexpr bool launchable(int64_t groups, int threads) { return groups * threads < (int64_t)1 << 32; }

void launch_append(hipStream_t st, const Cache& c, const Step& s, const Append& a);

// The two forms: whether all their launches are launchable, what they need.
bool absorbed_fits(const Cache& c, const Step& s, const Heads& h);
int64_t absorbed_workspace(const Cache& c, const Step& s, const Heads& h);
void launch_absorbed(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const Attend& a);
bool expanded_fits(const Cache& c, const Step& s, const Heads& h);
int64_t expanded_workspace(const Cache& c, const Step& s, const Heads& h);
void launch_expanded(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const Attend& a);

// Sequence whose rows include `row` (the same for the whole wavefront), and the token's place in it; -1 where there is none.
// The wavefront looks at 64 offsets at a time: two reads one behind the other for up to 4096 sequences, where halving takes twelve.
__device__ __forceinline__ int seq_of_row(const Cache& c, const Step& s, int row, int* token, Seq* q) {
    int lo = 0;
    if (s.row_offsets == nullptr) {
        lo = row / s.max_new;
    } else {
        const int lane = threadIdx.x & 63;
        int n = c.n_seq;  // candidates lo .. lo + n - 1; the one looked for is the last that begins at or before `row`
        while (n > 1) {
            const int step = (n + 63) / 64, at = lane * step;
            const bool before = at < n && s.row_offsets[lo + at] <= row;
            const uint64_t mask = __ballot(before);
            const int last = mask != 0 ? 63 - __builtin_clzll(mask) : 0;
            lo += last * step;
            n = min(step, n - last * step);
        }
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    *q = kkv8::sequence(c.max_len, s, lo);
    *token = row - q->row0;
    return *token >= 0 && *token < q->n_new ? lo : -1;
}

// The same for a row of every lane.
__device__ __forceinline__ int lane_seq_of_row(const Cache& c, const Step& s, int row, int* token, Seq* q) {
    int lo = 0;
    if (s.row_offsets == nullptr) {
        lo = row / s.max_new;
    } else {
        int hi = c.n_seq - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (s.row_offsets[mid] <= row) lo = mid;
            else hi = mid - 1;
        }
    }
    *q = kkv8::sequence(c.max_len, s, lo);
    *token = row - q->row0;
    return *token >= 0 && *token < q->n_new ? lo : -1;
}

}  // namespace klat
