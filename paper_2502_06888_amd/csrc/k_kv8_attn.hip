// Attention over the 8-bit key-value cache.
#include "kv8_kernels.h"

namespace kkv8 {
namespace {

constexpr float kEmpty = -1.0e30f;  // finite stand-in for "no slot seen yet"

__device__ __forceinline__ int seq_of_row(const Step& s, int n_seq, int row) {
    if (s.row_offsets == nullptr) return row / s.max_new;
    int lo = 0, hi = n_seq - 1;  // last sequence whose rows begin at or before `row`
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (s.row_offsets[mid] <= row) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Score of one slot (base 2): q (bf16) . K.
__device__ __forceinline__ float score(const uint16_t* q, const uint8_t* k, float kscale, int hd, float qscale) {
    float dot = 0.f;
    for (int d = 0; d < hd; d += 4) {
        const uint32_t w = *(const uint32_t*)(k + d);
        const u32x2 x = *(const u32x2*)(q + d);
        const uint32_t a = widen2<false>(w, kscale), b = widen2<true>(w, kscale);
        dot = __builtin_fmaf(bf_lo(x.x), bf_lo(a), dot);
        dot = __builtin_fmaf(bf_hi(x.x), bf_hi(a), dot);
        dot = __builtin_fmaf(bf_lo(x.y), bf_lo(b), dot);
        dot = __builtin_fmaf(bf_hi(x.y), bf_hi(b), dot);
    }
    return dot * qscale;
}

// One workgroup per (row, query head): 256 slots at a time, one score per thread, then all threads add their part of
// the slots to the elements they own.
__global__ __launch_bounds__(256) void attend_plain_kernel(Cache c, Step s, Attend a, float* lse) {
    __shared__ float p[256], red[256];
    __shared__ float vs[256];
    const int row = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, hk = h / (a.Hq / c.Hkv), tid = threadIdx.x;
    const int seq = seq_of_row(s, c.n_seq, row);
    const Seq q = sequence(c, s, seq);
    if (row < q.row0 || row >= q.row0 + q.n_new) return;
    const int sees = q.cached + row - q.row0 + 1;
    const int64_t base = (int64_t)seq * c.Hkv + hk, nb = c.max_len >> c.logb;
    const uint8_t *K = c.codes[0] + base * c.max_len * c.hd, *V = c.codes[1] + base * c.max_len * c.hd;
    const float *ks = c.scale[0] + base * nb, *vscale = c.scale[1] + base * nb;
    const uint16_t* qr = a.q.p + (int64_t)row * a.q.row + (int64_t)h * a.q.head;
    const int parts = 256 / c.hd, d = tid % c.hd, part = tid / c.hd;
    float m = kEmpty, l = 0.f, acc = 0.f;
    for (int j0 = 0; j0 < sees; j0 += 256) {
        const int j = j0 + tid;
        const float z = j < sees ? score(qr, K + (int64_t)j * c.hd, ks[j >> c.logb], c.hd, a.qscale) : kEmpty;
        red[tid] = z;
        vs[tid] = j < sees ? vscale[j >> c.logb] : 0.f;
        __syncthreads();
        for (int w = 128; w > 0; w >>= 1) {
            if (tid < w) red[tid] = fmaxf(red[tid], red[tid + w]);
            __syncthreads();
        }
        const float mn = fmaxf(m, red[0]), f = exp2f(m - mn);
        __syncthreads();
        m = mn;
        red[tid] = p[tid] = j < sees ? exp2f(z - mn) : 0.f;
        __syncthreads();
        for (int w = 128; w > 0; w >>= 1) {
            if (tid < w) red[tid] += red[tid + w];
            __syncthreads();
        }
        l = l * f + red[0];
        acc *= f;
        const int most = min(256, sees - j0);
        for (int i = part; i < most; i += parts)
            acc = __builtin_fmaf(p[i], bf_lo(widen2<false>(V[(int64_t)(j0 + i) * c.hd + d], vs[i])), acc);
        __syncthreads();
    }
    red[tid] = acc;
    __syncthreads();
    if (tid < c.hd) {
        for (int i = 1; i < parts; ++i) acc += red[i * c.hd + tid];
        const __bf16 o = (__bf16)(acc / l);
        a.out.p[(int64_t)row * a.out.row + (int64_t)h * a.out.head + tid] = __builtin_bit_cast(uint16_t, o);
    }
    if (tid == 0 && lse != nullptr) lse[(int64_t)row * a.Hq + h] = m + log2f(l);
}

// One thread per slot: the weights that all rows and query heads gave it.
__global__ __launch_bounds__(256) void weights_plain_kernel(Cache c, Step s, Attend a, const float* lse) {
    const int chunks = (c.max_len + 255) / 256, G = a.Hq / c.Hkv;
    const int64_t base = blockIdx.x / chunks;
    const int j = blockIdx.x % chunks * 256 + threadIdx.x, seq = (int)(base / c.Hkv), hk = (int)(base % c.Hkv);
    const Seq q = sequence(c, s, seq);
    if (j >= q.cached + q.n_new) return;
    float w = a.weight_in != nullptr && j < q.cached ? a.weight_in[base * c.max_len + j] : 0.f;
    const uint8_t* K = c.codes[0] + (base * c.max_len + j) * c.hd;
    const float ks = c.scale[0][base * (c.max_len >> c.logb) + (j >> c.logb)];
    for (int i = max(0, j - q.cached); i < q.n_new; ++i)
        for (int g = 0; g < G; ++g) {
            const int64_t row = q.row0 + i, h = hk * G + g;
            w += exp2f(score(a.q.p + row * a.q.row + h * a.q.head, K, ks, c.hd, a.qscale) - lse[row * a.Hq + h]);
        }
    a.weight_out[base * c.max_len + j] = w;
}

}  // namespace

int64_t attend_workspace(const Cache& c, const Step& s, int Hq, bool weights) {
    return weights ? ((int64_t)s.n_rows * Hq * 4 + 255) & ~(int64_t)255 : 0;
}

void launch_attend(hipStream_t st, const Cache& c, const Step& s, const Attend& a) {
    float* lse = a.weight_out != nullptr ? (float*)a.ws : nullptr;
    if (s.n_rows > 0)
        hipLaunchKernelGGL(attend_plain_kernel, dim3((unsigned)((int64_t)s.n_rows * a.Hq)), dim3(256), 0, st, c, s, a, lse);
    if (a.weight_out != nullptr)
        hipLaunchKernelGGL(weights_plain_kernel, dim3((unsigned)((int64_t)c.n_seq * c.Hkv * ((c.max_len + 255) / 256))),
                           dim3(256), 0, st, c, s, a, (const float*)lse);
}

}  // namespace kkv8
