// Filling the 8-bit key-value cache and evicting from it.
#include "kv8_kernels.h"

namespace kkv8 {
namespace {

// ---- append ------------------------------------------------------------------------------------------
//
// One unit of WAVES wavefronts per (sequence, head, K or V, block of slots that the new tokens fall into): the largest
// magnitude of the new rows, the scale, then the codes; the codes that the block held are rounded again only where the
// scale rose.  A lane takes 16-byte pieces of the rows (8 elements) and writes 8 codes.
template <int WAVES>
__global__ __launch_bounds__(256) void append_kernel(Cache c, Step s, Rows k, Rows v, int blocks) {
    constexpr int UNITS = 4 / WAVES, N = 64 * WAVES;
    __shared__ uint32_t most[4];
    const int wave = threadIdx.x >> 6;
    const int tid = (int)threadIdx.x % N;
    const int64_t unit = (int64_t)blockIdx.x * UNITS + (int)threadIdx.x / N;
    const int64_t pair = unit / (2 * blocks);
    const bool exists = pair < (int64_t)c.n_seq * c.Hkv;
    const int seq = exists ? (int)(pair / c.Hkv) : 0, head = exists ? (int)(pair % c.Hkv) : 0;
    const int rest = (int)(unit % (2 * blocks)), kv = rest & 1;
    const Seq q = sequence(c, s, seq);
    const int block = ((q.cached >> c.logb) + (rest >> 1));
    const int lo = max(q.cached, block << c.logb), hi = min(q.cached + q.n_new, (block + 1) << c.logb);
    const int n = exists ? max(hi - lo, 0) : 0;  // new slots of this block
    const Rows r = kv ? v : k;
    const int pieces = c.hd / 8, total = n * pieces;
    const uint16_t* src = r.p + (int64_t)(q.row0 + (lo - q.cached)) * r.row + (int64_t)head * r.head;
    uint32_t top = 0;
    for (int i = tid; i < total; i += N) {
        const u32x4 x = *(const u32x4*)(src + (int64_t)(i / pieces) * r.row + i % pieces * 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t a = x[j] & 0x7fffu, b = (x[j] >> 16) & 0x7fffu;  // magnitudes order as integers
            if (a < 0x7f80u) top = max(top, a);
            if (b < 0x7f80u) top = max(top, b);
        }
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, 64));
    const int64_t base = (int64_t)seq * c.Hkv + head;
    float* scale = c.scale[kv] + base * (c.max_len >> c.logb) + block;
    const bool begun = n > 0 && lo > (block << c.logb);
    const float before = begun ? *scale : 0.f;
    if (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) most[wave] = top;
        __syncthreads();  // everybody has read the scale, too
        top = max(max(most[0], most[1]), max(most[2], most[3]));
    }
    if (n == 0) return;
    const float now = fmaxf(least_scale(top), before);
    if (tid == 0) *scale = now;
    uint8_t* codes = c.codes[kv] + (base * c.max_len) * c.hd;
    if (begun && now != before) {
        const float by = before / now;
        uint32_t* old = (uint32_t*)(codes + (int64_t)(block << c.logb) * c.hd);
        const int words = (lo - (block << c.logb)) * c.hd / 4;
        for (int i = tid; i < words; i += N) old[i] = rescale4(old[i], by);
    }
    const float inv = 1.f / now;  // a power of two
    u32x2* dst = (u32x2*)(codes + (int64_t)lo * c.hd);
    for (int i = tid; i < total; i += N) {
        const u32x4 x = *(const u32x4*)(src + (int64_t)(i / pieces) * r.row + i % pieces * 8);
        u32x2 o;
        o.x = codes4(bf_lo(x.x) * inv, bf_hi(x.x) * inv, bf_lo(x.y) * inv, bf_hi(x.y) * inv);
        o.y = codes4(bf_lo(x.z) * inv, bf_hi(x.z) * inv, bf_lo(x.w) * inv, bf_hi(x.w) * inv);
        dst[i] = o;
    }
    if (kv == 0 && c.position != nullptr) {
        const int first = (s.next_position != nullptr ? s.next_position[seq] : q.cached) + lo - q.cached;
        for (int i = tid; i < n; i += N) c.position[base * c.max_len + lo + i] = first + i;
    }
}

// ---- evict -------------------------------------------------------------------------------------------

// Order of the weights as unsigned numbers: larger weight, larger key; NaN 0, recent slots the largest.
__device__ __forceinline__ uint32_t key_of(float w, bool recent) {
    if (recent) return 0xffffffffu;
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.f);  // -0 counts as 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive sum over the 256 threads of two counts packed into one word.
__device__ __forceinline__ uint32_t scan256(uint32_t v, uint32_t* total, uint32_t* part) {
    uint32_t inc = v;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)inc, d, 64);
        if (lane >= d) inc += o;
    }
    __syncthreads();  // `part` may still be read from the call before
    if (lane == 63) part[threadIdx.x >> 6] = inc;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += part[w];
    *total = part[0] + part[1] + part[2] + part[3];
    return before + inc - v;
}

// One workgroup per (sequence, head): the key of the keep-th largest weight digit by digit (four passes over 8 bits),
// then the chosen slots in order, the list of those that have to move, and what every slot below `keep` takes over.
__global__ __launch_bounds__(256) void select_kernel(Cache c, const int32_t* held, int max_held, int keep, int recent,
                                                     const int32_t* next_position, const float* weight_in,
                                                     float* weight_out, const int32_t* position_in,
                                                     int32_t* position_out, int32_t* sources, int32_t* kept) {
    __shared__ uint32_t hist[256], part[4], found[2];
    const int64_t pair = blockIdx.x;
    const int seq = (int)(pair / c.Hkv), tid = threadIdx.x;
    const int n = clampi(held[seq], 0, max_held);
    const float* win = weight_in + pair * c.max_len;
    float* wout = weight_out + pair * c.max_len;
    const int32_t* pin = position_in + pair * c.max_len;
    int32_t* pout = position_out + pair * c.max_len;
    int32_t* list = sources + pair * keep;
    int32_t* to = kept + pair * keep;
    if (n <= keep) {
        for (int i = tid; i < keep; i += 256) {
            to[i] = i < n ? i : -1;
            if (i < n) {
                if (wout != win) wout[i] = win[i];
                if (pout != pin) pout[i] = pin[i];
            }
        }
        return;
    }
    // positions from here on are recent; in 64 bits, since next - recent may pass the least int
    const int64_t young = (int64_t)(next_position != nullptr ? next_position[seq] : n) - recent;
    auto key = [&](int i) { return key_of(win[i], recent > 0 && pin[i] >= young); };
    uint32_t prefix = 0;
    int want = keep;  // how many of the slots that share the prefix are chosen
    for (int shift = 24; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        for (int i = tid; i < n; i += 256) {
            const uint32_t k = key(i);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        // thread t looks at digit 255 - t: how many lie above it
        uint32_t all;
        const uint32_t mine = hist[255 - tid], above = scan256(mine, &all, part);
        if (above < (uint32_t)want && above + mine >= (uint32_t)want) {
            found[0] = 255u - tid;
            found[1] = above;
        }
        __syncthreads();
        prefix |= found[0] << shift;
        want -= (int)found[1];
        __syncthreads();
    }
    // slots above the key are chosen, and the first `want` of those at it
    uint32_t ties = 0, moved = 0, holes = 0;
    for (int base = 0; base < n; base += 256) {
        const int i = base + tid;
        const uint32_t k = i < n ? key(i) : 0u;
        const bool tie = i < n && k == prefix;
        uint32_t all;
        const uint32_t rank = ties + scan256(tie ? 1u : 0u, &all, part);
        ties += all;
        const bool chosen = i < n && (k > prefix || (tie && rank < (uint32_t)want));
        const bool hole = i < keep && !chosen, source = i >= keep && chosen;
        const uint32_t at = scan256((hole ? 1u : 0u) | (source ? 1u << 16 : 0u), &all, part);
        if (source) list[moved + (at >> 16)] = i;
        if (i < keep) to[i] = hole ? -2 - (int)(holes + (at & 0xffffu)) : i;
        holes += all & 0xffffu;
        moved += all >> 16;
    }
    __syncthreads();
    for (int i = tid; i < keep; i += 256) {
        int from = to[i];
        if (from < 0) to[i] = from = list[-2 - from];
        if (from != i || wout != win) wout[i] = win[from];
        if (from != i || pout != pin) pout[i] = pin[from];
    }
}

// One workgroup per (sequence, head, block below `keep`): the codes that moved into it.
__global__ __launch_bounds__(256) void move_kernel(Cache c, int keep, const int32_t* kept) {
    const int blocks = keep >> c.logb, B = 1 << c.logb;
    const int64_t pair = blockIdx.x / blocks;
    const int block = blockIdx.x % blocks;
    const int32_t* from = kept + pair * keep + (block << c.logb);
    __shared__ int src[128];
    __shared__ int any;
    if (threadIdx.x == 0) any = 0;
    __syncthreads();
    if (threadIdx.x < (unsigned)B) {
        const int f = from[threadIdx.x];
        src[threadIdx.x] = f;
        if (f >= keep) any = 1;
    }
    __syncthreads();
    if (any == 0) return;
    const int words = c.hd / 4;
    for (int kv = 0; kv < 2; ++kv) {
        float* scale = c.scale[kv] + pair * (c.max_len >> c.logb);
        uint32_t* codes = (uint32_t*)(c.codes[kv] + pair * c.max_len * c.hd);
        const float before = scale[block];
        float now = before;
        for (int i = 0; i < B; ++i)
            if (src[i] >= keep) now = fmaxf(now, scale[src[i] >> c.logb]);
        __syncthreads();
        if (threadIdx.x == 0) scale[block] = now;
        for (int i = threadIdx.x; i < B * words; i += 256) {
            const int slot = i / words, f = src[slot];
            if (f < keep && (now == before || f < 0)) continue;
            const float by = (f >= keep ? scale[f >> c.logb] : before) / now;
            const uint32_t w = codes[(int64_t)f * words + i % words];
            codes[((int64_t)(block << c.logb) + slot) * words + i % words] = by == 1.f ? w : rescale4(w, by);
        }
    }
}

}  // namespace

void launch_append(hipStream_t st, const Cache& c, const Step& s, const Rows& k, const Rows& v) {
    const int B = 1 << c.logb;
    const int blocks = (s.max_new + B - 2) / B + 1;  // blocks that max_new tokens can fall into
    const int64_t units = (int64_t)c.n_seq * c.Hkv * 2 * blocks;
    if (s.max_new <= 4)
        hipLaunchKernelGGL(append_kernel<1>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st, c, s, k, v, blocks);
    else
        hipLaunchKernelGGL(append_kernel<4>, dim3((unsigned)units), dim3(256), 0, st, c, s, k, v, blocks);
}

static int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

int64_t evict_workspace(const Cache& c, int keep) { return 2 * up256((int64_t)c.n_seq * c.Hkv * keep * 4); }

void launch_evict(hipStream_t st, const Cache& c, const int32_t* held, int max_held, int keep, int recent,
                  const int32_t* next_position, const float* weight_in, float* weight_out, int32_t* position_out,
                  int32_t* kept, uint8_t* ws) {
    const int64_t pairs = (int64_t)c.n_seq * c.Hkv;
    int32_t* list = (int32_t*)ws;
    if (kept == nullptr) kept = (int32_t*)(ws + up256(pairs * keep * 4));
    hipLaunchKernelGGL(select_kernel, dim3((unsigned)pairs), dim3(256), 0, st, c, held, max_held, keep, recent,
                       next_position, weight_in, weight_out, c.position, position_out, list, kept);
    if (max_held > keep)
        hipLaunchKernelGGL(move_kernel, dim3((unsigned)(pairs * (keep >> c.logb))), dim3(256), 0, st, c, keep, kept);
}

}  // namespace kkv8
