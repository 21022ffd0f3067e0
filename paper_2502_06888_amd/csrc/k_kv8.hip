// Filling the 8-bit key-value cache and evicting from it.
#include "kv8_kernels.h"

namespace kkv8 {
namespace {

// ---- append ------------------------------------------------------------------------------------------
//
// One unit of WAVES wavefronts per (sequence, head, K or V, block of slots that the new tokens fall into): the largest
// magnitude of the new rows, the scale, then the codes; the codes that the block held are rounded again only where the
// scale rose.  A lane takes 16-byte pieces of the rows (8 elements), keeps them in registers between the two uses, and
// writes 8 codes.  Dividing by the scale is exact (a power of two), so a code has the one rounding to e4m3.
// Bound by the bytes for prompts (32 x 512 tokens of 8 heads of 128: 101 MB in 23.5 us, 4.3 TB/s, 4.8 being what a large copy
// reaches), by latency for single tokens (512 sequences: 7 us), where a unit is a wavefront: up to four tokens of 128
// elements are one piece per lane.
template <int WAVES>
__global__ __launch_bounds__(256) void append_kernel(Cache c, Step s, Rows k, Rows v, int blocks) {
    constexpr int UNITS = 4 / WAVES, N = 64 * WAVES, PER = WAVES == 1 ? 1 : 8;
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
    const int logp = c.hd == 128 ? 4 : c.hd == 64 ? 3 : 2, total = n << logp;  // pieces of 8 elements
    const uint16_t* src = r.p + (int64_t)(q.row0 + (lo - q.cached)) * r.row + (int64_t)head * r.head;
    // at most PER pieces per thread: a block of 128 slots of 128 elements, or four tokens for a wavefront
    u32x4 x[PER];
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = tid + u * N;
        if (i < total) x[u] = __builtin_nontemporal_load((const u32x4*)(src + (int64_t)(i >> logp) * r.row + (i & ((1 << logp) - 1)) * 8));
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        if (tid + u * N >= total) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t a = x[u][j] & 0x7fffu, b = (x[u][j] >> 16) & 0x7fffu;  // magnitudes order as integers
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
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = tid + u * N;
        if (i >= total) break;
        u32x2 o;
        o.x = codes4(bf_lo(x[u].x) * inv, bf_hi(x[u].x) * inv, bf_lo(x[u].y) * inv, bf_hi(x[u].y) * inv);
        o.y = codes4(bf_lo(x[u].z) * inv, bf_hi(x[u].z) * inv, bf_lo(x[u].w) * inv, bf_hi(x[u].w) * inv);
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

// Exclusive sum over the workgroup's kLong threads of two counts packed into one word.
constexpr int kLong = 1024;
__device__ __forceinline__ uint32_t scan_long(uint32_t v, uint32_t* total, uint32_t* part) {
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
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kLong / 64; ++w) {
        const uint32_t p = part[w];
        if (w < (int)(threadIdx.x >> 6)) before += p;
        all += p;
    }
    *total = all;
    return before + inc - v;
}

// Sum over the 16 lanes of a row, in every lane.
__device__ __forceinline__ int row16_sum(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false);  // row_ror by 8, 4, 2, 1
    v += __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, false);
    return v + __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, false);
}

// What a (sequence, head) pair selects from and writes to.
struct Select {
    const int32_t* held;
    int32_t max_held, keep, recent;
    const int32_t* next_position;
    const float* weight_in;
    float* weight_out;
    const int32_t* position_in;
    int32_t* position_out;
    int32_t* sources;  // [pair, keep], of select_long_kernel: chosen slots from `keep` on, in order
    int32_t* kept;     // [pair, keep] slot that each slot was before
};

// One group of WAVES wavefronts per (sequence, head), KPT keys per lane in registers (slot = step * lanes + lane).  The key
// of the keep-th largest weight is found by halving the range of keys, 32 times: the compares of a step leave a count in
// scalar registers, groups of several wavefronts add theirs up through LDS.  Then the ranks of the chosen slots,
// by ballots and one scan over the (step, wavefront) counts.  Reads weights and positions once.  Pairs that fill the chip
// take one wavefront each; a few pairs would leave it idle, so 16 wavefronts share one.
// The halving ends as soon as a bound parts off just `keep` keys, after 20 steps or so where weights differ.
// Bound by latency: 4096 pairs of 545 slots 19 us (45 MB), 32 pairs of 7500 slots 17 us.
template <int WAVES, int KPT>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void select_kernel(Cache c, Select a) {
    static_assert(WAVES == 1 || WAVES == 16);
    constexpr int GROUPS = WAVES == 1 ? 4 : 1, LANES = WAVES * 64, CELLS = KPT * WAVES;
    __shared__ int counts[2][WAVES];
    __shared__ uint32_t cells[GROUPS][CELLS];
    __shared__ uint16_t movers[GROUPS][KPT * LANES / 2];  // chosen slots from `keep` on, in order: at most half of all
    const int group = WAVES == 1 ? threadIdx.x >> 6 : 0, wave = WAVES == 1 ? 0 : threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int tid = wave * 64 + lane;
    const int64_t pair = (int64_t)blockIdx.x * GROUPS + group;
    const bool exists = pair < (int64_t)c.n_seq * c.Hkv;
    const int64_t at = exists ? pair : 0;
    const int seq = (int)(at / c.Hkv), keep = a.keep;
    const int n = exists ? clampi(a.held[seq], 0, a.max_held) : 0;
    const bool cut = n > keep;
    const float* win = a.weight_in + at * c.max_len;
    const int32_t* pin = a.position_in + at * c.max_len;
    float* wout = a.weight_out + at * c.max_len;
    int32_t* pout = a.position_out + at * c.max_len;
    uint16_t* list = movers[group];
    int32_t* to = a.kept + at * keep;
    // positions from here on are recent; in 64 bits, since next - recent may pass the least int
    const int64_t young = (int64_t)(a.next_position != nullptr ? a.next_position[seq] : n) - a.recent;
    uint32_t key[KPT];
    {  // unconditional reads (past n the last slot again), so that all are on their way at once
        float w[KPT];
        int32_t pos[KPT];
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
            const int i = clampi(j * LANES + tid, 0, max(n - 1, 0));
            w[j] = win[i];
            pos[j] = pin[i];
        }
#pragma unroll
        for (int j = 0; j < KPT; ++j) key[j] = cut && j * LANES + tid < n ? key_of(w[j], a.recent > 0 && pos[j] >= young) : 0u;
    }
    // keys past n count as 0, the least there is: they are told apart by their slot
    int phase = 0;
    auto count_over = [&](uint32_t v) {  // keys >= v, v > 0
        int sum = 0;
#pragma unroll
        for (int j = 0; j < KPT; ++j) sum += __popcll(__ballot(key[j] >= v));
        if (WAVES > 1) {
            if (lane == 0) counts[phase][wave] = sum;
            __syncthreads();
            sum = row16_sum(counts[phase][lane & 15]);  // WAVES == 16
            phase ^= 1;  // the next counts go elsewhere, so that one barrier is enough
        }
        return sum;
    };
    uint32_t best = 0;  // largest key that at least `keep` keys reach
    int want = -1;      // how many of the slots at it are chosen
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t v = best | 1u << bit;
        const int reach = count_over(v);
        if (reach >= keep) best = v;
        if (reach == keep) {  // just these: all that lie over v - 1
            best = v - 1;
            want = 0;
            break;
        }
    }
    if (want < 0) want = keep - (best == 0xffffffffu ? 0 : count_over(best + 1));
    // exclusive sums over the cells (step, wavefront) in order; a wavefront scans them, CELLS / 64 per lane
    auto scan = [&] {
        __syncthreads();
        if (wave == 0) {
            constexpr int PER = (CELLS + 63) / 64;
            uint32_t v[PER], mine = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                v[e] = lane * PER + e < CELLS ? cells[group][lane * PER + e] : 0u;
                mine += v[e];
            }
            uint32_t inc = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t o = (uint32_t)__shfl_up((int)inc, d, 64);
                if (lane >= d) inc += o;
            }
            uint32_t run = inc - mine;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (lane * PER + e < CELLS) cells[group][lane * PER + e] = run;
                run += v[e];
            }
        }
        __syncthreads();
    };
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const uint64_t ties = __ballot(j * LANES + tid < n && key[j] == best);
        if (lane == 0) cells[group][j * WAVES + wave] = (uint32_t)__popcll(ties);
    }
    scan();
    uint64_t chosen[KPT];
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = j * LANES + tid;
        const bool tie = i < n && key[j] == best;
        const uint64_t ties = __ballot(tie);
        const int rank = (int)cells[group][j * WAVES + wave] + __popcll(ties & below);
        chosen[j] = __ballot(i < n && (key[j] > best || (tie && rank < want)));
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = j * LANES + tid;
        const bool in = chosen[j] >> lane & 1;
        const uint64_t holes = __ballot(cut && i < keep && !in), sources = __ballot(cut && i >= keep && in);
        if (lane == 0) cells[group][j * WAVES + wave] = (uint32_t)__popcll(holes) | (uint32_t)__popcll(sources) << 16;
    }
    scan();
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = j * LANES + tid;
        const bool in = chosen[j] >> lane & 1;
        const uint64_t sources = __ballot(cut && i >= keep && in);
        if (cut && i >= keep && in) list[(cells[group][j * WAVES + wave] >> 16) + __popcll(sources & below)] = (uint16_t)i;
    }
    __syncthreads();
    // All reads before the writes, which may go to the same tensors: one wait instead of one per step.
    int from[KPT];
    float w[KPT];
    int32_t pos[KPT];
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = j * LANES + tid;
        const bool in = chosen[j] >> lane & 1;
        const uint64_t holes = __ballot(cut && i < keep && !in);
        from[j] = i < keep && i < n ? i : -1;
        if (cut && i < keep && !in) from[j] = list[(cells[group][j * WAVES + wave] & 0xffffu) + __popcll(holes & below)];
        w[j] = win[max(from[j], 0)];
        pos[j] = pin[max(from[j], 0)];
    }
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = j * LANES + tid;
        if (exists && i < keep) to[i] = from[j];
        if (from[j] < 0) continue;
        if (from[j] != i || wout != win) wout[i] = w[j];
        if (from[j] != i || pout != pin) pout[i] = pos[j];
    }
}

// The same for sequences of any length, kLong slots at a time: the key digit by digit (four passes over 8 bits), then the
// chosen slots in order.  Bound by latency: 8 pairs of 40000 slots, with the move, 129 us (by 256 threads 356), of 131072 364.
__global__ __launch_bounds__(kLong) void select_long_kernel(Cache c, Select a) {
    __shared__ uint32_t hist[256], part[kLong / 64], found[2];
    const int64_t pair = blockIdx.x;
    const int seq = (int)(pair / c.Hkv), tid = threadIdx.x, keep = a.keep;
    const int n = clampi(a.held[seq], 0, a.max_held);
    const float* win = a.weight_in + pair * c.max_len;
    float* wout = a.weight_out + pair * c.max_len;
    const int32_t* pin = a.position_in + pair * c.max_len;
    int32_t* pout = a.position_out + pair * c.max_len;
    int32_t* list = a.sources + pair * keep;
    int32_t* to = a.kept + pair * keep;
    if (n <= keep) {
        for (int i = tid; i < keep; i += kLong) {
            to[i] = i < n ? i : -1;
            if (i < n) {
                if (wout != win) wout[i] = win[i];
                if (pout != pin) pout[i] = pin[i];
            }
        }
        return;
    }
    const int64_t young = (int64_t)(a.next_position != nullptr ? a.next_position[seq] : n) - a.recent;
    auto key = [&](int i) { return key_of(win[i], a.recent > 0 && pin[i] >= young); };
    uint32_t prefix = 0;
    int want = keep;  // how many of the slots that share the prefix are chosen
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        for (int i = tid; i < n; i += kLong) {
            const uint32_t k = key(i);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        // thread t looks at digit 255 - t: how many lie above it
        uint32_t all;
        const uint32_t mine = tid < 256 ? hist[255 - tid] : 0u, above = scan_long(mine, &all, part);
        if (tid < 256 && above < (uint32_t)want && above + mine >= (uint32_t)want) {
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
    for (int base = 0; base < n; base += kLong) {
        const int i = base + tid;
        const uint32_t k = i < n ? key(i) : 0u;
        const bool tie = i < n && k == prefix;
        uint32_t all;
        const uint32_t rank = ties + scan_long(tie ? 1u : 0u, &all, part);
        ties += all;
        const bool chosen = i < n && (k > prefix || (tie && rank < (uint32_t)want));
        const bool hole = i < keep && !chosen, source = i >= keep && chosen;
        const uint32_t at = scan_long((hole ? 1u : 0u) | (source ? 1u << 16 : 0u), &all, part);
        if (source) list[moved + (at >> 16)] = i;
        if (i < keep) to[i] = hole ? -2 - (int)(holes + (at & 0xffffu)) : i;
        holes += all & 0xffffu;
        moved += all >> 16;
    }
    __syncthreads();
    for (int i = tid; i < keep; i += kLong) {
        int from = to[i];
        if (from < 0) to[i] = from = list[-2 - from];
        if (from != i || wout != win) wout[i] = win[from];
        if (from != i || pout != pin) pout[i] = pin[from];
    }
}

// One workgroup per (sequence, head) and 512 slots below `keep`: which of them moved, what that makes of the scales of their
// blocks, then the codes, 16 bytes per lane, those of K by half the threads and those of V by the others.  A block whose
// scale rises is rounded again as a whole.  Bound by latency (few slots of a block move): 4096 pairs of 8 blocks of which 31
// slots move take 24 us (47 with a wavefront per block), 32 pairs of 64 blocks of which 1900 move 11.
constexpr int kSpan = 512;
template <int HD>
__global__ __launch_bounds__(256) void move_kernel(Cache c, int keep, const int32_t* kept) {
    constexpr int LPS = HD / 16, SIDE = 128 / LPS, AHEAD = 4;  // lanes per slot, slots side by side, pieces on their way
    __shared__ int n_moved;
    __shared__ int32_t slots[kSpan], from[kSpan];   // slots that moved, and where they come from
    __shared__ uint32_t now[2][kSpan / 16];         // scales of K and V, as bits: positive, so they order as integers
    __shared__ float was[2][kSpan / 16];
    const int spans = (keep + kSpan - 1) / kSpan, tid = threadIdx.x;
    const int64_t pair = blockIdx.x / spans;
    const int s0 = (int)(blockIdx.x % spans) * kSpan, n = min(kSpan, keep - s0), blocks = n >> c.logb;
    const int32_t* list = kept + pair * keep + s0;
    const int64_t sb = pair * (c.max_len >> c.logb);
    if (tid == 0) n_moved = 0;
    if (tid < 2 * blocks) {
        const int kv = tid >= blocks, b = tid - kv * blocks;
        const float x = c.scale[kv][sb + (s0 >> c.logb) + b];
        was[kv][b] = x;
        now[kv][b] = __float_as_uint(x);
    }
    __syncthreads();
    for (int i = tid; i < n; i += 256) {
        const int f = list[i];
        if (f < keep) continue;
        const int at = atomicAdd(&n_moved, 1);  // in any order: every slot is moved by itself
        slots[at] = i;
        from[at] = f;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) atomicMax(&now[kv][i >> c.logb], __float_as_uint(c.scale[kv][sb + (f >> c.logb)]));
    }
    __syncthreads();
    const int moved = n_moved;
    if (moved == 0) return;
    const int kv = tid >> 7, lane = tid & 127;
    u32x4* codes = (u32x4*)(c.codes[kv] + pair * c.max_len * HD);
    for (int i = lane / LPS; i < moved; i += SIDE * AHEAD) {
        u32x4 x[AHEAD];
        float by[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {  // past the end: the last one again, unused
            const int f = from[min(i + u * SIDE, moved - 1)];
            x[u] = codes[(int64_t)f * LPS + lane % LPS];
            by[u] = c.scale[kv][sb + (f >> c.logb)];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (i + u * SIDE >= moved) break;
            const int slot = slots[i + u * SIDE];
            by[u] /= __uint_as_float(now[kv][slot >> c.logb]);  // powers of two
            if (by[u] != 1.f)
#pragma unroll
                for (int w = 0; w < 4; ++w) x[u][w] = rescale4(x[u][w], by[u]);
            codes[(int64_t)(s0 + slot) * LPS + lane % LPS] = x[u];
        }
    }
    for (int b = 0; b < blocks; ++b) {
        const float to = __uint_as_float(now[kv][b]), by = was[kv][b] / to;
        if (by == 1.f) continue;
        if (lane == 0) c.scale[kv][sb + (s0 >> c.logb) + b] = to;
        for (int i = (b << c.logb) + lane / LPS; i < (b + 1) << c.logb; i += SIDE) {  // slots that stayed
            if (list[i] != s0 + i) continue;
            const int64_t at = (int64_t)(s0 + i) * LPS + lane % LPS;
            u32x4 x = codes[at];
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] = rescale4(x[w], by);
            codes[at] = x;
        }
    }
}

}  // namespace

// Blocks that max_new tokens can fall into, and units of K and V over all pairs.
static int append_blocks(const Cache& c, const Step& s) { return (s.max_new + (1 << c.logb) - 2) / (1 << c.logb) + 1; }
static int64_t append_units(const Cache& c, const Step& s) { return (int64_t)c.n_seq * c.Hkv * 2 * append_blocks(c, s); }

bool append_fits(const Cache& c, const Step& s) { return append_units(c, s) <= kMostGroups; }

void launch_append(hipStream_t st, const Cache& c, const Step& s, const Rows& k, const Rows& v) {
    const int blocks = append_blocks(c, s);
    const int64_t units = append_units(c, s);
    if (s.max_new <= 4)
        hipLaunchKernelGGL(append_kernel<1>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st, c, s, k, v, blocks);
    else
        hipLaunchKernelGGL(append_kernel<4>, dim3((unsigned)units), dim3(256), 0, st, c, s, k, v, blocks);
}

static int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

static int64_t spans(const Cache& c, int keep) { return (int64_t)c.n_seq * c.Hkv * ((keep + kSpan - 1) / kSpan); }
bool evict_fits(const Cache& c, int keep) { return spans(c, keep) <= kMostGroups; }

int64_t evict_workspace(const Cache& c, int keep) { return 2 * up256((int64_t)c.n_seq * c.Hkv * keep * 4); }

void launch_evict(hipStream_t st, const Cache& c, const int32_t* held, int max_held, int keep, int recent,
                  const int32_t* next_position, const float* weight_in, float* weight_out, int32_t* position_out,
                  int32_t* kept, uint8_t* ws) {
    const int64_t pairs = (int64_t)c.n_seq * c.Hkv;
    if (kept == nullptr) kept = (int32_t*)(ws + up256(pairs * keep * 4));
    const Select a{held, max_held, keep, recent, next_position, weight_in, weight_out, c.position, position_out, (int32_t*)ws, kept};
    const int most = max_held > keep ? max_held : keep;  // slots that the lanes have to cover
    const unsigned p = (unsigned)pairs, p4 = (unsigned)((pairs + 3) / 4);
    // Up to 512 slots a wavefront per pair.  Up to 1024, and up to 2048, 16 wavefronts as long as the chip takes all pairs at once, one
    // and two workgroups on every unit; with more pairs one.  16 wavefronts / one, us: 500 slots of 8 pairs 8.8 / 8.1, of 4096 112 / 15;
    // 1000 of 8 pairs 9.5 / 13.8, of 256 12.2 / 16.2, of 384 18.3 / 16.7, of 4096 137 / 30; 1500 of 8 pairs 10.2 / 20.9, of 512 19.9 /
    // 24.0, of 640 26.5 / 26.3, of 4096 143 / 45; 2000 of 512 21.2 / 30.2, of 4096 150 / 76.
    // Beyond, 16 wavefronts up to 32 keys per lane (8 pairs of 32000 slots, with the move, 60 us, from memory by 256 threads 290), then from
    // memory.  No more keys per lane than needed, since the compares are what a step of the halving costs (8000 slots: 18 us with 8
    // keys per lane, 25 with 16).
    const bool one = pairs > (most <= 1024 ? 256 : 512);
    if (most <= 512) hipLaunchKernelGGL((select_kernel<1, 8>), dim3(p4), dim3(256), 0, st, c, a);
    else if (one && most <= 768) hipLaunchKernelGGL((select_kernel<1, 12>), dim3(p4), dim3(256), 0, st, c, a);
    else if (one && most <= 1024) hipLaunchKernelGGL((select_kernel<1, 16>), dim3(p4), dim3(256), 0, st, c, a);
    else if (one && most <= 1280) hipLaunchKernelGGL((select_kernel<1, 20>), dim3(p4), dim3(256), 0, st, c, a);
    else if (one && most <= 1536) hipLaunchKernelGGL((select_kernel<1, 24>), dim3(p4), dim3(256), 0, st, c, a);
    else if (one && most <= 2048) hipLaunchKernelGGL((select_kernel<1, 32>), dim3(p4), dim3(256), 0, st, c, a);
    else if (most <= 4096) hipLaunchKernelGGL((select_kernel<16, 4>), dim3(p), dim3(1024), 0, st, c, a);
    else if (most <= 8192) hipLaunchKernelGGL((select_kernel<16, 8>), dim3(p), dim3(1024), 0, st, c, a);
    else if (most <= 16384) hipLaunchKernelGGL((select_kernel<16, 16>), dim3(p), dim3(1024), 0, st, c, a);
    else if (most <= 32768) hipLaunchKernelGGL((select_kernel<16, 32>), dim3(p), dim3(1024), 0, st, c, a);
    else hipLaunchKernelGGL(select_long_kernel, dim3(p), dim3(kLong), 0, st, c, a);
    if (max_held <= keep) return;
    const dim3 grid((unsigned)spans(c, keep)), block(256);
    if (c.hd == 32) hipLaunchKernelGGL(move_kernel<32>, grid, block, 0, st, c, keep, kept);
    if (c.hd == 64) hipLaunchKernelGGL(move_kernel<64>, grid, block, 0, st, c, keep, kept);
    if (c.hd == 128) hipLaunchKernelGGL(move_kernel<128>, grid, block, 0, st, c, keep, kept);
}

}  // namespace kkv8
