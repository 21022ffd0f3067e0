// Attention over the latent cache in its expanded form: keys and values of every head made once for all new tokens, then
// ordinary attention.  For prompts: 2 * (nope + rope + v) operations per pair of tokens and head instead of
// 2 * (2 * latent + rope), at 2 * latent * (nope + v) per slot and head.
//
// Keys and values are kept as fp16, whose 11 bits leave the outputs as exact as their own rounding to bf16 does: over 3000 slots
// keys and values rounded to bf16 put them 4.3e-3 from 64 bits, as fp16 1.7e-3.  fp16 reaches from 2^-14 to 65504; what is outside is brought in
// by exact powers of two: one for each row of queries, one for the keys and one for the values of each head and tile of 64
// slots, 1 wherever the largest lies in 2^-6 .. 2^15 (of queries 2^-2 .. 2^15).  What is far below the largest of its tile, or row, falls below
// 2^-14 and so is off by 2^-25: by 2^-19 (2^-23) of the largest at most.  The part that carries the position stays bf16, as it came.
#include "latent_device.h"

namespace klat {
namespace {

constexpr int kSlots = 64, kRows = 128;  // slots of a tile, rows of a workgroup
// Weights of the softmax are 2^(score - reference + kLift) in fp16: at most 2^14 (kRise on top), full bits down to 2^-20 of the largest.
constexpr float kLift = 6.f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ f32x16 mfma32h(const u32x4 a, const u32x4 b, const f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), f16x2)); }
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 .. 127
// Exponent of a magnitude given by its bits, 0 for zero and what is not finite.
__device__ __forceinline__ int exponent(uint32_t bits) { return bits == 0 || bits >= 0x7f800000u ? 0 : max((int)(bits >> 23), 1) - 127; }
// Exponent by which a tile, or the first part of a query, is brought into the range of fp16; 0 from 2^LEAST to 2^15.
// Not below -120, so that both it and its negative are exponents of numbers of 32 bits: the smallest normal ones are 2^-6 then.
template <int LEAST>
__device__ __forceinline__ int shift_of(uint32_t largest) {
    const int e = exponent(largest);
    return largest == 0 || (e >= LEAST && e < 15) ? 0 : max(e - 8, -120);
}

// Stands for the exponent of values that are all zero: they set no scale.
constexpr int kNoValues = 1 << 20;

// Keys and values of heads head0 .. head0 + heads - 1 of the sequences, or of the prefix.
struct Made {
    int head0, heads, tiles;  // tiles of a sequence at most
    int each;                 // heads that a workgroup makes
    u32x4* kv;                // [sequence, head, tile]: keys, then values, in the order of the matrix instructions
    u32x4* pe;                // [sequence, tile]: the part that carries the position
    int2* shift;              // [sequence, head, tile] exponents taken off the keys and the values
    const u32x4* w;           // w_k and w_v of all heads, see order_kernel
    int per, ranges, row_tiles, part0;
};
// One launch: the first `before` workgroups have the prefix, the others the sequences.  (One behind the other, the smaller launch leaves most
// compute units alone: 5 prompts over a prefix of 8001 slots, 57 and 24 us of expand_kernel, 146 and 18 of expanded_kernel; in one 78 and 157.)
struct Both {
    Made pre, own;
    int before;
};

template <int NOPE, int DV, int DR>
struct Sizes {
    static constexpr int kKeys = kSlots * NOPE / 8, kValues = kSlots * DV / 8, kPe = kSlots * DR / 8;  // units of 16 bytes
    static constexpr int kTile = kKeys + kValues;
    static constexpr int kBytes = (kTile + kPe) * 16;
};

// Slots that the step's tokens see: of a sequence, or of the prefix.
__device__ __forceinline__ int slots_of(const Cache& c, const Step& s, bool prefix, int seq) {
    if (prefix) return c.prefix_len;
    const Seq q = kkv8::sequence(c.max_len, s, seq);
    return q.n_new > 0 ? q.cached + q.n_new : 0;
}

// w_k and w_v in the order in which expand_kernel's matrix instructions take them: [head][32 rows][16 latents][lane], 16 bytes a lane.  Read
// where they lie, a wavefront's rows are 32 lines of which it uses 32 bytes at a time: expand_kernel then waits for L2 (8192 slots of 32
// heads 152 us, from this copy 87 and 5 for the copy).  One workgroup per 32 rows.
__global__ __launch_bounds__(256) void order_kernel(Heads h, int latent, u32x4* out) {
    const int lane = threadIdx.x & 63, blocks = (h.nope + h.v) / 32, head = blockIdx.x / blocks, block = blockIdx.x % blocks;
    const bool key = block < h.nope / 32;
    const int row = (key ? block : block - h.nope / 32) * 32 + (lane & 31);
    const uint16_t* from = (key ? h.w_k + head * h.w_k_head : h.w_v + head * h.w_v_head) + (int64_t)row * latent + (lane >> 5) * 8;
    u32x4* to = out + (int64_t)blockIdx.x * (latent / 16) * 64 + lane;
    for (int f = wave_number() * 4; f < latent / 16; f += 16) {
        u32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *(const u32x4*)(from + (f + i) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[(f + i) * 64] = x[i];
    }
}

// Keys and values of 128 slots for some heads, one after the other: the latents lie in LDS (up to 128 KiB) for all of them, w_k
// and w_v come from L2 into registers, 64 latents ahead.  A wavefront makes 32 elements of the keys (w_k c^T: a lane has one
// slot and four elements side by side) and 32 of the values (c w_v^T: one element and eight slots, in the order in which the weights of the
// softmax come out of the scores), which is how the attention's matrix instructions take them.  8003 slots of 32 heads, latents of 512: 67 GFLOP in
// 87 us, 0.77 PFLOP/s, matrix cores 34 % busy; every workgroup asks L2 for all of w_k and w_v of its heads.
constexpr int expand_waves(int nope, int v) { return (nope > v ? nope : v) / 32; }  // of 64 slots
// Wavefronts of a SIMD: as many workgroups as the LDS holds.
constexpr int expand_occupancy(int latent, int waves) { return waves * 2 * (latent == 512 ? 1 : latent == 256 ? 2 : 4) >= 8 ? 2 : 1; }
template <int DC, int NOPE, int DV>
__global__ __launch_bounds__(128 * expand_waves(NOPE, DV), expand_occupancy(DC, expand_waves(NOPE, DV))) void expand_kernel(Cache c, Step s, Heads h, Both both) {
    constexpr int G = DC / 64, KEYS = NOPE / 32, VALUES = DV / 32, WAVES = expand_waves(NOPE, DV), TILE = kSlots * (NOPE + DV) / 8;
    __shared__ u32x4 lds[G * 128 * 8];
    __shared__ uint32_t seen[2][2][WAVES];  // [odd and even heads][tile of 64][wavefront]
    __shared__ uint32_t largest[2][2];  // [keys, values][tile of 64]
    __shared__ int bad[128];
    const int lane = threadIdx.x & 63, wave = wave_number() % WAVES, half = wave_number() / WAVES, col = lane & 31, grp = lane >> 5;
    const bool prefix = (int)blockIdx.x < both.before;
    const Made& m = prefix ? both.pre : both.own;
    const int block = prefix ? blockIdx.x : blockIdx.x - both.before, pairs_of = (m.tiles + 1) / 2;
    const int pair = block % pairs_of, rest = block / pairs_of;
    const int seq = prefix ? 0 : rest % c.n_seq, first = (prefix ? rest : rest / c.n_seq) * m.each;
    const int total = slots_of(c, s, prefix, seq), j0 = pair * 128;
    if (j0 >= total) return;
    const int width = c.latent + c.rope;
    const uint16_t* C = prefix ? c.prefix : c.rows + (int64_t)seq * c.max_len * width;
    {
        const uint32_t at = lds_address(lds);
        const int in8 = lane >> 3;
        for (int i = wave_number(); i < 16; i += 2 * WAVES) {
            const int slot = i * 8 + in8;
            const uint32_t from = (uint32_t)min(j0 + slot, total - 1) * (uint32_t)(width * 2) + ((lane & 7) ^ twist(slot)) * 16;
#pragma unroll
            for (int g = 0; g < G; ++g) copy_to_lds((const uint8_t*)C + g * 128, from, __builtin_amdgcn_readfirstlane(at + g * 16384 + i * 1024));
        }
    }
    if (first == 0) {  // the part that carries the position, once
        const int units = c.rope / 8;
        for (int i = threadIdx.x; i < 128 * units; i += 128 * WAVES) {
            const int l = i & 63, unit = i >> 6;  // [tile][32 slots][16 elements][lane]
            const int f = unit % (units / 2), slot = unit / (units / 2) * 32 + (l & 31);
            if (j0 + slot / 64 * 64 < total) {
                const u32x4 x = *(const u32x4*)(C + (int64_t)min(j0 + slot, total - 1) * width + c.latent + f * 16 + (l >> 5) * 8);
                m.pe[(((int64_t)seq * m.tiles + pair * 2 + slot / 64) * (units / 2) * 2 + (slot / 32 & 1) * (units / 2) + f) * 64 + l] = x;
            }
        }
    }
    const bool keys = wave < KEYS, values = wave < VALUES;
    // past the last head the last one is asked for again, and not used
    constexpr int BLOCK = DC / 16 * 64;
    const auto from = [&](int head) { return m.w + (int64_t)(m.head0 + min(head, m.heads - 1)) * (KEYS + VALUES) * BLOCK + lane; };
    const int block_k = (keys ? wave : 0) * BLOCK, block_v = (KEYS + (values ? wave : 0)) * BLOCK;
    u32x4 wk[4], wv[4];
    auto load = [&](const u32x4* p, int g) {
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            wk[f] = p[block_k + (g * 4 + f) * 64];
            wv[f] = p[block_v + (g * 4 + f) * 64];
        }
    };
    load(from(first), 0);
    uint32_t at[4];  // unit 2 * f + grp of the lane's slot
#pragma unroll
    for (int f = 0; f < 4; ++f) at[f] = lds_address(lds) + (uint32_t)((half * 64 + col) * 128 + ((2 * f + grp) ^ twist(col)) * 16);
    wait_copies<0>();
    __syncthreads();
    for (int head = first; head < min(first + m.each, m.heads); ++head) {
        f32x16 k[2], v[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) k[t][i] = v[t][i] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            u32x4 a[4], b[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                a[f] = wk[f];
                b[f] = wv[f];
            }
            if (g + 1 < G) load(from(head), g + 1);
            else load(from(head + 1), 0);
#pragma unroll
            for (int f = 0; f < 4; ++f)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 x = read_lds(at[f] + g * 16384 + t * 4096);
                    k[t] = mfma32(a[f], x, k[t]);
                    v[t] = mfma32(x, b[f], v[t]);
                }
        }
        // Whether every tile is within the range of fp16 as it is: nothing from 2^15 on (infinities and NaN among that), something from 2^-6 on.
        uint32_t a = 0, b = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            a = max(a, __float_as_uint(k[i >> 4][i & 15]) & 0x7fffffffu);
            b = max(b, __float_as_uint(v[i >> 4][i & 15]) & 0x7fffffffu);
        }
        constexpr uint32_t kBig = (127u + 15) << 23, kSome = (127u - 6) << 23;
        const uint32_t mine = (keys ? (__any(a >= kBig) ? 1u : 0u) | (__any(a >= kSome) ? 2u : 0u) : 0u) |
                              (values ? (__any(b >= kBig) ? 4u : 0u) | (__any(b >= kSome) ? 8u : 0u) : 0u);
        if (lane == 0) seen[head & 1][half][wave] = mine;
        __syncthreads();
        uint32_t all[2] = {0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            all[0] |= seen[head & 1][0][w];
            all[1] |= seen[head & 1][1][w];
        }
        const bool plain = all[0] == 10u && all[1] == 10u;
        if (!plain) {  // the exponents of the largest, and the slots with something that is not finite
            if (threadIdx.x < 4) largest[threadIdx.x >> 1][threadIdx.x & 1] = 0;
            if (threadIdx.x < 128) bad[threadIdx.x] = 0;  // (a workgroup has at least 128 threads)
            __syncthreads();
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint32_t a = 0, b = 0;
                bool odd = false;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t x = __float_as_uint(k[t][i]) & 0x7fffffffu, y = __float_as_uint(v[t][i]) & 0x7fffffffu;
                    odd |= x >= 0x7f800000u;
                    a = max(a, x >= 0x7f800000u ? 0u : x);
                    if (y >= 0x7f800000u) {
                        if (values) bad[half * 64 + t * 32 + row_of(i, grp)] = 1;
                        v[t][i] = 0.f;
                    } else {
                        b = max(b, y);
                    }
                }
                if (odd && keys) bad[half * 64 + t * 32 + col] = 1;
                if (keys) atomicMax(&largest[0][half], a);
                if (values) atomicMax(&largest[1][half], b);
            }
            __syncthreads();
        }
        const int64_t tile = ((int64_t)seq * m.heads + head) * m.tiles + pair * 2 + half;
        const bool there = j0 + half * 64 < total;
        u32x4* to = m.kv + tile * TILE;
        const int down[2] = {plain ? 0 : shift_of<-6>(largest[0][half]), plain ? 0 : shift_of<-6>(largest[1][half])};
        if (there && wave == 0 && lane == 0) m.shift[tile] = make_int2(down[0], !plain && largest[1][half] == 0 ? kNoValues : down[1]);
        const float fk = power(-down[0]), fv = power(-down[1]);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (there && keys) {
                const bool out = !plain && bad[half * 64 + t * 32 + col] != 0;  // then no row that sees the slot stays finite
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    u32x2 x;
                    x.x = out ? 0x7e007e00u : pack_f16(k[t][4 * i] * fk, k[t][4 * i + 1] * fk);
                    x.y = out ? 0x7e007e00u : pack_f16(k[t][4 * i + 2] * fk, k[t][4 * i + 3] * fk);
                    ((u32x2*)(to + (t * (NOPE / 16) + wave * 2 + (i >> 1)) * 64 + col + 32 * (i & 1)))[grp] = x;
                }
            }
            if (there && values) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    u32x4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = pack_f16(v[t][8 * u + 2 * i] * fv, v[t][8 * u + 2 * i + 1] * fv);
                    to[kSlots * NOPE / 8 + ((t * 2 + u) * VALUES + wave) * 64 + lane] = x;
                }
            }
        }
        if (!plain) __syncthreads();  // `largest` and `bad` may be set anew
    }
}

// Attention of 128 rows (32 a wavefront) of one head: scores and sums transposed, so that a lane has one row, its softmax needs no
// exchange but one between two lanes, and the weights are the second operand of the sums as they stand.  Tiles come in turn into two
// buffers, without registers.  2 prompts of about 4000 tokens, 32 heads: 335 GFLOP in 359 us, 0.93 PFLOP/s, 75 % of what a large library product reaches;
// matrix cores half busy, the clock at the card's power limit.
template <int NOPE, int DV, int DR>
__global__ __launch_bounds__(256, 2) void expanded_kernel(Cache c, Step s, Heads h, Attend a, Both both, Parts parts) {
    typedef Sizes<NOPE, DV, DR> Z;
    constexpr int KF = NOPE / 16, PF = DR / 16, VB = DV / 32;
    __shared__ u32x4 lds[2][Z::kBytes / 16];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5;
    const bool prefix = (int)blockIdx.x < both.before;
    const Made& m = prefix ? both.pre : both.own;
    const int block = prefix ? blockIdx.x : blockIdx.x - both.before, pairs = (prefix ? 1 : c.n_seq) * m.heads;
    const int pair = block % pairs, rest = block / pairs;
    const int seq = pair / m.heads, head = pair % m.heads;
    const int range = rest % m.ranges, tile = m.row_tiles - 1 - rest / m.ranges;  // those that see the most slots first
    Seq q{0, s.n_rows, 0};
    if (!prefix) q = kkv8::sequence(c.max_len, s, seq);
    const int rows = q.n_new, row0 = tile * kRows, first = range * m.per;
    if (row0 >= rows) return;
    const int sees = prefix ? c.prefix_len : q.cached + min(row0 + kRows, rows);  // slots that the last row sees
    const int end = min(first + m.per, sees);
    if (first >= end) return;
    const int r = row0 + wave * 32 + col, mine = min(r, rows - 1);
    const int limit = prefix ? c.prefix_len : q.cached + mine + 1;
    const int wave_least = prefix ? c.prefix_len : q.cached + min(row0 + wave * 32, rows - 1) + 1;
    const int wave_most = prefix ? c.prefix_len : q.cached + min(row0 + wave * 32 + 31, rows - 1) + 1;
    const bool active = row0 + wave * 32 < rows;
    const uint8_t* kv = (const uint8_t*)(m.kv + (int64_t)pair * m.tiles * Z::kTile);
    const uint8_t* pe = (const uint8_t*)(m.pe + (int64_t)seq * m.tiles * Z::kPe);
    const int2* shift = m.shift + (int64_t)pair * m.tiles;
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane(lds_address(&lds[0][0]) + wave * 1024);
    auto copy = [&](int buf, int j0) {
        const uint8_t* from = kv + (int64_t)(j0 / kSlots) * (Z::kTile * 16);
#pragma unroll
        for (int i = 0; i < Z::kTile / 256; ++i) copy_to_lds(from + i * 4096, threadIdx.x * 16, lds_at + buf * Z::kBytes + i * 4096);
        const uint8_t* from_pe = pe + (int64_t)(j0 / kSlots) * (Z::kPe * 16);
#pragma unroll
        for (int i = 0; i < Z::kPe / 256; ++i) copy_to_lds(from_pe + i * 4096, threadIdx.x * 16, lds_at + buf * Z::kBytes + Z::kTile * 16 + i * 4096);
    };
    copy(0, first);
    int2 down = shift[first / kSlots];

    u32x4 qf[KF], qp[PF];
    int query_scale;  // exponent taken off the row's first part
    {
        const uint16_t* p = a.q.p + (int64_t)(q.row0 + mine) * a.q.row + (int64_t)(m.head0 + head) * a.q.head + grp * 8;
        uint32_t top = 0;
#pragma unroll
        for (int f = 0; f < KF; ++f) {
            qf[f] = *(const u32x4*)(p + f * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, max(qf[f][i] << 16 & 0x7fffffffu, qf[f][i] & 0x7fff0000u));
        }
#pragma unroll
        for (int f = 0; f < PF; ++f) qp[f] = *(const u32x4*)(p + NOPE + f * 16);
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
        query_scale = shift_of<-2>(top);
#pragma unroll
        for (int f = 0; f < KF; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                qf[f][i] = pack_f16(__builtin_amdgcn_ldexpf(bf_lo(qf[f][i]), -query_scale), __builtin_amdgcn_ldexpf(bf_hi(qf[f][i]), -query_scale));
#pragma unroll
        for (int f = 0; f < KF; ++f) asm volatile("" : "+v"(qf[f]));  // waited for here, not in the loop
#pragma unroll
        for (int f = 0; f < PF; ++f) asm volatile("" : "+v"(qp[f]));
    }
    f32x16 acc[VB];
#pragma unroll
    for (int b = 0; b < VB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
    const bool queries_scaled = __any(query_scale != 0);
    float ref = kEmpty, sum = 0.f;
    int scale = 0;     // exponent of the row's sums: that of the values they were last made of
    bool odd = false;  // whether any tile so far had one (the same for the wavefront)
    const int within = min(limit, end) - 4 * grp;
    int buf = 0;
    for (int j0 = first; j0 < end; j0 += kSlots, buf ^= 1) {
        wait_copies<0>();
        __syncthreads();  // the slots are there, and nobody reads the other buffer any more
        const int2 now_down = down;
        if (j0 + kSlots < end) {
            copy(buf ^ 1, j0 + kSlots);
            down = shift[(j0 + kSlots) / kSlots];
        }
        if (!active || j0 >= wave_most) continue;
        f32x16 z[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[t][i] = 0.f;
#pragma unroll
            for (int f = 0; f < KF; ++f) z[t] = mfma32h(lds[buf][(t * KF + f) * 64 + lane], qf[f], z[t]);
        }
        // What was taken off queries and keys comes back, before the part that carries the position is added as it is.
        const int key_scale = __builtin_amdgcn_readfirstlane(now_down.x);
        if (queries_scaled || key_scale != 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[t][i] = __builtin_amdgcn_ldexpf(z[t][i], query_scale + key_scale);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int f = 0; f < PF; ++f) z[t] = mfma32(lds[buf][Z::kTile + (t * PF + f) * 64 + lane], qp[f], z[t]);
        if (j0 + kSlots > wave_least || j0 + kSlots > end) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (t * 32 + row_of(i, 0) >= within - j0) z[t][i] = -__builtin_inff();
        }
        float top = z[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, z[t][i]);
        top *= a.qscale;
        if (__any(top > ref + kRise)) {
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float now = top > ref + kRise ? ceilf(top) : ref;
            const float f = __builtin_amdgcn_exp2f(ref - now);
            ref = now;
            sum *= f;
#pragma unroll
            for (int b = 0; b < VB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[b][i] *= f;
        }
        exponents_of_rows(ref, -kLift, a.qscale, [&](auto&& of) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[t][i] = of(z[t][i]);
        });
        u32x4 w[4];
        float part = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(z[u >> 1][(u & 1) * 8 + i]);
                part += p[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) w[u][i] = pack_f16(p[2 * i], p[2 * i + 1]);
        }
        sum += part;
        // Sums go over to the exponent of the tile's values, up or down and exactly, where one of the tile's weights is not 0 in fp16, so that
        // the weights keep their bits, and values that hardly count, or that the row does not see, change nothing for it.  Below sums that
        // would leave 32 bits (2^64 times the tile's and more) the tile counts as 0.
        const int tile_scale = __builtin_amdgcn_readfirstlane(now_down.y);
        if (odd || tile_scale != 0) {
            odd = true;
            uint32_t any = 0, largest = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) any |= w[u][i];
            any |= (uint32_t)__shfl_xor((int)any, 32, 64);
            const bool moves = any != 0 && scale != tile_scale && tile_scale != kNoValues;
            if (__any(moves)) {
#pragma unroll
                for (int b = 0; b < VB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) largest = max(largest, __float_as_uint(acc[b][i]) & 0x7fffffffu);
                largest = max(largest, (uint32_t)__shfl_xor((int)largest, 32, 64));
                const int to = !moves ? scale : largest == 0 ? tile_scale : max(tile_scale, scale + exponent(largest) - 100);
#pragma unroll
                for (int b = 0; b < VB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[b][i] = __builtin_amdgcn_ldexpf(acc[b][i], scale - to);
                scale = to;
                if (moves && to != tile_scale) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) w[u] = u32x4{0u, 0u, 0u, 0u};
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int b = 0; b < VB; ++b) acc[b] = mfma32h(lds[buf][Z::kKeys + (u * VB + b) * 64 + lane], w[u], acc[b]);
    }
    sum += __shfl_xor(sum, 32, 64);
    const float up = power(scale);
    if (parts.all > 1) {
        if (r < rows) {
            // a range's mean, not its sum: no larger than its values are
            const float mean = sum == 0.f ? 0.f : 1.f / sum;
            const int64_t at = ((int64_t)(q.row0 + r) * h.n + m.head0 + head) * parts.all + m.part0 + range;
#pragma unroll
            for (int b = 0; b < VB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = acc[b][4 * i + j] * mean * up;
                    *(f32x4*)(parts.acc + at * DV + b * 32 + row_of(4 * i, grp)) = y;
                }
            if (grp == 0) parts.ml[at] = make_float2(ref, sum);
        }
        return;
    }
    // The rows go through the buffers, which are done with, so that each leaves in one piece; 16-byte pieces lie at an xor of the row.
    const float inv = 1.f / sum;
    constexpr int PPR = DV / 8;  // pieces of a row
    __syncthreads();
    u32x4* out = &lds[0][0] + wave * 32 * PPR;
    static_assert(4 * 32 * PPR * 16 <= 2 * Z::kBytes, "the rows fit the buffers");
#pragma unroll
    for (int b = 0; b < VB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x2 x;
            x.x = pack_bf16(acc[b][4 * i] * inv * up, acc[b][4 * i + 1] * inv * up);
            x.y = pack_bf16(acc[b][4 * i + 2] * inv * up, acc[b][4 * i + 3] * inv * up);
            ((u32x2*)(out + col * PPR + ((b * 4 + i) ^ (col % PPR))))[grp] = x;
        }
#pragma unroll
    for (int i = 0; i < PPR / 2; ++i) {
        const int in = i * (64 / PPR) + lane / PPR, row = row0 + wave * 32 + in;
        if (row < rows)
            *(u32x4*)(a.out.p + (int64_t)(q.row0 + row) * a.out.row + (int64_t)(m.head0 + head) * a.out.head + lane % PPR * 8) = out[in * PPR + (lane % PPR ^ in % PPR)];
    }
}

// Rows whose slots were cut into parts: the parts' means with their shares of the weights, brought to the largest reference.  One wavefront per
// row and 64 / (DV / 4) heads.
template <int DV>
__global__ __launch_bounds__(256) void merge_kernel(Cache c, Step s, Heads h, RowsOut out, Parts parts) {
    constexpr int LANES = DV / 4, HEADS = 64 / LANES;
    const int lane = threadIdx.x & 63, groups = (h.n + HEADS - 1) / HEADS;
    const int64_t item = (int64_t)blockIdx.x * 4 + wave_number();
    const int row = (int)(item / groups), head = (int)(item % groups) * HEADS + lane / LANES;
    if (row >= s.n_rows) return;
    Seq q;
    int token;
    const int seq = seq_of_row(c, s, row, &token, &q);
    if (seq < 0 || head >= h.n) return;
    const int own = (q.cached + token + parts.per) / parts.per;  // parts of the slots that the row sees
    const int n = own + parts.all - parts.own;
    const int64_t at = ((int64_t)row * h.n + head) * parts.all;
    float ref = kEmpty, sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
        const float2 ml = parts.ml[at + (k < own ? k : parts.own + k - own)];
        const float now = fmaxf(ref, ml.x);
        sum = __builtin_fmaf(ml.y, __builtin_amdgcn_exp2f(ml.x - now), sum * __builtin_amdgcn_exp2f(ref - now));
        ref = now;
    }
    const float inv = 1.f / sum;
    for (int k = 0; k < n; ++k) {
        const int64_t i = at + (k < own ? k : parts.own + k - own);
        const float2 ml = parts.ml[i];
        const float f = ml.y * __builtin_amdgcn_exp2f(ml.x - ref) * inv;
        const f32x4 y = *(const f32x4*)(parts.acc + i * DV + lane % LANES * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(y[j], f, x[j]);
    }
    u32x2 w;
    w.x = pack_bf16(x[0], x[1]);
    w.y = pack_bf16(x[2], x[3]);
    *(u32x2*)(out.p + (int64_t)row * out.row + (int64_t)head * out.head + lane % LANES * 4) = w;
}

// How a step is run, from its sizes and bounds.
struct Plan {
    Made own, pre;
    Parts parts;
    int heads;  // at a time
    int64_t o_ml, o_w, o_own_kv, o_own_pe, o_own_shift, o_pre_kv, o_pre_pe, o_pre_shift, bytes;
    int64_t own_groups, pre_groups, own_expand, pre_expand, merges;  // workgroups of the launches of a set of heads
};

int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

// Slots of a range, so that about `aim` workgroups get 512 slots and more.  Sequences: 1024, since tiles late in a long one see the most slots and
// would be left alone at the end (3 chunks of 267 to 800 tokens behind up to 6001 slots, 240 workgroups whole: 140 us, in four ranges 83 and 7 to
// merge).  The prefix, of which all tiles see the same: 512 (5 prompts of 97 to 300 tokens over 8001 slots, in two ranges 140 and 9, in four 140 and 14).
int range_of(int64_t most, int64_t groups, int64_t aim) {
    int64_t n = groups > 0 ? aim / groups : 1;
    n = min(n, most / 512);
    if (n < 1) n = 1;
    return (int)(((most + n - 1) / n + kSlots - 1) / kSlots * kSlots);
}

// Heads that one workgroup of expand_kernel makes: the fewest rounds of a workgroup per compute unit, each of its heads and, about as
// long as one of them, its latents' way into LDS.
int heads_each(int64_t tiles, int heads) {
    int best = 1;
    int64_t least = INT64_MAX;
    for (int n = 1; n <= heads && n <= 32; ++n) {
        const int64_t rounds = (tiles * ((heads + n - 1) / n) + 255) / 256, cost = rounds * (n + 1);
        if (cost < least) {
            least = cost;
            best = n;
        }
    }
    return best;
}

Plan plan(const Cache& c, const Step& s, const Heads& h) {
    Plan p{};
    if (s.n_rows == 0) return p;
    const int64_t most = min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len);
    const int64_t tiles = (most + kSlots - 1) / kSlots, pre_tiles = (c.prefix_len + kSlots - 1) / kSlots;
    // Keys and values of as many heads at a time as keep them within the last-level cache of 256 MiB, one at least.
    const int64_t per_head = (c.n_seq * tiles + pre_tiles) * kSlots * (h.nope + h.v) * 2;
    const int64_t fit = ((int64_t)192 << 20) / per_head, rounds = fit < 1 ? h.n : (h.n + fit - 1) / fit;
    p.heads = (int)((h.n + rounds - 1) / rounds);
    const int64_t own_rows = (s.max_new + kRows - 1) / kRows, pre_rows = ((int64_t)s.n_rows + kRows - 1) / kRows;
    // row tiles that are there: about half a tile over each sequence's share of the rows
    const int64_t about = min(c.n_seq * own_rows, (int64_t)s.n_rows / kRows + (c.n_seq + 1) / 2 + 1);
    p.own.tiles = (int)tiles;
    p.own.row_tiles = (int)own_rows;
    p.own.per = range_of(most, about * p.heads, 1024);
    p.own.ranges = (int)((most + p.own.per - 1) / p.own.per);
    p.parts.per = p.own.per;
    p.parts.own = p.parts.all = p.own.ranges;
    p.own.each = heads_each(c.n_seq * ((tiles + 1) / 2), p.heads);
    p.own_expand = c.n_seq * ((tiles + 1) / 2) * ((p.heads + p.own.each - 1) / p.own.each);
    p.own_groups = (int64_t)c.n_seq * p.heads * own_rows * p.own.ranges;
    p.parts.pre_per = 1;
    if (c.prefix_len > 0) {
        p.pre.tiles = (int)pre_tiles;
        p.pre.row_tiles = (int)pre_rows;
        p.pre.per = range_of(c.prefix_len, pre_rows * p.heads, 512);
        p.pre.ranges = (int)((c.prefix_len + p.pre.per - 1) / p.pre.per);
        p.pre.part0 = p.parts.own;
        p.parts.pre_per = p.pre.per;
        p.parts.all += p.pre.ranges;
        p.pre.each = heads_each((pre_tiles + 1) / 2, p.heads);
        p.pre_expand = ((pre_tiles + 1) / 2) * ((p.heads + p.pre.each - 1) / p.pre.each);
        p.pre_groups = (int64_t)p.heads * pre_rows * p.pre.ranges;
    }
    const int64_t items = p.parts.all > 1 ? (int64_t)s.n_rows * h.n * p.parts.all : 0;
    const int per_wave = 64 / (h.v / 4);
    p.merges = items > 0 ? ((int64_t)s.n_rows * ((h.n + per_wave - 1) / per_wave) + 3) / 4 : 0;
    const int64_t tile = (int64_t)kSlots * (h.nope + h.v) * 2, pe = (int64_t)kSlots * c.rope * 2;
    int64_t o = up256(items * h.v * 4);
    auto take = [&](int64_t bytes) {
        const int64_t at = o;
        o += up256(bytes);
        return at;
    };
    p.o_ml = take(items * 8);
    p.o_w = take((int64_t)h.n * (h.nope + h.v) * c.latent * 2);
    p.o_own_kv = take(c.n_seq * p.heads * tiles * tile);
    p.o_own_pe = take(c.n_seq * tiles * pe);
    p.o_own_shift = take(c.n_seq * p.heads * tiles * 8);
    p.o_pre_kv = take(p.heads * pre_tiles * tile);
    p.o_pre_pe = take(pre_tiles * pe);
    p.o_pre_shift = take(p.heads * pre_tiles * 8);
    p.bytes = o;
    return p;
}

struct Call {
    hipStream_t st;
    Cache c;
    Step s;
    Heads h;
    Attend a;
    Parts parts;
};

template <int DC, int NOPE, int DV>
void launch_expand(const Call& k, const Both& m, int64_t groups) {
    hipLaunchKernelGGL((expand_kernel<DC, NOPE, DV>), dim3((unsigned)groups), dim3(128 * expand_waves(NOPE, DV)), 0, k.st, k.c, k.s, k.h, m);
}
template <int NOPE, int DV>
void launch_expand_sizes(const Call& k, const Both& m, int64_t groups) {
    if (k.c.latent == 128) launch_expand<128, NOPE, DV>(k, m, groups);
    if (k.c.latent == 256) launch_expand<256, NOPE, DV>(k, m, groups);
    if (k.c.latent == 512) launch_expand<512, NOPE, DV>(k, m, groups);
}
template <int NOPE, int DV>
void launch_attention(const Call& k, const Both& m, int64_t groups) {
    const dim3 grid((unsigned)groups), block(256);
    if (k.c.rope == 32) hipLaunchKernelGGL((expanded_kernel<NOPE, DV, 32>), grid, block, 0, k.st, k.c, k.s, k.h, k.a, m, k.parts);
    if (k.c.rope == 64) hipLaunchKernelGGL((expanded_kernel<NOPE, DV, 64>), grid, block, 0, k.st, k.c, k.s, k.h, k.a, m, k.parts);
}
template <int NOPE, int DV>
void launch_set(const Call& k, Both m, int64_t pre_expand, int64_t own_expand, int64_t pre_groups, int64_t own_groups) {
    m.before = (int)pre_expand;
    launch_expand_sizes<NOPE, DV>(k, m, pre_expand + own_expand);
    m.before = (int)pre_groups;
    launch_attention<NOPE, DV>(k, m, pre_groups + own_groups);
}
template <int NOPE>
void launch_nope(const Call& k, const Both& m, int64_t pre_expand, int64_t own_expand, int64_t pre_groups, int64_t own_groups) {
    if (k.h.v == 32) launch_set<NOPE, 32>(k, m, pre_expand, own_expand, pre_groups, own_groups);
    if (k.h.v == 64) launch_set<NOPE, 64>(k, m, pre_expand, own_expand, pre_groups, own_groups);
    if (k.h.v == 128) launch_set<NOPE, 128>(k, m, pre_expand, own_expand, pre_groups, own_groups);
}

}  // namespace

int64_t expanded_workspace(const Cache& c, const Step& s, const Heads& h) { return plan(c, s, h).bytes; }

bool expanded_fits(const Cache& c, const Step& s, const Heads& h) {
    const Plan p = plan(c, s, h);
    return launchable(p.own_groups + p.pre_groups, 256) && launchable(p.own_expand + p.pre_expand, 128 * expand_waves(h.nope, h.v)) &&
           launchable(p.merges, 256);
}

void launch_expanded(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const Attend& a) {
    Plan p = plan(c, s, h);
    p.parts.acc = (float*)a.ws;
    p.parts.ml = (float2*)(a.ws + p.o_ml);
    const Call k{st, c, s, h, a, p.parts};
    hipLaunchKernelGGL(order_kernel, dim3((unsigned)(h.n * (h.nope + h.v) / 32)), dim3(256), 0, st, h, c.latent, (u32x4*)(a.ws + p.o_w));
    for (int head = 0; head < h.n; head += p.heads) {
        const int heads = min(p.heads, h.n - head);
        auto made = [&](Made m, int64_t kv, int64_t pe, int64_t shift) {
            m.head0 = head;
            m.heads = heads;
            m.kv = (u32x4*)(a.ws + kv);
            m.pe = (u32x4*)(a.ws + pe);
            m.shift = (int2*)(a.ws + shift);
            m.w = (const u32x4*)(a.ws + p.o_w);
            return m;
        };
        // the last set of heads may be smaller: its launches have the workgroups of its own heads
        auto of_heads = [&](int64_t groups) { return groups / p.heads * heads; };
        auto of_each = [&](int64_t groups, int each) { return groups / ((p.heads + each - 1) / each) * ((heads + each - 1) / each); };
        const Both both{made(p.pre, p.o_pre_kv, p.o_pre_pe, p.o_pre_shift), made(p.own, p.o_own_kv, p.o_own_pe, p.o_own_shift), 0};
        const int64_t pre_expand = c.prefix_len > 0 ? of_each(p.pre_expand, p.pre.each) : 0, own_expand = of_each(p.own_expand, p.own.each);
        const int64_t pre_groups = of_heads(p.pre_groups), own_groups = of_heads(p.own_groups);
        if (h.nope == 32) launch_nope<32>(k, both, pre_expand, own_expand, pre_groups, own_groups);
        if (h.nope == 64) launch_nope<64>(k, both, pre_expand, own_expand, pre_groups, own_groups);
        if (h.nope == 128) launch_nope<128>(k, both, pre_expand, own_expand, pre_groups, own_groups);
    }
    if (p.merges > 0) {
        const dim3 grid((unsigned)p.merges), block(256);
        if (h.v == 32) hipLaunchKernelGGL(merge_kernel<32>, grid, block, 0, st, c, s, h, a.out, p.parts);
        if (h.v == 64) hipLaunchKernelGGL(merge_kernel<64>, grid, block, 0, st, c, s, h, a.out, p.parts);
        if (h.v == 128) hipLaunchKernelGGL(merge_kernel<128>, grid, block, 0, st, c, s, h, a.out, p.parts);
    }
}

}  // namespace klat
