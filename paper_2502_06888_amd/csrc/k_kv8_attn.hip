// Attention over the 8-bit key-value cache.
//
// o = softmax(q K^T) V with K and V dequantised on the way into the matrix instructions: a scale is a power of two, so
// code * scale is exact in bf16 and the conversion instruction applies it for nothing.  Products are bf16, sums and
// softmax statistics fp32, base-2 exponentials with log2(e) folded into the factor of the scores.
#include "kv8_kernels.h"

namespace kkv8 {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kEmpty = -1.0e30f;  // finite stand-in for "no slot seen yet"
// The reference of a running softmax lies kAbove over the largest score at the time it was set, and is set anew once a
// score comes closer than kNear: the sums are not rescaled for every new maximum, and as weights stay below 2^-kNear,
// the sums of 2^20 slots of any finite values stay finite.
constexpr float kAbove = 28.f, kNear = 20.f;

__device__ __forceinline__ int seq_of_row(const Step& s, int n_seq, int row) {
    if (s.row_offsets == nullptr) return row / s.max_new;
    int lo = 0, hi = n_seq - 1;  // last sequence whose rows begin at or before `row`
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (s.row_offsets[mid] <= row) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ bf16x8 as_bf16x8(const u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ f32x4 mfma16(const u32x4 a, const u32x4 b, const f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
// Eight codes (two words) as bf16 times `scale`.
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi, float scale) {
    return u32x4{widen2<false>(lo, scale), widen2<true>(lo, scale), widen2<false>(hi, scale), widen2<true>(hi, scale)};
}
// Bit 7 of each byte of four codes that is NaN (0x7f or 0xff).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// Bytes of four words transposed: o[b] holds byte b of a[0], a[1], a[2], a[3].
__device__ __forceinline__ void transpose4(const uint32_t (&a)[4], uint32_t (&o)[4]) {
    const uint32_t t0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), t1 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
    const uint32_t t2 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), t3 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
    o[0] = __builtin_amdgcn_perm(t2, t0, 0x05040100u);
    o[1] = __builtin_amdgcn_perm(t2, t0, 0x07060302u);
    o[2] = __builtin_amdgcn_perm(t3, t1, 0x05040100u);
    o[3] = __builtin_amdgcn_perm(t3, t1, 0x07060302u);
}

// ---- few new tokens: bound by the bytes of the cache ----------------------------------------------------
//
// One workgroup of four wavefronts per (sequence, key-value head, range of slots); all rows (token, query head of the
// group) of the pair share what is read, in tiles of 8.  A wavefront takes 32 slots at a time, in two tiles of 16:
//   scores    S^T[slot][row] = K Q^T, 16x16x32: lane l holds row l%16 and slots 4*(l/16)..+3 of each tile;
//   sums      O[row][element] = P V with the eight weights a lane holds as its eight steps of the reduction, so that the
//             weights never leave their lane: V is read by slots in that order, byte-transposed in registers.
// A tile of 16 matrix rows serves 8 rows twice: the second half multiplies what rounding the weights to bf16 left over,
// so the weights count with 16 bits at no matrix cost.
struct Split {
    int per, ranges;    // slots of a range (a multiple of 128), ranges of a sequence at most
    int tile_rows;      // rows the buffers below hold per pair
    int score_stride;   // slots a row of `scores` holds, a multiple of 32
    float* acc;         // [pair, range, row, hd] unnormalised sums; with float2 `ml` (reference, sum of weights)
    float2* ml;
    float* scores;      // [pair, row, slot] products q . K
    float2* final_ml;   // [pair, row] of the whole sequence: reference, 1 / sum of weights
};

template <int HD, int NT, bool SCORES>
__global__ __launch_bounds__(256, NT == 1 ? 4 : 3) void decode_kernel(Cache c, Step s, Attend a, Split sp) {
    constexpr int KW = HD / 16;             // words of a K row that a lane holds: HD/4 bytes
    constexpr int VT = HD / 16;             // tiles of 16 elements of the sums
    constexpr int VW = VT >= 4 ? VT / 4 : 1;  // words of a V row that a lane holds: VT bytes
    __shared__ float sm_o[4][NT * 8][HD];
    __shared__ float2 sm_ml[4][NT * 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    const int range = blockIdx.x % sp.ranges, pair = blockIdx.x / sp.ranges;
    const int seq = pair / c.Hkv, hk = pair % c.Hkv, G = a.Hq / c.Hkv;
    const Seq q = sequence(c, s, seq);
    const int len = q.cached + q.n_new, rows = q.n_new * G;
    const int first = range * sp.per, end = min(first + sp.per, len);
    if (rows == 0 || first >= end) return;
    const int64_t base = (int64_t)seq * c.Hkv + hk;
    const uint8_t *K = c.codes[0] + base * c.max_len * HD, *V = c.codes[1] + base * c.max_len * HD;
    const float *ks = c.scale[0] + base * (c.max_len >> c.logb), *vs = c.scale[1] + base * (c.max_len >> c.logb);

    u32x4 qf[NT][HD / 32];
    int limit[NT];  // slots that the lane's row sees
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = t * 8 + (col & 7);
        const bool there = r < rows;
        const int token = there ? r / G : 0, head = there ? r % G : 0;
        limit[t] = q.cached + token + 1;
        const uint16_t* p = a.q.p + (int64_t)(q.row0 + token) * a.q.row + (int64_t)(hk * G + head) * a.q.head;
#pragma unroll
        for (int f = 0; f < HD / 32; ++f) {
            const int d = HD == 32 ? grp * 8 : (f >> 1) * 64 + grp * 16 + (f & 1) * 8;
            qf[t][f] = there ? *(const u32x4*)(p + d) : u32x4{0u, 0u, 0u, 0u};
        }
    }
    f32x4 acc[NT][VT];
    float m[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t] = kEmpty;
        l[t] = 0.f;
#pragma unroll
        for (int v = 0; v < VT; ++v) acc[t][v] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    uint32_t kr[2][KW], vr[8][VW];
    float ksc[2], vsc[2];
    // slots past the end re-read the last one (in bounds and at hand)
    auto load_k = [&](int p0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t* p = K + (int64_t)min(p0 + t * 16 + col, end - 1) * HD;
            ksc[t] = ks[min(p0 + t * 16, end - 1) >> c.logb];
            if constexpr (HD == 32) {
                const u32x2 x = *(const u32x2*)(p + grp * 8);
                kr[t][0] = x.x;
                kr[t][1] = x.y;
            } else {
#pragma unroll
                for (int h = 0; h < HD / 64; ++h) {
                    const u32x4 x = *(const u32x4*)(p + h * 64 + grp * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) kr[t][h * 4 + i] = x[i];
                }
            }
        }
    };
    auto load_v = [&](int p0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint8_t* p = V + (int64_t)min(p0 + (j >> 2) * 16 + grp * 4 + (j & 3), end - 1) * HD + col * VT;
            if constexpr (HD == 128) {
                const u32x2 x = *(const u32x2*)p;
                vr[j][0] = x.x;
                vr[j][1] = x.y;
            } else if constexpr (HD == 64) {
                vr[j][0] = *(const uint32_t*)p;
            } else {
                vr[j][0] = *(const uint16_t*)p;
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) vsc[t] = vs[min(p0 + t * 16, end - 1) >> c.logb];
    };
    int p0 = first + wave * 32;
    if (p0 < end) {
        load_k(p0);
        load_v(p0);
    }
    for (; p0 < end; p0 += 128) {
        f32x4 z[NT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            u32x4 kf[HD / 32];
#pragma unroll
            for (int f = 0; f < HD / 32; ++f) kf[f] = widen8(kr[t][2 * f], kr[t][2 * f + 1], ksc[t]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                z[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int f = 0; f < HD / 32; ++f) z[n][t] = mfma16(kf[f], qf[n][f], z[n][t]);
            }
        }
        if (p0 + 128 < end) load_k(p0 + 128);
        const bool whole = p0 + 32 <= q.cached + 1 && p0 + 32 <= end;  // every row sees all 32 slots
        if (!whole) {
#pragma unroll
            for (int j = 0; j < 8; ++j)  // weight 0 alone would make NaN of a NaN code
                if (p0 + (j >> 2) * 16 + grp * 4 + (j & 3) >= end)
#pragma unroll
                    for (int w = 0; w < VW; ++w) vr[j][w] = 0u;
        }
        // A NaN code of V must not reach rows that do not see its slot: weight 0 times NaN is NaN.  Where a chunk that
        // some rows see in part holds one, the products are formed without it and put back for those who see it.
        bool odd = false;
        if (!whole) {
            uint32_t nan = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < VW; ++w) nan |= nan_bytes(vr[j][w]);
            odd = __any(nan != 0);
        }
        u32x4 pf[NT], seen[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (SCORES && col < 8 && n * 8 + col < rows) {
                float* to = sp.scores + ((int64_t)pair * sp.tile_rows + n * 8 + col) * sp.score_stride + p0 + grp * 4;
                *(f32x4*)to = z[n][0];
                *(f32x4*)(to + 16) = z[n][1];
            }
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = z[n][j >> 2][j & 3] * a.qscale;
            if (!whole) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int slot = p0 + (j >> 2) * 16 + grp * 4 + (j & 3);
                    if (slot >= limit[n] || slot >= end) x[j] = -__builtin_inff();
                }
                if (odd)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        seen[n][j] = (x[2 * j] == -__builtin_inff() ? 0u : 0x3f80u) | (x[2 * j + 1] == -__builtin_inff() ? 0u : 0x3f800000u);
            }
            float top = x[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
            if (__any(top > m[n] - kNear)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float mn = top > m[n] - kNear ? fmaxf(m[n], top + kAbove) : m[n];
                const float f = __builtin_amdgcn_exp2f(m[n] - mn);
                m[n] = mn;
                l[n] *= f;
#pragma unroll
                for (int r = 0; r < 4; ++r) {  // sums of row 4*grp + r; its factor is in the lanes of that column
                    const float g = __shfl(f, grp * 4 + r, 64);
#pragma unroll
                    for (int v = 0; v < VT; ++v) acc[n][v][r] *= g;
                }
            }
            float pr[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                pr[j] = __builtin_amdgcn_exp2f(x[j] - m[n]);
                l[n] += pr[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t hi = pack_bf16(pr[2 * j], pr[2 * j + 1]);
                const uint32_t lo = pack_bf16(pr[2 * j] - bf_lo(hi), pr[2 * j + 1] - bf_hi(hi));
                pf[n][j] = col < 8 ? hi : lo;
            }
        }
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            uint32_t in[2][4], tr[2][4];
#pragma unroll
            for (int j = 0; j < 8; ++j) in[j >> 2][j & 3] = vr[j][w];
            transpose4(in[0], tr[0]);
            transpose4(in[1], tr[1]);
            if (odd) {
#pragma unroll
                for (int b = 0; b < (VT < 4 ? VT : 4); ++b) {
                    const uint32_t na = nan_bytes(tr[0][b]), nb = nan_bytes(tr[1][b]);
                    // 0x38 is 1.0: bytes of ones where the code is NaN
                    const u32x4 where = widen8((na >> 7) * 0x38u, (nb >> 7) * 0x38u, 1.f);
                    tr[0][b] &= ~((na >> 7) * 0xffu);
                    tr[1][b] &= ~((nb >> 7) * 0xffu);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const f32x4 hit = mfma16(seen[n], where, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (hit[r] > 0.f) acc[n][w * 4 + b][r] = __builtin_nanf("");
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < (VT < 4 ? VT : 4); ++b) {
                const u32x4 vf = {widen2<false>(tr[0][b], vsc[0]), widen2<true>(tr[0][b], vsc[0]),
                                  widen2<false>(tr[1][b], vsc[1]), widen2<true>(tr[1][b], vsc[1])};
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[n][w * 4 + b] = mfma16(pf[n], vf, acc[n][w * 4 + b]);
            }
        }
        if (p0 + 128 < end) load_v(p0 + 128);
    }
    // the lane groups of a column, the two halves of the weights, then the wavefronts
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16, 64);
        l[n] += __shfl_xor(l[n], 32, 64);
        if (lane < 8) sm_ml[wave][n * 8 + lane] = make_float2(m[n], l[n]);
#pragma unroll
        for (int v = 0; v < VT; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float o = acc[n][v][r] + __shfl_xor(acc[n][v][r], 32, 64);
                if (grp < 2) sm_o[wave][n * 8 + grp * 4 + r][col * VT + v] = o;
            }
    }
    __syncthreads();
    const int many = (len + sp.per - 1) / sp.per;  // ranges of this sequence
    const int total = min(rows, NT * 8) * HD;
    for (int i = threadIdx.x * 4; i < total; i += 1024) {
        const int r = i / HD, d = i % HD;
        float mm = kEmpty;
#pragma unroll
        for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sm_ml[w][r].x);
        float ll = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(sm_ml[w][r].x - mm);
            ll += sm_ml[w][r].y * f;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += sm_o[w][r][d + j] * f;
        }
        if (many > 1) {
            const int64_t at = ((int64_t)pair * sp.ranges + range) * sp.tile_rows + r;
            *(f32x4*)(sp.acc + at * HD + d) = o;
            if (d == 0) sp.ml[at] = make_float2(mm, ll);
        } else {
            const float inv = 1.f / ll;
            u32x2 w;
            w.x = pack_bf16(o[0] * inv, o[1] * inv);
            w.y = pack_bf16(o[2] * inv, o[3] * inv);
            *(u32x2*)(a.out.p + (int64_t)(q.row0 + r / G) * a.out.row + (int64_t)(hk * G + r % G) * a.out.head + d) = w;
            if (SCORES && d == 0) sp.final_ml[(int64_t)pair * sp.tile_rows + r] = make_float2(mm, inv);
        }
    }
}

// Adds up the ranges of one (pair, row): one wavefront, HD/4 lanes per range.
template <int HD>
__global__ __launch_bounds__(256) void merge_kernel(Cache c, Step s, Attend a, Split sp) {
    constexpr int LPR = HD / 4, SIDE = 64 / LPR;
    const int lane = threadIdx.x & 63, sub = lane % LPR;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int pair = (int)(item / sp.tile_rows), r = (int)(item % sp.tile_rows);
    if (pair >= c.n_seq * c.Hkv) return;
    const int seq = pair / c.Hkv, hk = pair % c.Hkv, G = a.Hq / c.Hkv;
    const Seq q = sequence(c, s, seq);
    const int many = (q.cached + q.n_new + sp.per - 1) / sp.per;
    if (r >= q.n_new * G || many <= 1) return;
    const int64_t at = (int64_t)pair * sp.ranges * sp.tile_rows + r;
    float m = kEmpty, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m2, float l2, const f32x4& o2) {
        const float mn = fmaxf(m, m2), fa = __builtin_amdgcn_exp2f(m - mn), fb = __builtin_amdgcn_exp2f(m2 - mn);
        l = l * fa + l2 * fb;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = o[j] * fa + o2[j] * fb;
        m = mn;
    };
    for (int i = lane / LPR; i < many; i += SIDE) {
        const float2 e = sp.ml[at + (int64_t)i * sp.tile_rows];
        add(e.x, e.y, *(const f32x4*)(sp.acc + (at + (int64_t)i * sp.tile_rows) * HD + sub * 4));
    }
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) {
        const float m2 = __shfl_xor(m, off, 64), l2 = __shfl_xor(l, off, 64);
        f32x4 o2;
#pragma unroll
        for (int j = 0; j < 4; ++j) o2[j] = __shfl_xor(o[j], off, 64);
        add(m2, l2, o2);
    }
    if (lane < LPR) {
        const float inv = 1.f / l;
        u32x2 w;
        w.x = pack_bf16(o[0] * inv, o[1] * inv);
        w.y = pack_bf16(o[2] * inv, o[3] * inv);
        *(u32x2*)(a.out.p + (int64_t)(q.row0 + r / G) * a.out.row + (int64_t)(hk * G + r % G) * a.out.head + sub * 4) = w;
        if (sp.final_ml != nullptr && sub == 0) sp.final_ml[(int64_t)pair * sp.tile_rows + r] = make_float2(m, inv);
    }
}

// One thread per slot: what the rows of its pair gave it, from the products kept by decode_kernel.
__global__ __launch_bounds__(256) void weights_kernel(Cache c, Step s, Attend a, Split sp, int chunks) {
    const int64_t pair = blockIdx.x / chunks;
    const int j = blockIdx.x % chunks * 256 + threadIdx.x, seq = (int)(pair / c.Hkv), G = a.Hq / c.Hkv;
    const Seq q = sequence(c, s, seq);
    if (j >= q.cached + q.n_new) return;
    float w = a.weight_in != nullptr && j < q.cached ? a.weight_in[pair * c.max_len + j] : 0.f;
    for (int r = max(0, j - q.cached) * G; r < q.n_new * G; ++r) {
        const float2 ml = sp.final_ml[pair * sp.tile_rows + r];
        const float z = sp.scores[(pair * sp.tile_rows + r) * sp.score_stride + j];
        w += __builtin_amdgcn_exp2f(z * a.qscale - ml.x) * ml.y;
    }
    a.weight_out[pair * c.max_len + j] = w;
}

// ---- many new tokens (first form: one score per thread) -----------------------------------------------------

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

int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

// How a step is run, from its sizes and bounds.
struct Plan {
    int tiles;  // row tiles of decode_kernel, 0: many new tokens
    Split sp;
    int64_t o_ml, o_scores, o_final, bytes;
};

Plan plan(const Cache& c, const Step& s, int Hq, bool weights) {
    Plan p{};
    const int64_t pairs = (int64_t)c.n_seq * c.Hkv, rows = (int64_t)s.max_new * (Hq / c.Hkv);
    const int most = (int)min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len);
    p.tiles = rows <= 8 ? 1 : rows <= 16 ? 2 : 0;
    if (p.tiles == 0) {
        p.bytes = weights ? up256((int64_t)s.n_rows * Hq * 4) : 0;
        return p;
    }
    const int64_t want = 1024 * 2;  // workgroups
    int64_t per = ((int64_t)most * pairs / want + 127) / 128 * 128;
    per = per < 256 ? 256 : per;
    int64_t ranges = (most + per - 1) / per;
    if (ranges < 1) ranges = 1;
    p.sp.per = (int)per;
    p.sp.ranges = (int)ranges;
    p.sp.tile_rows = p.tiles * 8;
    p.sp.score_stride = (most + 31) / 32 * 32;
    int64_t o = 0;
    const int64_t items = ranges > 1 ? pairs * ranges * p.sp.tile_rows : 0;
    o += up256(items * c.hd * 4);
    p.o_ml = o;
    o += up256(items * 8);
    p.o_scores = o;
    if (weights) o += up256(pairs * p.sp.tile_rows * p.sp.score_stride * 4);
    p.o_final = o;
    if (weights) o += up256(pairs * p.sp.tile_rows * 8);
    p.bytes = o;
    return p;
}

template <int HD, int NT>
void launch_decode(hipStream_t st, const Cache& c, const Step& s, const Attend& a, const Split& sp) {
    const dim3 grid((unsigned)((int64_t)c.n_seq * c.Hkv * sp.ranges)), block(256);
    if (a.weight_out != nullptr)
        hipLaunchKernelGGL((decode_kernel<HD, NT, true>), grid, block, 0, st, c, s, a, sp);
    else
        hipLaunchKernelGGL((decode_kernel<HD, NT, false>), grid, block, 0, st, c, s, a, sp);
    if (sp.ranges > 1)
        hipLaunchKernelGGL(merge_kernel<HD>, dim3((unsigned)(((int64_t)c.n_seq * c.Hkv * sp.tile_rows + 3) / 4)), block, 0, st, c, s, a, sp);
}

template <int HD>
void launch_hd(hipStream_t st, const Cache& c, const Step& s, const Attend& a, const Plan& p) {
    if (p.tiles == 1) launch_decode<HD, 1>(st, c, s, a, p.sp);
    if (p.tiles == 2) launch_decode<HD, 2>(st, c, s, a, p.sp);
}

}  // namespace

int64_t attend_workspace(const Cache& c, const Step& s, int Hq, bool weights) { return plan(c, s, Hq, weights).bytes; }

void launch_attend(hipStream_t st, const Cache& c, const Step& s, const Attend& a) {
    Plan p = plan(c, s, a.Hq, a.weight_out != nullptr);
    if (p.tiles > 0) {
        p.sp.acc = (float*)a.ws;
        p.sp.ml = (float2*)(a.ws + p.o_ml);
        p.sp.scores = (float*)(a.ws + p.o_scores);
        p.sp.final_ml = a.weight_out != nullptr ? (float2*)(a.ws + p.o_final) : nullptr;
        if (s.n_rows > 0) {
            if (c.hd == 32) launch_hd<32>(st, c, s, a, p);
            if (c.hd == 64) launch_hd<64>(st, c, s, a, p);
            if (c.hd == 128) launch_hd<128>(st, c, s, a, p);
        }
        if (a.weight_out != nullptr) {
            const int chunks = (p.sp.score_stride + 255) / 256;
            if (chunks > 0)
                hipLaunchKernelGGL(weights_kernel, dim3((unsigned)((int64_t)c.n_seq * c.Hkv * chunks)), dim3(256), 0, st, c, s, a, p.sp, chunks);
        }
        return;
    }
    float* lse = a.weight_out != nullptr ? (float*)a.ws : nullptr;
    if (s.n_rows > 0)
        hipLaunchKernelGGL(attend_plain_kernel, dim3((unsigned)((int64_t)s.n_rows * a.Hq)), dim3(256), 0, st, c, s, a, lse);
    if (a.weight_out != nullptr)
        hipLaunchKernelGGL(weights_plain_kernel, dim3((unsigned)((int64_t)c.n_seq * c.Hkv * ((c.max_len + 255) / 256))),
                           dim3(256), 0, st, c, s, a, (const float*)lse);
}

}  // namespace kkv8
