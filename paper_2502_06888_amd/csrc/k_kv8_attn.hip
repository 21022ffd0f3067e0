// Attention over the 8-bit key-value cache.
//
// o = softmax(q K^T) V with K and V dequantised on the way into the matrix instructions: a scale is a power of two, so
// code * scale is exact in bf16 and the conversion instruction applies it for nothing.  Products are bf16, sums and
// softmax statistics fp32, base-2 exponentials with log2(e) folded into the factor of the scores.
#include <type_traits>

#include "attn_device.h"
#include "kv8_kernels.h"

namespace kkv8 {
namespace {

using namespace kattn;

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
// One workgroup of W wavefronts, four or eight, per (sequence, key-value head, range of slots); all rows (token, query head of the
// group) of the pair share what is read, in tiles of 8.  A wavefront takes 32 slots at a time, in two tiles of 16:
//   scores    S^T[slot][row] = K Q^T, 16x16x32: lane l holds row l%16 and slots 4*(l/16)..+3 of each tile;
//   sums      O[row][element] = P V with the eight weights a lane holds as its eight steps of the reduction, so that the
//             weights never leave their lane: V is read by slots in that order, byte-transposed in registers.
// A tile of 16 matrix rows serves 8 rows twice: the second half multiplies what rounding the weights to bf16 left over,
// so the weights count with 16 bits at no matrix cost.
// Bound by the bytes where there are enough of them: 512 sequences of 513 slots, 8 heads of 128 (538 MB of codes) take 90 us,
// 6.0 TB/s; with the weights summed 114.  4 sequences of 7500 slots and 6 query heads per group (61 MB) take 15 us and 5 for
// merge and weights, 1 of 701 slots 10: latency.
constexpr int kRows = 128, kSlots = 64;  // rows and slots of a tile where there are many new tokens

struct Split {
    int per, ranges;    // slots of a range (a multiple of 128, with many new tokens of 64), ranges of a sequence at most
    int tile_rows;      // rows the buffers below hold per pair
    int score_stride;   // slots a row of `scores` holds, a multiple of 16
    float* acc;         // [pair, range, row, hd] unnormalised sums; with float2 `ml` (reference, sum of weights)
    float2* ml;
    float* scores;      // [pair, row, slot] products q . K
    int waves;          // of a workgroup of decode_kernel
    int lds_scores;     // bytes of LDS that hold those of a pair instead, 0: they are in `scores`
    float2* final_ml;   // [pair, row] with many new tokens: reference of all ranges, 2^-kAbove / sum of weights
    u32x4* packed;      // [pair, tile of kSlots] dequantised (see Tile), or null
    int32_t* odd;       // [pair, tile]
    int packed_tiles;   // tiles per pair
    float* part;        // [split of the rows, pair, slot] weights of prompt_weights_kernel where it splits the rows
    int splits;
};

template <bool STREAM, class T>
__device__ __forceinline__ T fetch(const T* p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(p);
    else return *p;
}

// Where the products q . K go: nowhere, to the workspace, or into LDS (where they fit and a sequence is one range).
enum { kNoScores, kScores, kScoresLds };

template <int HD, int NT, int SCORES, bool STREAM, int W>
__global__ __launch_bounds__(W * 64, NT * HD <= 64 ? 4 : NT * HD <= 128 ? 3 : 2) void decode_kernel(Cache c, Step s, Attend a, Split sp) {
    constexpr int KW = HD / 16;             // words of a K row that a lane holds: HD/4 bytes
    constexpr int VT = HD / 16;             // tiles of 16 elements of the sums
    constexpr int VW = VT >= 4 ? VT / 4 : 1;  // words of a V row that a lane holds: VT bytes
    __shared__ float sm_o[W][NT * 8][HD];
    __shared__ float2 sm_ml[W][NT * 8], done[NT * 8];
    extern __shared__ __attribute__((aligned(16))) float lds_scores[];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 15, grp = lane >> 4;
    const int range = blockIdx.x % sp.ranges, pair = blockIdx.x / sp.ranges;
    const int seq = pair / c.Hkv, hk = pair % c.Hkv, G = a.Hq / c.Hkv;
    const Seq q = sequence(c, s, seq);
    const int len = q.cached + q.n_new, rows = q.n_new * G;
    const int first = range * sp.per, end = min(first + sp.per, len);
    const int64_t base = (int64_t)seq * c.Hkv + hk;
    const int many = (len + sp.per - 1) / sp.per;  // ranges of this sequence
    float* scores = SCORES == kScoresLds ? lds_scores : sp.scores + (int64_t)pair * sp.tile_rows * sp.score_stride;
    if (SCORES && rows == 0 && many <= 1 && range == 0)  // no new tokens: the weights stay
        for (int j = threadIdx.x; j < len; j += W * 64) a.weight_out[base * c.max_len + j] = a.weight_in != nullptr ? a.weight_in[base * c.max_len + j] : 0.f;
    if (rows == 0 || first >= end) return;
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
                const u32x2 x = fetch<STREAM>((const u32x2*)(p + grp * 8));
                kr[t][0] = x.x;
                kr[t][1] = x.y;
            } else {
#pragma unroll
                for (int h = 0; h < HD / 64; ++h) {
                    const u32x4 x = fetch<STREAM>((const u32x4*)(p + h * 64 + grp * 16));
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
                const u32x2 x = fetch<STREAM>((const u32x2*)p);
                vr[j][0] = x.x;
                vr[j][1] = x.y;
            } else if constexpr (HD == 64) {
                vr[j][0] = fetch<STREAM>((const uint32_t*)p);
            } else {
                vr[j][0] = fetch<STREAM>((const uint16_t*)p);
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
    auto chunk = [&](auto whole_) {
        constexpr bool whole = decltype(whole_)::value;  // every row sees all 32 slots
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
        if (p0 + 32 * W < end) load_k(p0 + 32 * W);
        bool odd = false;
        if (!whole) {  // weight 0 times a NaN code would be NaN: such codes are taken out, and put back where they are seen
            uint32_t nan = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    if (p0 + (j >> 2) * 16 + grp * 4 + (j & 3) >= end) vr[j][w] = 0u;
                    const uint32_t n = nan_bytes(vr[j][w]);
                    vr[j][w] &= ~((n >> 7) * 0xffu);
                    nan |= n;
                }
            odd = __any(nan != 0);
        }
        u32x4 pf[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (SCORES != kNoScores && col < 8 && n * 8 + col < rows) {
                float* to = scores + (int64_t)(n * 8 + col) * sp.score_stride + p0 + grp * 4;
                *(f32x4*)to = z[n][0];
                *(f32x4*)(to + 16) = z[n][1];
            }
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = z[n][j >> 2][j & 3];
            if (!whole) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int slot = p0 + (j >> 2) * 16 + grp * 4 + (j & 3);
                    if (slot >= limit[n] || slot >= end) x[j] = -__builtin_inff();
                }
            }
            float top = x[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
            top *= a.qscale;
            if (__any(top > m[n] + kRise)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float mn = top > m[n] + kRise ? reference_of(top) : m[n];
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
            exponents(m[n], kAbove, a.qscale, [&](auto&& of) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = of(x[j]);
            });
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                pr[j] = __builtin_amdgcn_exp2f(x[j]);
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
#pragma unroll
            for (int b = 0; b < (VT < 4 ? VT : 4); ++b) {
                const u32x4 vf = {widen2<false>(tr[0][b], vsc[0]), widen2<true>(tr[0][b], vsc[0]),
                                  widen2<false>(tr[1][b], vsc[1]), widen2<true>(tr[1][b], vsc[1])};
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[n][w * 4 + b] = mfma16(pf[n], vf, acc[n][w * 4 + b]);
            }
        }
        if (p0 + 32 * W < end) load_v(p0 + 32 * W);
        if (odd) {
            for (int j = p0; j < min(p0 + 32, end); ++j)
#pragma unroll
                for (int v = 0; v < VT; ++v) {
                    if ((V[(int64_t)j * HD + col * VT + v] & 0x7f) != 0x7f) continue;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (j <= q.cached + (n * 8 + ((grp * 4 + r) & 7)) / G) acc[n][v][r] = __builtin_nanf("");
                }
        }
    };
    const int sure = min(end, q.cached + 1);
    for (; p0 + 32 <= sure; p0 += 32 * W) chunk(std::true_type{});
    for (; p0 < end; p0 += 32 * W) chunk(std::false_type{});
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
    const int total = min(rows, NT * 8) * HD;
    for (int i = threadIdx.x * 4; i < total; i += W * 256) {
        const int r = i / HD, d = i % HD;
        float mm = kEmpty;
#pragma unroll
        for (int w = 0; w < W; ++w) mm = fmaxf(mm, sm_ml[w][r].x);
        float ll = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
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
            if (SCORES && d == 0) done[r] = make_float2(mm, inv * kBelow);
        }
    }
    if (!SCORES || many > 1) return;
    __syncthreads();  // statistics and scores are there, those of this workgroup
    bool far = false;
    for (int r = 0; r < rows; ++r) far |= fabsf(done[r].x) > kFar;
    for (int j = threadIdx.x; j < len; j += W * 64) {
        float w = a.weight_in != nullptr && j < q.cached ? a.weight_in[base * c.max_len + j] : 0.f;
        for (int r = max(0, j - q.cached) * G; r < rows; ++r) {
            const float z = scores[(int64_t)r * sp.score_stride + j];
            w += __builtin_amdgcn_exp2f(far ? apart(z, a.qscale, done[r].x) : __builtin_fmaf(z, a.qscale, -done[r].x)) * done[r].y;
        }
        a.weight_out[base * c.max_len + j] = w;
    }
}

struct Partial {  // running softmax over ranges: reference, sum of weights, four elements of the sums
    float m = kEmpty, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float m2, float l2, const f32x4& o2) {
        const float mn = fmaxf(m, m2), fa = __builtin_amdgcn_exp2f(m - mn), fb = __builtin_amdgcn_exp2f(m2 - mn);
        l = l * fa + l2 * fb;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = o[j] * fa + o2[j] * fb;
        m = mn;
    }
    // ranges i, i + by, .. of the row whose first partial sums are at `at`, four requested before the first is used
    template <int HD>
    __device__ __forceinline__ void add_ranges(const Split& sp, int64_t at, int i, int by, int many, int element) {
        constexpr int AHEAD = 4;
        for (; i < many; i += AHEAD * by) {
            float2 e[AHEAD];
            f32x4 x[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {  // past the end: the last one again, unused
                const int64_t from = at + (int64_t)min(i + u * by, many - 1) * sp.tile_rows;
                e[u] = sp.ml[from];
                x[u] = *(const f32x4*)(sp.acc + from * HD + element);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (i + u * by < many) add(e[u].x, e[u].y, x[u]);
        }
    }
    __device__ __forceinline__ void add_lanes(int from) {  // lanes `from`, 2 * from, .. apart
        for (int off = from; off < 64; off <<= 1) {
            const float m2 = __shfl_xor(m, off, 64), l2 = __shfl_xor(l, off, 64);
            f32x4 o2;
#pragma unroll
            for (int j = 0; j < 4; ++j) o2[j] = __shfl_xor(o[j], off, 64);
            add(m2, l2, o2);
        }
    }
    __device__ __forceinline__ void write(uint16_t* to) const {
        const float inv = 1.f / l;
        u32x2 w;
        w.x = pack_bf16(o[0] * inv, o[1] * inv);
        w.y = pack_bf16(o[2] * inv, o[3] * inv);
        *(u32x2*)to = w;
    }
};

// Few new tokens, sequences of several ranges.  The first workgroups add up the ranges of a (pair, row): WIDE one each, four
// wavefronts of 64 / (HD/4) ranges side by side, else one in each wavefront; the others take 256 slots of a pair each:
// what its rows gave them, from the products kept by decode_kernel and the statistics of all ranges.
template <int HD, bool WIDE>
__global__ __launch_bounds__(256) void finish_kernel(Cache c, Step s, Attend a, Split sp, int merges, int chunks) {
    constexpr int LPR = HD / 4, SIDE = 64 / LPR;
    __shared__ float4 sums[4][LPR];
    __shared__ float2 stat[16];
    const int lane = threadIdx.x & 63, wave = wave_number(), G = a.Hq / c.Hkv;
    const bool merging = (int)blockIdx.x < merges;
    const int item = !merging ? blockIdx.x - merges : WIDE ? blockIdx.x : blockIdx.x * 4 + wave;
    const int pair = item / (merging ? sp.tile_rows : chunks), seq = pair / c.Hkv;
    if (pair >= c.n_seq * c.Hkv) return;
    const Seq q = sequence(c, s, seq);
    const int len = q.cached + q.n_new, rows = q.n_new * G, many = (len + sp.per - 1) / sp.per;
    if (merging) {
        const int r = item % sp.tile_rows;
        if (r >= rows || many <= 1) return;
        const int64_t at = (int64_t)pair * sp.ranges * sp.tile_rows + r;
        Partial t;
        t.add_ranges<HD>(sp, at, (WIDE ? wave * SIDE : 0) + lane / LPR, (WIDE ? 4 : 1) * SIDE, many, lane % LPR * 4);
        t.add_lanes(LPR);
        if (!WIDE) {
            if (lane < LPR) t.write(a.out.p + (int64_t)(q.row0 + r / G) * a.out.row + (int64_t)(pair % c.Hkv * G + r % G) * a.out.head + lane * 4);
            return;
        }
        if (lane < LPR) sums[wave][lane] = make_float4(t.o[0], t.o[1], t.o[2], t.o[3]);
        if (lane == 0) stat[wave] = make_float2(t.m, t.l);
        __syncthreads();
        if (wave != 0 || lane >= LPR) return;
        for (int w = 1; w < 4; ++w) t.add(stat[w].x, stat[w].y, f32x4{sums[w][lane].x, sums[w][lane].y, sums[w][lane].z, sums[w][lane].w});
        t.write(a.out.p + (int64_t)(q.row0 + r / G) * a.out.row + (int64_t)(pair % c.Hkv * G + r % G) * a.out.head + lane * 4);
        return;
    }
    if (many <= 1) return;  // done by decode_kernel
    const int j0 = item % chunks * 256, j = j0 + threadIdx.x;
    if (j0 >= len) return;
    for (int r = wave * 4; r < rows; r += 16)  // 16 lanes per row
        if (const int row = r + lane / 16; true) {
            float m = kEmpty, l = 0.f;
            for (int i = lane % 16; i < many && row < rows; i += 16) {
                const float2 e = sp.ml[((int64_t)pair * sp.ranges + i) * sp.tile_rows + row];
                const float mn = fmaxf(m, e.x);
                l = l * __builtin_amdgcn_exp2f(m - mn) + e.y * __builtin_amdgcn_exp2f(e.x - mn);
                m = mn;
            }
            for (int off = 1; off < 16; off <<= 1) {
                const float m2 = __shfl_xor(m, off, 64), l2 = __shfl_xor(l, off, 64), mn = fmaxf(m, m2);
                l = l * __builtin_amdgcn_exp2f(m - mn) + l2 * __builtin_amdgcn_exp2f(m2 - mn);
                m = mn;
            }
            if (lane % 16 == 0 && row < rows) stat[row] = make_float2(m, 1.f / l * kBelow);
        }
    __syncthreads();
    if (j >= len) return;
    bool far = false;
    for (int r = 0; r < rows; ++r) far |= fabsf(stat[r].x) > kFar;
    const int64_t at = (int64_t)pair * c.max_len + j;
    float w = a.weight_in != nullptr && j < q.cached ? a.weight_in[at] : 0.f;
    for (int r = max(0, j - q.cached) * G; r < rows; ++r) {
        const float z = sp.scores[((int64_t)pair * sp.tile_rows + r) * sp.score_stride + j];
        w += __builtin_amdgcn_exp2f(far ? apart(z, a.qscale, stat[r].x) : __builtin_fmaf(z, a.qscale, -stat[r].x)) * stat[r].y;
    }
    a.weight_out[at] = w;
}

// Many new tokens: adds up the ranges of R rows of a pair, one wavefront, whose reads are on their way together.  Bound by
// latency: a wavefront reads lengths, statistics and sums one after the other.  So one row where the chip takes all wavefronts
// at once, four where it does not: 40000 rows of which 31000 exist, in 2 ranges, 10 us instead of 16; 1024 in 59 ranges 5 us more.
template <int HD, int R>
__global__ __launch_bounds__(256) void merge_kernel(Cache c, Step s, Attend a, Split sp) {
    constexpr int LPR = HD / 4, SIDE = 64 / LPR, AHEAD = R > 1 ? 2 : 4;
    const int lane = threadIdx.x & 63, G = a.Hq / c.Hkv;
    const int64_t item = (int64_t)blockIdx.x * 4 + wave_number();
    const int groups = sp.tile_rows / R, pair = (int)(item / groups), r0 = (int)(item % groups) * R;
    if (pair >= c.n_seq * c.Hkv) return;
    const Seq q = sequence(c, s, pair / c.Hkv);
    const int rows = q.n_new * G;
    if (r0 >= rows) return;
    const int many = (q.cached + min(r0 / kRows * kRows + kRows - 1, rows - 1) / G + sp.per) / sp.per;  // of what the rows' tile sees
    if (many <= 1) return;
    const int64_t at = (int64_t)pair * sp.ranges * sp.tile_rows + r0;
    Partial t[R];
    for (int i = lane / LPR; i < many; i += AHEAD * SIDE) {
        float2 e[AHEAD][R];
        f32x4 x[AHEAD][R];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int k = 0; k < R; ++k) {  // past the end: the last ones again, unused
                const int64_t from = at + (int64_t)min(i + u * SIDE, many - 1) * sp.tile_rows + min(k, rows - 1 - r0);
                e[u][k] = sp.ml[from];
                x[u][k] = *(const f32x4*)(sp.acc + from * HD + lane % LPR * 4);
            }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (i + u * SIDE < many) t[k].add(e[u][k].x, e[u][k].y, x[u][k]);
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        t[k].add_lanes(LPR);
        const int r = r0 + k;
        if (lane >= LPR || r >= rows) continue;
        t[k].write(a.out.p + (int64_t)(q.row0 + r / G) * a.out.row + (int64_t)(pair % c.Hkv * G + r % G) * a.out.head + lane * 4);
        if (sp.final_ml != nullptr && lane == 0) sp.final_ml[(int64_t)pair * sp.tile_rows + r] = make_float2(t[k].m, 1.f / t[k].l * kBelow);
    }
}

// ---- many new tokens: bound by the matrix cores ---------------------------------------------------------------
//
// One workgroup of four wavefronts per (sequence, key-value head, 128 rows, range of slots); a row is a (token, query
// head of the group), so the heads that share K and V share a tile of them: 64 slots as bf16 in LDS, the next 64 on
// their way.  A wavefront has 32 rows: S^T[slot][row] = K Q^T and O^T[element][row] = V^T P^T, 32x32x16.  Lane l
// holds row l%32 throughout, so softmax statistics and rescaling stay in the lane, and the weights of a lane are its
// operand of the second product as they are: slots 4*(l/32)..+3 and 8 + 4*(l/32)..+3 of each 16.
//
// A tile lies in LDS in the order in which the matrix instructions take it: units of 64 lanes x 16 bytes, read
// and written without bank conflicts; unit (t, f) of K: lane l holds slot 32t + l%32, elements 16f + 8*(l/32)..+7; unit
// (u, m) of V: element 32m + l%32, the eight slots of 16u.. in the order above, at place v_place.
//
// Where a tile serves many row tiles it is dequantised once, by pack_kernel, into the workspace in this order, and
// comes from there into LDS without passing through registers; else the workgroup dequantises it on the way.
// The weights are rounded once, to bf16 (by up to 2^-8), as the operand of the second product; their sum takes the unrounded
// ones.  The 16 bits that decode_kernel gives them for nothing would be a second product here, of the two that bound the kernel.
//
// Two prompts of 3907 and 4096 tokens, 32 / 8 heads of 128: 265 to 271 us, 9 of them for dequantising ahead, 1.0 PFLOP/s (a large
// library product of bf16 reaches 1.30 on this card): the matrix cores are busy 50 % of the time at the 1.9 GHz that the power
// limit leaves, vector instructions (half of them exponentials) 44 %, two wavefronts per SIMD.  32 prompts of 512 tokens:
// 129 us, 0.53 PFLOP/s and 2.3 TB/s: the start and end of a tile of rows weigh as much as its 4.5 steps.
template <int HD>
struct Tile {
    static constexpr int kUnits = HD / 8;            // of K, and of V
    static constexpr int kBytes = 2 * kUnits * 1024;  // K, then V
    static constexpr int kPieces = kBytes / 4096;     // of 16 bytes per thread
    __device__ __forceinline__ static int v_slot(int group, int j) { return (group >> 1) * 16 + (group & 1) * 4 + (j & 3) + (j >> 2) * 8; }

    // Place of (element % 32, half of the slots) in a unit of V with elements 32m..: spread so that both the threads that
    // write four neighbouring elements and the lanes that read 32 touch every bank once.
    __device__ __forceinline__ static int v_place(int e, int half, int m) {
        return ((e >> 2) ^ ((e >> 1) & 1)) | ((e & 1) << 3 ^ (m >> 1) << 3) | ((e >> 1) & 1) << 4 | half << 5;
    }

    // Codes on their way.  Items of 32 bytes: HD*2 of K (a slot's 32 elements), HD*2 of V (four elements of eight slots).
    static constexpr int kItems = HD * 2;
    static constexpr bool kBoth = kItems == 256;
    uint32_t kr[8], vr[8];
    float ksc, vsc;
    __device__ __forceinline__ static int v_item() { return kBoth ? (int)threadIdx.x : (int)threadIdx.x - kItems; }
    __device__ __forceinline__ static bool has_k() { return kBoth || (int)threadIdx.x < kItems; }
    __device__ __forceinline__ static bool has_v() { return kBoth || ((int)threadIdx.x >= kItems && (int)threadIdx.x < 2 * kItems); }

    // slots past `total` re-read the last one
    __device__ __forceinline__ void load(const Cache& c, const uint8_t* K, const uint8_t* V, const float* ks, const float* vs, int j0, int total) {
        // 32-bit offsets from the uniform pointers: a cache row has at most 2^27 bytes
        if (has_k()) {
            const int slot = min(j0 + ((int)threadIdx.x & 63), total - 1);
            const u32x4* p = (const u32x4*)(K + (uint32_t)(slot * HD + ((int)threadIdx.x >> 6) * 32));
            const u32x4 a = p[0], b = p[1];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                kr[w] = a[w];
                kr[4 + w] = b[w];
            }
            ksc = ks[(uint32_t)(slot >> c.logb)];
        }
        if (has_v()) {
            const int quad = v_item() % (HD / 4), group = v_item() / (HD / 4);
            if (j0 + kSlots <= total) {  // one address for the eight slots
                const uint8_t* p = V + (uint32_t)((j0 + v_slot(group, 0)) * HD + quad * 4);
#pragma unroll
                for (int j = 0; j < 8; ++j) vr[j] = *(const uint32_t*)(p + (j & 3) * HD + (j >> 2) * 8 * HD);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    vr[j] = *(const uint32_t*)(V + (uint32_t)(min(j0 + v_slot(group, j), total - 1) * HD + quad * 4));
            }
            vsc = vs[(uint32_t)(min(j0 + (group >> 1) * 16, total - 1) >> c.logb)];
        }
    }
    // Into a tile at `to`.  Codes of V past `total` count as 0, and so do NaN ones where `part` is set (weight 0 times NaN
    // would reach rows that do not see the slot); returns whether there were such.
    template <class P>
    __device__ __forceinline__ bool store(P to, int j0, int total, bool part) {
        uint32_t nan = 0;
        if (has_k()) {
            const int slot = threadIdx.x & 63, p = threadIdx.x >> 6;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                to[((slot >> 5) * (HD / 16) + 2 * p + (w >> 1)) * 64 + (slot & 31) + 32 * (w & 1)] = widen8(kr[2 * w], kr[2 * w + 1], ksc);
        }
        if (has_v()) {
            const int quad = v_item() % (HD / 4), group = v_item() / (HD / 4);
            if (part) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j0 + v_slot(group, j) >= total) vr[j] = 0u;
                    const uint32_t n = nan_bytes(vr[j]);
                    vr[j] &= ~((n >> 7) * 0xffu);
                    nan |= n;
                }
            }
            uint32_t in[2][4], tr[2][4];
#pragma unroll
            for (int j = 0; j < 8; ++j) in[j >> 2][j & 3] = vr[j];
            transpose4(in[0], tr[0]);
            transpose4(in[1], tr[1]);
#pragma unroll
            for (int b = 0; b < 4; ++b)
                to[(kUnits + (group >> 1) * (HD / 32) + (quad >> 3)) * 64 + v_place((quad & 7) * 4 + b, group & 1, quad >> 3)] = widen8(tr[0][b], tr[1][b], vsc);
        }
        return nan != 0;
    }
};

// The slots that a step's tokens see, dequantised tile by tile; `odd` notes the tiles of V with NaN codes, which are left out.
template <int HD>
__global__ __launch_bounds__(256) void pack_kernel(Cache c, Step s, u32x4* packed, int32_t* odd, int tiles) {
    __shared__ int any;
    const int pairs = c.n_seq * c.Hkv, pair = blockIdx.x % pairs, tile = blockIdx.x / pairs, j0 = tile * kSlots;
    const Seq q = sequence(c, s, pair / c.Hkv);
    const int total = q.cached + q.n_new;
    if (j0 >= total || q.n_new == 0) return;
    const int64_t base = (int64_t)pair * c.max_len, sb = (int64_t)pair * (c.max_len >> c.logb);
    Tile<HD> t;
    t.load(c, c.codes[0] + base * HD, c.codes[1] + base * HD, c.scale[0] + sb, c.scale[1] + sb, j0, total);
    if (threadIdx.x == 0) any = 0;
    __syncthreads();
    if (t.store(packed + ((int64_t)pair * tiles + tile) * (Tile<HD>::kBytes / 16), j0, total, true)) any = 1;
    __syncthreads();
    if (threadIdx.x == 0) odd[(int64_t)pair * tiles + tile] = any;
}

// A workgroup takes `each` row tiles of its pair, one after the other (with one range): the first slots and the rows of q of
// the next one come while the last one ends.  Tiles see the more slots the later they are, so those of a workgroup are
// taken from both ends.
template <int HD, bool PACKED>
__global__ __launch_bounds__(256, 2) void prompt_kernel(Cache c, Step s, Attend a, Split sp, int groups, int each) {
    __shared__ u32x4 lds[2][Tile<HD>::kBytes / 16];
    __shared__ int nan[2];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5;
    // the pairs side by side, so that the tiles of one keep to an XCD
    const int pairs = c.n_seq * c.Hkv;
    const int pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
    const int range = rest % sp.ranges, group = rest / sp.ranges;
    const int seq = pair / c.Hkv, hk = pair % c.Hkv, G = a.Hq / c.Hkv;
    const Seq q = sequence(c, s, seq);
    const int rows = q.n_new * G, total = q.cached + q.n_new, first = range * sp.per;
    const int row_tiles = (rows + kRows - 1) / kRows;
    // k-th row tile of the workgroup, -1 where there is none (later ones then do not exist, either)
    auto tile_of = [&](int k) {
        const int i = k * groups + (k & 1 ? groups - 1 - group : group);
        return k < each && i < row_tiles ? row_tiles - 1 - i : -1;
    };
    auto sees_of = [&](int tile) { return q.cached + min(tile * kRows + kRows - 1, rows - 1) / G + 1; };  // slots its last row sees
    int tile = tile_of(0);
    if (tile < 0 || first >= sees_of(tile)) return;
    const int64_t base = (int64_t)seq * c.Hkv + hk;
    const uint8_t *K = c.codes[0] + base * c.max_len * HD, *V = c.codes[1] + base * c.max_len * HD;
    const float *ks = c.scale[0] + base * (c.max_len >> c.logb), *vs = c.scale[1] + base * (c.max_len >> c.logb);
    const uint8_t* packed = (const uint8_t*)sp.packed + (int64_t)pair * sp.packed_tiles * Tile<HD>::kBytes;
    const int32_t* odd = sp.odd + (int64_t)pair * sp.packed_tiles;

    u32x4 qf[HD / 16];
    auto load_q = [&](int tile) {
        const int r = min(tile * kRows + wave * 32 + col, rows - 1);
        const uint16_t* p = a.q.p + (int64_t)(q.row0 + r / G) * a.q.row + (int64_t)(hk * G + r % G) * a.q.head + grp * 8;
#pragma unroll
        for (int f = 0; f < HD / 16; ++f) qf[f] = *(const u32x4*)(p + f * 16);
    };
    Tile<HD> next;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)&lds[0][0];
    const uint32_t wave_at = __builtin_amdgcn_readfirstlane(lds_at + wave * 1024);
    auto copy = [&](int buf, int j0) {  // 64 slots, 16 bytes per thread and piece
        const uint8_t* from = packed + (int64_t)(j0 / kSlots) * Tile<HD>::kBytes;
#pragma unroll
        for (int i = 0; i < Tile<HD>::kPieces; ++i)
            copy_to_lds(from + i * 4096, threadIdx.x * 16, wave_at + buf * Tile<HD>::kBytes + i * 4096);
    };
    // `least`: slots that the first row of the tile that uses them sees
    auto store = [&](int buf, int j0, int least) {
        if (next.store(lds[buf], j0, total, j0 + kSlots > least)) nan[buf] = j0 + 1;
    };
    if (PACKED) {
        copy(0, first);
    } else {
        if (threadIdx.x < 2) nan[threadIdx.x] = 0;
        __syncthreads();
        next.load(c, K, V, ks, vs, first, total);
        store(0, first, q.cached + tile * kRows / G + 1);
        next.load(c, K, V, ks, vs, first + kSlots < sees_of(tile) ? first + kSlots : first, total);  // the one after it
    }
    load_q(tile);
    const int v_at = Tile<HD>::v_place(col, grp, 0);
    int buf = 0;
    for (int k = 0; tile >= 0; ++k) {
        const int row0 = tile * kRows, sees = sees_of(tile), end = min(first + sp.per, sees);
        const int least = q.cached + row0 / G + 1;  // slots that the first row sees
        const int r = row0 + wave * 32 + col;
        const int limit = q.cached + min(r, rows - 1) / G + 1;
        const int wave_least = q.cached + min(row0 + wave * 32, rows - 1) / G + 1;
        const int wave_most = q.cached + min(row0 + wave * 32 + 31, rows - 1) / G + 1;
        const int within = min(limit, end) - 4 * grp;  // slots of this range that the row sees, less the lane's own offset
        const bool active = row0 + wave * 32 < rows;
        const int tile_next = tile_of(k + 1);
        f32x16 acc[HD / 32];
#pragma unroll
        for (int m = 0; m < HD / 32; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][i] = 0.f;
        float ref = kEmpty, sum = 0.f;
        // q is waited for here: a wait in the loop would be one for the copies of the next slots, too
#pragma unroll
        for (int f = 0; f < HD / 16; ++f) asm volatile("" : "+v"(qf[f]));
        for (int j0 = first; j0 < end; j0 += kSlots, buf ^= 1) {
            if (PACKED) wait_copies<0>();
            __syncthreads();  // the slots are there, and nobody reads the other buffer any more
            const bool more = j0 + kSlots < end;
            if (more || tile_next >= 0) {  // the next slots, or the first ones again for the next rows
                if (PACKED) {
                    copy(buf ^ 1, more ? j0 + kSlots : first);
                } else {
                    store(buf ^ 1, more ? j0 + kSlots : first, more ? least : q.cached + tile_next * kRows / G + 1);
                    const int then = (more ? j0 + kSlots : first) + kSlots;  // and the ones after that
                    next.load(c, K, V, ks, vs, then < (more ? end : sees_of(tile_next)) ? then : first, total);
                }
            }
            if (!active || j0 >= wave_most) continue;
            const bool holes = PACKED ? odd[j0 / kSlots] != 0 : nan[buf] == j0 + 1;
            f32x16 z[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int i = 0; i < 16; ++i) z[t][i] = 0.f;
#pragma unroll
                for (int f = 0; f < HD / 16; ++f) z[t] = mfma32(lds[buf][(t * (HD / 16) + f) * 64 + lane], qf[f], z[t]);
            }
            const bool whole = j0 + kSlots <= wave_least && j0 + kSlots <= end;
            if (!whole) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (t * 32 + row_of(i, 0) >= within - j0) z[t][i] = -__builtin_inff();
                    }
            }
            float top = z[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, z[t][i]);
            top *= a.qscale;
            if (__any(top > ref + kRise)) {
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float now = top > ref + kRise ? reference_of(top) : ref;
                const float f = __builtin_amdgcn_exp2f(ref - now);
                ref = now;
                sum *= f;
#pragma unroll
                for (int m = 0; m < HD / 32; ++m)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[m][i] *= f;
            }
            exponents(ref, kAbove, a.qscale, [&](auto&& of) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[t][i] = of(z[t][i]);
            });
            u32x4 pf[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(z[u >> 1][(u & 1) * 8 + i]);
                    sum += p[i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) pf[u][i] = pack_bf16(p[2 * i], p[2 * i + 1]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int m = 0; m < HD / 32; ++m) acc[m] = mfma32(lds[buf][(Tile<HD>::kUnits + u * (HD / 32) + m) * 64 + (v_at ^ (m >> 1) << 3)], pf[u], acc[m]);
            if (holes) {  // NaN codes that were left out: back in for the rows that see them
                for (int j = j0; j < min(j0 + kSlots, end); ++j)
#pragma unroll
                    for (int m = 0; m < HD / 32; ++m)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (j < limit && (V[(int64_t)j * HD + m * 32 + row_of(i, grp)] & 0x7f) == 0x7f) acc[m][i] = __builtin_nanf("");
            }
        }
        if (tile_next >= 0) load_q(tile_next);
        sum += __shfl_xor(sum, 32, 64);
        if ((sees + sp.per - 1) / sp.per > 1) {  // several ranges: merged later
            if (r < rows) {
                const int64_t at = ((int64_t)pair * sp.ranges + range) * sp.tile_rows + r;
#pragma unroll
                for (int m = 0; m < HD / 32; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *(f32x4*)(sp.acc + at * HD + m * 32 + row_of(i * 4, grp)) = f32x4{acc[m][4 * i], acc[m][4 * i + 1], acc[m][4 * i + 2], acc[m][4 * i + 3]};
                if (grp == 0) sp.ml[at] = make_float2(ref, sum);
            }
        } else {
            const float inv = 1.f / sum;
            if (sp.final_ml != nullptr && grp == 0 && r < rows) sp.final_ml[(int64_t)pair * sp.tile_rows + r] = make_float2(ref, inv * kBelow);
            // The rows go through the buffer that is done with, so that each leaves in one piece; its 16-byte pieces lie
            // at an xor of the row, which spreads them over the banks.
            constexpr int PPR = HD / 8;  // pieces of a row
            __syncthreads();
            u32x4* mine = &lds[buf ^ 1][0] + wave * 32 * PPR;
#pragma unroll
            for (int m = 0; m < HD / 32; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    u32x2 w;
                    w.x = pack_bf16(acc[m][4 * i] * inv, acc[m][4 * i + 1] * inv);
                    w.y = pack_bf16(acc[m][4 * i + 2] * inv, acc[m][4 * i + 3] * inv);
                    ((u32x2*)(mine + col * PPR + ((m * 4 + i) ^ (col % PPR))))[grp] = w;
                }
            // the lane's rows, 64 / PPR apart
            constexpr int APART = 64 / PPR;
            int at = row0 + wave * 32 + lane / PPR, g = at % G;
            uint16_t* o = a.out.p + (int64_t)(q.row0 + at / G) * a.out.row + (int64_t)(hk * G + g) * a.out.head + lane % PPR * 8;
            const int step_g = APART % G;
            const int64_t step = (int64_t)(APART / G) * a.out.row + (int64_t)step_g * a.out.head, wrap = a.out.row - (int64_t)G * a.out.head;
#pragma unroll
            for (int i = 0; i < PPR / 2; ++i) {
                const int in = i * APART + lane / PPR;
                // past the caches, which K and V need: 32 prompts of 512 tokens 126 us instead of 130, 64 of 256 95 and 100
                if (at < rows) __builtin_nontemporal_store(mine[in * PPR + (lane % PPR ^ in % PPR)], (u32x4*)o);
                at += APART;
                o += step;
                g += step_g;
                if (g >= G) {
                    g -= G;
                    o += wrap;
                }
            }
        }
        tile = tile_next;
    }
}

// The weights of 128 slots (32 per wavefront, K in registers) from all rows that see them: S^T again, then
// exp2(score - reference) * 2^-kAbove / sum with the row's statistics, which are the lane's; added up over the rows in the lane, over
// the lanes at the end.  32 rows of q at a time come into LDS in the order of the matrix instructions, shared by the
// wavefronts, three tiles ahead of their use.  Bound by the exponentials and, next to them, the matrix cores: 1941 tokens of 2
// query heads per group over up to 6801 slots (39 GFLOP of the first product) 72 us.
constexpr int kWeightSlots = 128;
template <int HD>
__global__ __launch_bounds__(256, 4) void prompt_weights_kernel(Cache c, Step s, Attend a, Split sp, int chunks) {
    constexpr int F = HD / 16, U = F < 4 ? 1 : F / 4;  // units of 32 rows; units that a wavefront copies
    constexpr int RING = 4;                            // tiles of 32 rows in LDS, RING - 1 of them on their way
    __shared__ u32x4 qt[RING][F * 64];
    __shared__ float2 ml[RING][32];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5;
    const int pairs = c.n_seq * c.Hkv;
    const int pair = blockIdx.x % pairs, chunk = blockIdx.x / pairs % chunks, split = blockIdx.x / pairs / chunks;
    const int seq = pair / c.Hkv, hk = pair % c.Hkv, G = a.Hq / c.Hkv;
    const Seq q = sequence(c, s, seq);
    const int total = q.cached + q.n_new, rows = q.n_new * G;
    const int w0 = chunk * kWeightSlots, j0 = w0 + wave * 32;
    if (w0 >= total) return;
    const int64_t base = (int64_t)pair * c.max_len;
    u32x4 kf[F];
    {
        const int slot = min(j0 + col, total - 1);
        const float sc = c.scale[0][(int64_t)pair * (c.max_len >> c.logb) + (slot >> c.logb)];
        const uint8_t* K = c.codes[0] + (base + slot) * HD + grp * 8;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const u32x2 x = *(const u32x2*)(K + f * 16);
            kf[f] = widen8(x.x, x.y, sc);
        }
#pragma unroll
        for (int f = 0; f < F; ++f) asm volatile("" : "+v"(kf[f]));  // waited for here, not in the loop
    }
    float w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = 0.f;
    // tiles of 32 rows from the first that sees one of the slots on, those of this split
    const int tile0 = max(0, w0 - q.cached) * G / 32, tiles = (rows + 31) / 32 - tile0;
    const int r_first = (tile0 + tiles * split / sp.splits) * 32, r_end = (tile0 + tiles * (split + 1) / sp.splits) * 32;
    const uint32_t qt_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)&qt[0][0];
    const uint32_t ml_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float2*)&ml[0][0];
    const float* stats = (const float*)(sp.final_ml + (int64_t)pair * sp.tile_rows);
    // The lane's row of q in the next tile to copy, stepped on by 32 rows; past the end the last row again.
    const uint16_t* heads = a.q.p + (int64_t)hk * G * a.q.head + grp * 8;
    const uint16_t* last = heads + (int64_t)(q.row0 + q.n_new - 1) * a.q.row + (int64_t)(G - 1) * a.q.head;
    int row = r_first + col, g = row % G;
    const uint16_t* from = heads + (int64_t)(q.row0 + row / G) * a.q.row + (int64_t)g * a.q.head;
    const int step_g = 32 % G;
    const int64_t step = (int64_t)(32 / G) * a.q.row + (int64_t)step_g * a.q.head, wrap = a.q.row - (int64_t)G * a.q.head;
    // U + 1 copies of every wavefront, so that it can count them (where there are more wavefronts than units some copy
    // the same, and so do all the statistics)
    auto copy = [&](int at, int r0) {
        const uint16_t* p = row < rows ? from : last;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int f = (wave * U + i) % F;
            copy_to_lds(p + f * 16, __builtin_amdgcn_readfirstlane(qt_at + (at * F + f) * 1024));
        }
        copy_word_to_lds(stats + min(r0 + (lane >> 1), rows - 1) * 2 + (lane & 1), __builtin_amdgcn_readfirstlane(ml_at + at * 256));
        row += 32;
        from += step;
        g += step_g;
        if (g >= G) {
            g -= G;
            from += wrap;
        }
    };
    if (rows > 0) {  // a sequence without new tokens has no row of q, and its weights stay
#pragma unroll
        for (int i = 0; i < RING - 1; ++i) copy(i, r_first + i * 32);
    }
    const int r_see = (j0 - q.cached) * G, r_whole = (j0 + 31 - q.cached) * G;  // first rows that see a slot of the wavefront, and all
    int at = 0;
    for (int r0 = r_first; r0 < r_end; r0 += 32, at = (at + 1) % RING) {
        wait_copies<(RING - 2) * (U + 1)>();  // all but the two youngest tiles
        __syncthreads();
        copy((at + RING - 1) % RING, r0 + (RING - 1) * 32);  // past the end: again, so that the count stays
        if (r0 + 31 < r_see) continue;
        const float2 stat = ml[at][col];
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
        for (int f = 0; f < F; ++f) z = mfma32(kf[f], qt[at][f * 64 + lane], z);
        exponents(stat.x, 0.f, a.qscale, [&](auto&& of) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = of(z[i]);
        });
        if (r0 + 32 <= rows && r0 >= r_whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                w[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(z[i]), stat.y, w[i]);
        } else {
            const int within = r0 + col < rows ? q.cached + (r0 + col) / G + 1 - j0 - 4 * grp : 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = __builtin_amdgcn_exp2f(z[i]) * stat.y;
                w[i] += row_of(i, 0) < within ? x : 0.f;
            }
        }
    }
    wait_copies<0>();
    // Sums over the 32 lanes of a row of registers: each step hands half of a lane's registers to its partner, so that 16 exchanges
    // do (each register through all lanes would be 80).  Lane l ends up with the slot of register l/2 % 16.
#pragma unroll
    for (int half = 8; half >= 1; half /= 2) {
        const bool up = (lane & 2 * half) != 0;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float keep = up ? w[i + half] : w[i], give = up ? w[i] : w[i + half];
            w[i] = keep + __shfl_xor(give, 2 * half, 64);
        }
    }
    float x = w[0] + __shfl_xor(w[0], 1, 64);
    const int slot = j0 + row_of(col >> 1, grp);
    if ((col & 1) == 0 && slot < total) {
        if (sp.splits > 1) {
            sp.part[((int64_t)split * pairs + pair) * sp.score_stride + slot] = x;
            return;
        }
        if (a.weight_in != nullptr && slot < q.cached) x += a.weight_in[base + slot];
        a.weight_out[base + slot] = x;
    }
}

// Where the rows were split: what the splits gave each slot, in order.
__global__ __launch_bounds__(256) void sum_weights_kernel(Cache c, Step s, Attend a, Split sp) {
    const int pairs = c.n_seq * c.Hkv, pair = blockIdx.x % pairs, slot = blockIdx.x / pairs * 256 + (int)threadIdx.x;
    const Seq q = sequence(c, s, pair / c.Hkv);
    if (slot >= q.cached + q.n_new) return;
    const int64_t at = (int64_t)pair * c.max_len + slot;
    float w = a.weight_in != nullptr && slot < q.cached ? a.weight_in[at] : 0.f;
    for (int i = 0; i < sp.splits; ++i) w += sp.part[((int64_t)i * pairs + pair) * sp.score_stride + slot];
    a.weight_out[at] = w;
}

int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

// How a step is run, from its sizes and bounds.
struct Plan {
    int tiles;  // row tiles of decode_kernel; 0: many new tokens, in `row_tiles` tiles of kRows
    int row_tiles, each;  // `each`: row tiles of a workgroup
    Split sp;
    int64_t o_ml, o_scores, o_final, o_part, o_packed, o_odd, bytes;
};

// Slots of a range where there are many new tokens: `rows` in about `tiles` row tiles, which see `most` slots at most.
// More row tiles than compute units stay whole: 352 tiles of 8700 slots take 286 us, and 278 in the best of all splits; 384 of 8500
// 271 and 274; 512 of 4000 to 6000 181 and 227.  Fewer are split into as many ranges as make one workgroup per unit, two, or two rounds
// of two, by what a split costs in steps of kSlots of a workgroup alone on its unit: two run at 1.45 times that (1.6 and 2.3 us), each
// has three more for its start and end, a merge costs a launch and fp32 sums written and read.  Whole / as chosen: 128 tiles of 8500
// slots 213 / 96 us, 256 of 16500 409 / 321, 80 of 4300 110 / 46, 24 of 260 to 2060 32 / 15.
int64_t prompt_range(int64_t most, int64_t tiles, int64_t rows) {
    const int64_t steps = (most + kSlots - 1) / kSlots;
    int64_t best = steps;
    double least = (double)steps + 3.;
    if (tiles > 256 || tiles < 1) return best * kSlots;
    for (int fill = 1; fill <= 4 && steps >= 8; fill *= 2) {
        int64_t n = 256 * fill / tiles;
        n = n > steps / 4 ? steps / 4 : n;
        const int64_t per = (steps + n - 1) / n, ranges = (steps + per - 1) / per, groups = tiles * ranges;
        const double rounds = groups <= 512 ? 1. : (groups / 512. + (groups + 511) / 512) / 2;  // the last one not quite full
        const double cost = (groups <= 256 ? 1. : 1.45 * rounds) * (double)(per + 3) + 1. + rows * ranges / (70. * kRows);
        if (cost < least) {
            least = cost;
            best = per;
        }
    }
    return best * kSlots;
}

int64_t weight_chunks(const Split& sp) { return (sp.score_stride + kWeightSlots - 1) / kWeightSlots; }

Plan plan(const Cache& c, const Step& s, int Hq, bool weights) {
    Plan p{};
    const int64_t pairs = (int64_t)c.n_seq * c.Hkv, rows = (int64_t)s.max_new * (Hq / c.Hkv);
    const int most = (int)min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len);
    // decode_kernel up to 16 rows, the most whose sums its registers hold.  4 tokens of 4 query heads that way / as a prompt: 64
    // sequences of 1000 slots 29 / 36 us, 512 of 512 146 / 163, 8 of 8000 32 / 39; 3 tokens of 512 with weights 165 / 340.
    p.tiles = rows == 0 ? 0 : rows <= 8 ? 1 : rows <= 16 ? 2 : 0;  // without rows prompt_weights_kernel carries the weights over
    p.row_tiles = (int)((rows + kRows - 1) / kRows);
    p.sp.tile_rows = p.tiles > 0 ? p.tiles * 8 : p.row_tiles * kRows;
    int64_t per;
    if (p.tiles > 0) {
        // About 512 workgroups of 256 slots and more: a range costs its start, its end and its sums written and read.  Aiming at
        // 512, 1024, 4096 workgroups: 1 sequence of 32000 slots 20, 23, 23 us; 4 of 8000 22, 24, 24; 64 of 750 21, 29, 33;
        // 256 of 100 to 1500 96, 117, 149; 16 of 2000 19, 21, 21.
        per = ((int64_t)most * pairs / 512 + 127) / 128 * 128;
        per = per < 256 ? 256 : per;
        // Short sequences whole, since that takes one launch.  1 sequence, heads of 128, in ranges / whole: 300 slots 9.9 / 7.9 us, 700
        // 10.3 / 9.9, 1000 10.4 / 11.2, with weights 600 11.9 / 11.0, 700 11.1 / 11.8; of 64: 1500 11.1 / 10.9, with weights 1000 11.9 /
        // 11.1; of 32: 1500 11.1 / 9.9, with weights 11.9 / 12.9.  48 sequences of 700: 21.7 / 16.1.
        if (most <= (weights ? c.hd == 128 ? 640 : 1024 : c.hd == 128 ? 768 : 1536)) per = (most + 127) / 128 * 128;
    } else {
        const int64_t rows2 = 2 * s.n_rows * (int64_t)(Hq / c.Hkv) / kRows, about = (rows2 + c.n_seq + 1) / 2;  // half a tile over each
        const int64_t tiles = c.Hkv * (about > c.n_seq ? about : (int64_t)c.n_seq);
        per = prompt_range(most, min(pairs * p.row_tiles, tiles), s.n_rows * (int64_t)Hq);
    }
    per = min(per, ((int64_t)most + 127) / 128 * 128);
    const int64_t ranges = most > per ? (most + per - 1) / per : 1;
    p.sp.per = (int)per;
    p.sp.ranges = (int)ranges;
    p.sp.score_stride = (most + 31) / 32 * 32;
    // Short prompts: two row tiles and more per workgroup while 1024 workgroups remain (32 prompts of 512 tokens 150 us
    // with one, 145 with two, 144 with four); long ones keep the order of the heaviest first (two prompts of 4096: 277, 281, 284).
    p.each = 1;
    while (ranges == 1 && most <= 1024 && p.each < 4 && pairs * p.row_tiles >= 1024 * p.each) p.each *= 2;
    int64_t o = 0;
    const int64_t items = ranges > 1 ? pairs * ranges * p.sp.tile_rows : 0;
    o += up256(items * c.hd * 4);
    p.o_ml = o;
    o += up256(items * 8);
    p.o_scores = o;
    if (weights && p.tiles > 0) {
        // The products stay in LDS where a sequence is one range and they fit the 64 KiB that a workgroup can have beside the
        // sums: 512 sequences of 513 slots 114 us instead of 137, 96 of up to 3002 (48 KB, two workgroups per unit) 52, not 63.
        // From 32 KiB on, where few workgroups share a unit, they have eight wavefronts.  Four / eight: 96 of up to 3002 slots
        // (48 KB) 53 / 41 us, 200 of 2101 (34 KB) 103 / 94, 256 of 1001 with 8 rows (33 KB) 69 / 64, 200 of up to 1701 (28 KB) 45 / 48.
        const int64_t stride = (most + 63) / 64 * 64 + 16, lds = rows * stride * 4;  // rows 16 banks apart
        const auto room = [&](int waves) { return (64 << 10) - p.tiles * 8 * (4 * waves * c.hd + 8 * waves + 8); };
        if (ranges == 1 && lds <= room(4)) {
            p.sp.waves = lds > (32 << 10) && lds <= room(8) ? 8 : 4;
            p.sp.score_stride = (int)stride;
            p.sp.lds_scores = (int)lds;
        } else {
            o += up256(pairs * p.sp.tile_rows * p.sp.score_stride * 4);
        }
    }
    p.o_final = o;
    p.sp.splits = 1;
    if (weights && p.tiles == 0) {
        o += up256(pairs * p.sp.tile_rows * 8);
        // prompt_weights_kernel: where the slots alone make less than 450 workgroups the rows are split, too, down to eight tiles of
        // 32; with 64 tiles and more per split up to 2048 workgroups, since those of late slots see few rows.  The whole call, not
        // split / split: 1 prompt of 700 tokens of 16/2 heads 106 / 38 us, of 32/8 heads 77 / 41, of 4096 415 / 278, 2 of 4096
        // 564 / 490; splits of four tiles and of two instead of eight: 700 tokens of 16/2 heads 42 and 53.
        const int64_t groups = pairs * weight_chunks(p.sp), split = groups > 0 ? max(min(900 / groups, rows / 256), min(2048 / groups, rows / 2048)) : 1;
        p.sp.splits = split > 1 ? (int)split : 1;
    }
    p.o_part = o;
    if (p.sp.splits > 1) o += up256(p.sp.splits * pairs * p.sp.score_stride * 4);
    p.o_packed = o;
    // Dequantised once where many row tiles use a tile, and the copy stays under 4 GiB.  Ahead / on the way: 32 prompts of 512
    // (16 row tiles) 144 / 134 us, 16 of 1024 (32) 212 / 217, 8 of 2048 (64) 319 / 343, 1 of 4096 (128) 232 / 270.
    const int64_t tiles = (most + kSlots - 1) / kSlots, copy = pairs * tiles * kSlots * c.hd * 4;
    if (p.tiles == 0 && p.row_tiles >= 32 && copy <= (int64_t)4 << 30) {
        p.sp.packed_tiles = (int)tiles;
        o += up256(copy);
        p.o_odd = o;
        o += up256(pairs * tiles * 4);
    }
    p.bytes = o;
    return p;
}

// Workgroups of the launches of a step.
struct Grids {
    int64_t attend;           // decode_kernel or prompt_kernel
    int64_t pack;             // pack_kernel
    int64_t merges, chunks;   // merge_kernel; with few new tokens finish_kernel, `chunks` per pair behind them
    int64_t weights, sums;    // prompt_weights_kernel, sum_weights_kernel
};
Grids grids(const Cache& c, const Step& s, const Plan& p, bool weights) {
    Grids g{};
    const int64_t pairs = (int64_t)c.n_seq * c.Hkv, rows = pairs * p.sp.tile_rows;
    if (s.n_rows > 0) {
        g.attend = pairs * p.sp.ranges * (p.tiles > 0 ? 1 : (p.row_tiles + p.each - 1) / p.each);
        g.pack = pairs * p.sp.packed_tiles;
        if (p.sp.ranges > 1 && p.tiles > 0) {
            g.merges = p.sp.ranges > 8 ? rows : (rows + 3) / 4;
            g.chunks = weights ? (p.sp.score_stride + 255) / 256 : 0;
        } else if (p.sp.ranges > 1) {
            g.merges = rows <= 4 * 2048 ? (rows + 3) / 4 : (rows / 4 + 3) / 4;
        }
    }
    if (weights && p.tiles == 0) {
        g.weights = pairs * weight_chunks(p.sp) * p.sp.splits;
        if (p.sp.splits > 1) g.sums = pairs * ((p.sp.score_stride + 255) / 256);
    }
    return g;
}

template <int HD, int NT>
void launch_decode(hipStream_t st, const dim3& grid, const Cache& c, const Step& s, const Attend& a, const Split& sp) {
    // Caches beyond the last-level cache of 256 MiB are read past it: 512 sequences of 513 slots (538 MB) 98 us with ordinary
    // loads, 91 without; 4 of 8000 (61 MB), read again before they are evicted, 31 and 32.
    const bool stream = (int64_t)c.n_seq * c.Hkv * min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len) * HD * 2 > (256 << 20);
    auto launch = [&](auto mode) {
        constexpr int SCORES = decltype(mode)::value;
        const unsigned lds = SCORES == kScoresLds ? (unsigned)sp.lds_scores : 0u;
        if constexpr (SCORES == kScoresLds && NT * HD <= 64) {  // with larger sums eight wavefronts leave no 32 KiB
            if (sp.waves == 8) {
                if (stream) hipLaunchKernelGGL((decode_kernel<HD, NT, SCORES, true, 8>), grid, dim3(512), lds, st, c, s, a, sp);
                else hipLaunchKernelGGL((decode_kernel<HD, NT, SCORES, false, 8>), grid, dim3(512), lds, st, c, s, a, sp);
                return;
            }
        }
        if (stream) hipLaunchKernelGGL((decode_kernel<HD, NT, SCORES, true, 4>), grid, dim3(256), lds, st, c, s, a, sp);
        else hipLaunchKernelGGL((decode_kernel<HD, NT, SCORES, false, 4>), grid, dim3(256), lds, st, c, s, a, sp);
    };
    if (a.weight_out == nullptr) launch(std::integral_constant<int, kNoScores>{});
    else if (sp.lds_scores > 0) launch(std::integral_constant<int, kScoresLds>{});
    else launch(std::integral_constant<int, kScores>{});
}

template <int HD>
void launch_hd(hipStream_t st, const Cache& c, const Step& s, const Attend& a, const Plan& p) {
    const Grids g = grids(c, s, p, a.weight_out != nullptr);
    const auto grid = [](int64_t n) { return dim3((unsigned)n); };
    const dim3 block(256);
    const int groups = (int)(g.attend / ((int64_t)c.n_seq * c.Hkv * p.sp.ranges));  // of a pair and range
    if (g.attend > 0) {
        if (p.tiles == 1) launch_decode<HD, 1>(st, grid(g.attend), c, s, a, p.sp);
        else if (p.tiles == 2) launch_decode<HD, 2>(st, grid(g.attend), c, s, a, p.sp);
        else if (g.pack > 0) {
            hipLaunchKernelGGL(pack_kernel<HD>, grid(g.pack), block, 0, st, c, s, p.sp.packed, p.sp.odd, p.sp.packed_tiles);
            hipLaunchKernelGGL((prompt_kernel<HD, true>), grid(g.attend), block, 0, st, c, s, a, p.sp, groups, p.each);
        } else
            hipLaunchKernelGGL((prompt_kernel<HD, false>), grid(g.attend), block, 0, st, c, s, a, p.sp, groups, p.each);
    }
    if (g.merges > 0) {
        const dim3 all = grid(g.merges + (int64_t)c.n_seq * c.Hkv * g.chunks);
        if (p.tiles > 0 && p.sp.ranges > 8) hipLaunchKernelGGL((finish_kernel<HD, true>), all, block, 0, st, c, s, a, p.sp, (int)g.merges, (int)g.chunks);
        else if (p.tiles > 0) hipLaunchKernelGGL((finish_kernel<HD, false>), all, block, 0, st, c, s, a, p.sp, (int)g.merges, (int)g.chunks);
        else if ((int64_t)c.n_seq * c.Hkv * p.sp.tile_rows <= 4 * 2048) hipLaunchKernelGGL((merge_kernel<HD, 1>), all, block, 0, st, c, s, a, p.sp);
        else hipLaunchKernelGGL((merge_kernel<HD, 4>), all, block, 0, st, c, s, a, p.sp);
    }
    if (g.weights > 0) hipLaunchKernelGGL(prompt_weights_kernel<HD>, grid(g.weights), block, 0, st, c, s, a, p.sp, (int)weight_chunks(p.sp));
    if (g.sums > 0) hipLaunchKernelGGL(sum_weights_kernel, grid(g.sums), block, 0, st, c, s, a, p.sp);
}

}  // namespace

bool attend_fits(const Cache& c, const Step& s, int Hq, bool weights) {
    const Plan p = plan(c, s, Hq, weights);
    const Grids g = grids(c, s, p, weights);
    const int64_t pairs = (int64_t)c.n_seq * c.Hkv, most = min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len);
    if (weights && pairs * ((most + kWeightSlots - 1) / kWeightSlots) > kMostGroups) return false;  // whichever kernel sums them
    return g.attend <= kMostGroups && g.pack <= kMostGroups && g.merges + pairs * g.chunks <= kMostGroups &&
           g.weights <= kMostGroups && g.sums <= kMostGroups;
}

int64_t attend_workspace(const Cache& c, const Step& s, int Hq, bool weights) { return plan(c, s, Hq, weights).bytes; }

void launch_attend(hipStream_t st, const Cache& c, const Step& s, const Attend& a) {
    Plan p = plan(c, s, a.Hq, a.weight_out != nullptr);
    p.sp.acc = (float*)a.ws;
    p.sp.ml = (float2*)(a.ws + p.o_ml);
    p.sp.scores = (float*)(a.ws + p.o_scores);
    p.sp.part = (float*)(a.ws + p.o_part);
    p.sp.packed = (u32x4*)(a.ws + p.o_packed);
    p.sp.odd = (int32_t*)(a.ws + p.o_odd);
    p.sp.final_ml = a.weight_out != nullptr ? (float2*)(a.ws + p.o_final) : nullptr;
    if (c.hd == 32) launch_hd<32>(st, c, s, a, p);
    if (c.hd == 64) launch_hd<64>(st, c, s, a, p);
    if (c.hd == 128) launch_hd<128>(st, c, s, a, p);
}

}  // namespace kkv8
