// Attention over the latent cache in its absorbed form: all heads of all new tokens of a sequence are rows of one matrix
// A [rows, latent + rope], and z = A C^T, u = softmax(z) C[:, :latent] with the cache's rows C as keys and as values.
//
// A row of C has 1152 bytes (512 + 64) and takes part in 2 * (2 * 512 + 64) operations per row of A: bound by the bytes of
// the cache up to about 60 rows of A, by the matrix cores and the LDS that feeds them beyond.  Measured: 512 sequences of 513 slots, 32 heads,
// 302 MB in 61 us; 48 of 80 to 6001 slots, 128 heads, 105 us; 16384 rows over 4000 slots 200 us: a workgroup of 64 rows takes 64 slots in 3.2
// us, of which the products are 1.3 and the reads from LDS 1.4; the rest are the phases between barriers, which all wavefronts go through together.
// Each holds rows and sums both, so its registers are full and it cannot run one step's scores under another's sums; wavefronts that only
// score beside others that only sum have not been tried.
#include "latent_device.h"

namespace klat {
namespace {

// How C lies in LDS: tiles of 32 slots, cut into groups of 64 elements (128 bytes), a group being 32 slots x 8 units of 16 bytes.
// Unit u of slot r is at place u ^ twist(r): then neither the reads by slots (16 lanes, one unit each; keys) nor the transposed ones
// (8 slots, 64 bytes each; values) meet in a bank.  Rows whose width is half a group more than whole groups fill the last one twice.
template <int DC, int DR>
struct Tile {
    static constexpr int kWidth = DC + DR, kGroups = (kWidth + 63) / 64, kBytes = kGroups * 4096;
    static constexpr bool kHalf = kWidth % 64 != 0;
};

struct Run {  // the rows of the sequences over their own slots, or all rows over the prefix
    int H, row_tiles;  // tiles of 32 * MT rows of a sequence (of the prefix: of all)
    int per, ranges;   // slots of a range, ranges at most
    int part0;         // where the launch's parts are among a row's
    bool packed;       // see place_of
    float qscale;
    const uint16_t* a;  // [row, head, 2 * latent + rope], see absorb_kernel
    Parts parts;
};
struct Both {  // one launch: the first `before` workgroups have the prefix, the others the sequences
    Run pre, own;
    int before;
};

// The lane, counted anew.  The loop below has no register to spare: what it needs of the lane now and then is made of this, where the compiler would
// keep each address in a register of its own and then, short of them, read every key right before its products (48
// sequences of 80 to 6001 slots, 128 heads 120 us, so 106).
__device__ __forceinline__ int lane_now() {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(l));
    return l;
}

struct Place {
    int seq, tile, range;
};

// Work of a workgroup among what the sequences have of it: whole ranges, then last ones of half a range and more, then the shorter ones, so that the
// long ones start first and every XCD gets as many.  Laid out by the bounds, where a workgroup of a short sequence finds nothing to do, one XCD has
// more than its compute units take at once and another none: 48 sequences of 80 to 6001 slots, 128 heads 143 us so
// (and in three ranges, see split), packed 121.
template <int M>
__device__ __forceinline__ bool place_of(const Cache& c, const Step& s, const Run& run, int block, int blocks, Place* at) {
    const int lane = threadIdx.x & 63;
    int left = block;
    // two tiles of a range to one XCD, which then reads its slots once
    if (run.row_tiles > 1 && (left | 15) < blocks) left = (left & ~15) + (left & 7) * 2 + (left >> 3 & 1);
    for (int kind = 0; kind < 3; ++kind)
        for (int first = 0; first < c.n_seq; first += 64) {
            int tiles = 0, full = 0, here = 0;
            if (first + lane < c.n_seq) {
                const Seq q = kkv8::sequence(c.max_len, s, first + lane);
                if (q.n_new > 0) {
                    tiles = (q.n_new * run.H + M - 1) / M;
                    full = (q.cached + q.n_new) / run.per;
                    const int rest = q.cached + q.n_new - full * run.per;
                    here = kind == 0 ? tiles * full : rest > 0 && (2 * rest >= run.per) == (kind == 1) ? tiles : 0;
                }
            }
            int upto = here;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int y = __shfl_up(upto, d, 64);
                if (lane >= d) upto += y;
            }
            const uint64_t has = __ballot(upto > left);
            if (has != 0) {
                const int who = __builtin_ctzll(has);
                const int in = left - __builtin_amdgcn_readlane(upto - here, who), n = __builtin_amdgcn_readlane(tiles, who);
                at->seq = first + who;
                at->tile = n - 1 - in % n;  // those that see the most slots first
                at->range = kind == 0 ? in / n : __builtin_amdgcn_readlane(full, who);
                return true;
            }
            left -= __builtin_amdgcn_readlane(upto, 63);
        }
    return false;
}

// A workgroup of 4 * MT wavefronts takes 32 * MT rows of A and a range of slots, SUB tiles at a time (a step; the next one comes
// meanwhile, without registers):
//   scores  z^T = C A^T, 16 slots x 16 rows, 16x16x32: a wavefront has 16 rows of A (in registers, as two bf16: see absorb_kernel; the
//           second halves double the work of this product) and one half of every tile.  A lane has one row and four slots.
//   sums    u^T = C^T w, 32 latents x 32 rows, 32x32x16: a wavefront has some blocks of 32 latents for all rows.  The weights go through LDS,
//           the values are read from it transposed.
// So a tile is read once from memory for all rows, its keys by the wavefronts of half the rows each and its values once; the sums take
// 64 registers and the rows 136, which leaves two wavefronts to a SIMD.
// References of the softmax are whole numbers, so that bringing sums or weights from one to another is exact.  The two wavefronts of a row
// set theirs by their own halves; behind the barrier everybody sees both and goes on with the larger one.
template <int DC, int DR, int MT, bool STREAM>
__global__ __launch_bounds__(256 * MT, 2) void absorbed_kernel(Cache c, Step s, Both both) {
    typedef Tile<DC, DR> T;
    constexpr int WAVES = 4 * MT, GROUPS = 2 * MT, SUB = MT, M = 32 * MT;
    constexpr int KEYS = T::kWidth / 32, LOW = DC / 32;               // products of a score: first halves, second ones
    constexpr int BLOCKS = DC / 32 * MT / WAVES;                      // (block of latents, 32 rows) of a wavefront
    constexpr int ROW_TILES = BLOCKS >= MT ? MT : 1;                  // of them 32-row tiles
    constexpr int COLS = BLOCKS / ROW_TILES;                          // and blocks of latents
    constexpr int STEP = SUB * T::kBytes, RING = 2 * STEP, SUMS = M * DC * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[RING > SUMS ? RING : SUMS];
    __shared__ __attribute__((aligned(16))) uint8_t weights[SUB * M * 64];  // [tile][row][32 slots] bf16
    __shared__ float sm_ref[2][M], sm_sum[2][M];
    __shared__ int sm_limit[M];  // slots of the range that a row sees end here
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5, c16 = lane & 15, g16 = lane >> 4;
    const int rows16 = wave % GROUPS, half = wave / GROUPS;
    const bool prefix = (int)blockIdx.x < both.before;
    const Run run = prefix ? both.pre : both.own;
    const int block = prefix ? blockIdx.x : blockIdx.x - both.before;
    // of the prefix the ranges, each to its XCD; of a sequence the row tiles one behind the other, so that they read its slots together
    Place at{0, run.row_tiles - 1 - block / run.ranges, block % run.ranges};
    if (!prefix) {
        if (run.packed) {
            if (!place_of<M>(c, s, run, block, (int)gridDim.x - both.before, &at)) return;
        } else {
            const int rest = block / c.n_seq;
            at = Place{block % c.n_seq, run.row_tiles - 1 - rest % run.row_tiles, rest / run.row_tiles};
        }
    }
    const int seq = __builtin_amdgcn_readfirstlane(at.seq), tile = __builtin_amdgcn_readfirstlane(at.tile), range = __builtin_amdgcn_readfirstlane(at.range);
    Seq q{0, s.n_rows, 0};
    if (!prefix) q = kkv8::sequence(c.max_len, s, seq);
    q.row0 = __builtin_amdgcn_readfirstlane(q.row0);
    q.n_new = __builtin_amdgcn_readfirstlane(q.n_new);
    q.cached = __builtin_amdgcn_readfirstlane(q.cached);
    const int rows = q.n_new * run.H, row0 = tile * M;
    if (row0 >= rows) return;
    const int first = range * run.per;
    const int sees = prefix ? c.prefix_len : q.cached + (min(row0 + M, rows) - 1) / run.H + 1;  // slots that the last row sees
    const int end = min(first + run.per, sees);
    if (first >= end) return;
    const uint16_t* C = prefix ? c.prefix : c.rows + (int64_t)seq * c.max_len * T::kWidth;
    const int mine = min(row0 + rows16 * 16 + c16, rows - 1);                    // the lane's row, for the scores
    if (g16 == 0 && half == 0) sm_limit[rows16 * 16 + c16] = min(prefix ? c.prefix_len : q.cached + mine / run.H + 1, end);
    const int all_see = prefix ? c.prefix_len : q.cached + row0 / run.H + 1;     // slots that every row sees
    const int64_t row_head = (int64_t)q.row0 * run.H + row0;

    // copies: a wavefront brings 8 slots x 8 units at a time, one quarter of a tile
    const uint32_t lds_at = lds_address(lds);
    const int quarter = wave & 3, sub = wave >> 2;
    const uint32_t copy_at = __builtin_amdgcn_readfirstlane(lds_at + sub * T::kBytes + quarter * 1024);
    auto copy = [&](int buf, int j0) {
        const int l = lane_now(), in8 = l >> 3;
        const uint32_t unit_at = (uint32_t)(((l & 7) ^ twist(quarter * 8 + in8)) * 16);
        const uint32_t slot = (uint32_t)min(j0 + sub * 32 + quarter * 8 + in8, end - 1);  // past the end the last one again
        const uint32_t at = slot * (T::kWidth * 2) + unit_at;
#pragma unroll
        for (int g = 0; g < T::kGroups; ++g) {
            const bool cut = T::kHalf && g == T::kGroups - 1;  // the row ends within the group
            const uint32_t from = cut ? slot * (T::kWidth * 2) + (unit_at & 63) : at, to = copy_at + buf * STEP + g * 4096;
            if constexpr (STREAM) stream_to_lds((const uint8_t*)C + g * 128, from, to);
            else copy_to_lds((const uint8_t*)C + g * 128, from, to);
        }
    };
    copy(0, first);

    u32x4 hi[KEYS], lo[LOW];
    {
        const uint16_t* p = run.a + (row_head + (mine - row0)) * (T::kWidth + DC) + g16 * 8;
#pragma unroll
        for (int f = 0; f < KEYS; ++f) hi[f] = *(const u32x4*)(p + f * 32);
#pragma unroll
        for (int f = 0; f < LOW; ++f) lo[f] = *(const u32x4*)(p + T::kWidth + f * 32);
#pragma unroll
        for (int f = 0; f < KEYS; ++f) asm volatile("" : "+v"(hi[f]));  // waited for here, not in the loop
#pragma unroll
        for (int f = 0; f < LOW; ++f) asm volatile("" : "+v"(lo[f]));
    }
    f32x16 acc[COLS][ROW_TILES];
#pragma unroll
    for (int b = 0; b < COLS; ++b)
#pragma unroll
        for (int r = 0; r < ROW_TILES; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[b][r][i] = 0.f;
    const int block0 = (MT > 1 && ROW_TILES == 1 ? wave & 3 : wave) * COLS, tile32 = MT > 1 && ROW_TILES == 1 ? wave >> 2 : 0;
    float ref = kEmpty, sum = 0.f, sums_ref[ROW_TILES];
#pragma unroll
    for (int r = 0; r < ROW_TILES; ++r) sums_ref[r] = kEmpty;

    // the lane's places in a tile: units 4 * (f % 2) + g16 of its slot
    const int key_slot = half * 16 + c16;
    uint32_t key_at[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) key_at[f] = lds_at + (uint32_t)(key_slot * 128 + ((4 * f + g16) ^ twist(key_slot)) * 16);
    const uint32_t weights_at = lds_address(weights);

    const int steps = (end - first + SUB * 32 - 1) / (SUB * 32);
    for (int t = 0; t < steps; ++t) {
        const int j0 = first + t * SUB * 32, buf = t & 1;
        wait_copies<0>();
        __syncthreads();  // the step's tiles are there, and nobody reads the ones before it any more
        if (t + 1 < steps) copy(buf ^ 1, j0 + SUB * 32);
        // A latent that is not finite, in a slot that some row of the workgroup does not see, would reach that row as 0 times it.
        // In tiles where that can be, such slots give up their latents and get NaN in the part that only the scores read:
        // the rows that see them become NaN, as they have to, and no others.  Done by the wavefront that brought the slots.
        if (all_see < sees && j0 + SUB * 32 > all_see) {
            const int l = lane_now();
            const uint32_t at = lds_at + buf * STEP + sub * T::kBytes;
#pragma unroll 1
            for (int slot = quarter * 8; slot < quarter * 8 + 8; ++slot) {
                const uint32_t to = at + (l >> 3) * 4096 + slot * 128 + ((l & 7) ^ twist(slot)) * 16;
                // word by word: registers are short here
                bool bad = false;
#pragma unroll 1
                for (int e = 0; e < 16 && l * 8 < DC; e += 4) {
                    const uint32_t x = read_lds_word(to + e);
                    bad |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
                }
                if (__any(bad)) {
#pragma unroll 1
                    for (int e = 0; e < 16; e += 4) {
                        if (l * 8 < DC) write_lds_word(to + e, 0u);
                        if (l == 0) write_lds_word(at + (DC / 64) * 4096 + slot * 128 + twist(slot) * 16 + e, 0x7fff7fffu);
                    }
                }
            }
            __syncthreads();
        }
        // two chains of products, which do not wait for one another: of the two tiles, or of one tile's first and second halves
        f32x4 z[2];
        z[0] = z[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < KEYS; ++f)
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const u32x4 k = read_lds(key_at[f & 1] + buf * STEP + u * T::kBytes + (f >> 1) * 4096);
                z[u] = mfma16(k, hi[f], z[u]);
                if (f < LOW) z[SUB == 1 ? 1 : u] = mfma16(k, lo[f], z[SUB == 1 ? 1 : u]);
            }
        // four keys on their way ahead of their products: left to itself the compiler, short of registers, waits for every one
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < SUB * KEYS - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, 8, 0);
        if (SUB == 1) z[0] += z[1];
        const int l = lane_now(), my_row = rows16 * 16 + (l & 15);
        float top = -__builtin_inff();
        if (j0 + SUB * 32 > all_see || j0 + SUB * 32 > end) {
            const int within = sm_limit[my_row] - j0 - half * 16 - 4 * (l >> 4);
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i >= within - u * 32) z[u][i] = -__builtin_inff();
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, z[u][i]);
        top *= run.qscale;
        if (__any(top > ref + kRise)) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float now = top > ref + kRise ? ceilf(top) : ref;
            sum *= __builtin_amdgcn_exp2f(ref - now);
            ref = now;
        }
        exponents_of_rows(ref, kAbove, run.qscale, [&](auto&& of) {
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[u][i] = of(z[u][i]);
        });
        // weights: 64 bytes a row, its four units at an xor of the row
        const uint32_t put_at = weights_at + (uint32_t)(my_row * 64 + ((half * 2 + (l >> 5)) ^ (my_row >> 2 & 3)) * 16 + (l >> 4 & 1) * 8);
        u32x2 w[SUB];
        // Rounded to bf16: the products take both factors in one type, and the latents are read as they lie in the cache.  The sum is that of the
        // weights as rounded: then one slot that has nearly all of it counts nearly exactly.
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            w[u].x = pack_bf16(__builtin_amdgcn_exp2f(z[u][0]), __builtin_amdgcn_exp2f(z[u][1]));
            w[u].y = pack_bf16(__builtin_amdgcn_exp2f(z[u][2]), __builtin_amdgcn_exp2f(z[u][3]));
            sum += (bf_lo(w[u].x) + bf_hi(w[u].x)) + (bf_lo(w[u].y) + bf_hi(w[u].y));
            write_lds2(put_at + u * M * 64, w[u]);
        }
        if ((l >> 4) == 0) sm_ref[half][my_row] = ref;
        __syncthreads();
        // the references of a wavefront's lanes: row `lane` of all (32 of them twice with MT = 1)
        const float both0 = sm_ref[0][l & (M - 1)], both1 = sm_ref[1][l & (M - 1)];
        if (__any(both0 != both1)) {  // the same for the whole workgroup: halves that are behind bring their weights up
            const float now = fmaxf(ref, sm_ref[half ^ 1][my_row]), f = __builtin_amdgcn_exp2f(ref - now);
            sum *= f;
            ref = now;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
                write_lds2(put_at + u * M * 64, u32x2{pack_bf16(bf_lo(w[u].x) * f, bf_hi(w[u].x) * f), pack_bf16(bf_lo(w[u].y) * f, bf_hi(w[u].y) * f)});
            __syncthreads();
        }
        float now[ROW_TILES];
        bool moved = false;
#pragma unroll
        for (int r = 0; r < ROW_TILES; ++r) {
            const int row = (tile32 + r) * 32 + (l & 31);
            now[r] = fmaxf(sm_ref[0][row], sm_ref[1][row]);
            moved |= now[r] != sums_ref[r];
        }
        if (__any(moved)) {
#pragma unroll
            for (int r = 0; r < ROW_TILES; ++r) {
                const float f = __builtin_amdgcn_exp2f(sums_ref[r] - now[r]);
                sums_ref[r] = now[r];
#pragma unroll
                for (int b = 0; b < COLS; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[b][r][i] *= f;
            }
        }
        // Blocks of values AHEAD - 1 of their products, with the weights of half a tile: the order is laid down, since the compiler,
        // short of registers, would wait for every read.
        constexpr int AHEAD = MT == 2 ? 2 : 3, ITEMS = 2 * SUB * COLS;
        // four slots of 16 elements for the transposed reads
        uint32_t value_at[2][2];
#pragma unroll
        for (int odd = 0; odd < 2; ++odd)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int slot = 8 * (l >> 5) + 4 * j + (l >> 2 & 3), unit = odd * 4 + (l >> 4 & 1) * 2 + (l >> 1 & 1);
                value_at[odd][j] = lds_at + (uint32_t)(slot * 128 + (unit ^ twist(slot)) * 16 + (l & 1) * 8);
            }
        const uint32_t get_at = weights_at + (uint32_t)((tile32 * 32 + (l & 31)) * 64), get_xor = (uint32_t)(l >> 2 & 3);
        u32x4 p[2][ROW_TILES], v[AHEAD];
        auto fetch = [&](int n) {
            const int u = n / COLS >> 1, h = n / COLS & 1, b = n % COLS;
            if (b == 0) {
#pragma unroll
                for (int r = 0; r < ROW_TILES; ++r) p[h][r] = read_lds(get_at + u * M * 64 + r * 2048 + ((h * 2 + (l >> 5)) ^ get_xor) * 16);
            }
            const int odd = COLS > 1 ? b & 1 : block0 & 1;  // block0 is even wherever there is more than one block
            const uint32_t at = buf * STEP + u * T::kBytes + ((block0 + b) >> 1) * 4096 + h * 2048;
            v[n % AHEAD] = join(read_transposed((odd ? value_at[1][0] : value_at[0][0]) + at), read_transposed((odd ? value_at[1][1] : value_at[0][1]) + at));
        };
#pragma unroll
        for (int n = 0; n < AHEAD - 1; ++n) fetch(n);
#pragma unroll
        for (int n = 0; n < ITEMS; ++n) {
            if (n + AHEAD - 1 < ITEMS) fetch(n + AHEAD - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = 0; r < ROW_TILES; ++r) acc[n % COLS][r] = mfma32(v[n % AHEAD], p[n / COLS & 1][r], acc[n % COLS][r]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (g16 == 0) sm_sum[half][rows16 * 16 + c16] = sum;
    __syncthreads();  // the tiles are done with, too

    // The sums go through LDS, so that a row leaves in one piece; its 16-byte units lie at an xor of the row.
    constexpr int UNITS = DC / 4;
#pragma unroll
    for (int b = 0; b < COLS; ++b)
#pragma unroll
        for (int r = 0; r < ROW_TILES; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = (tile32 + r) * 32 + col, unit = (block0 + b) * 8 + 2 * i + grp;
                ((f32x4*)lds)[row * UNITS + (unit ^ (row & 31))] = f32x4{acc[b][r][4 * i], acc[b][r][4 * i + 1], acc[b][r][4 * i + 2], acc[b][r][4 * i + 3]};
            }
    __syncthreads();
    const int64_t item = row_head * run.parts.all + run.part0 + range;
    for (int i = threadIdx.x; i < M * UNITS; i += WAVES * 64) {
        const int row = i / UNITS, unit = i % UNITS;
        if (row0 + row < rows) ((f32x4*)(run.parts.acc + (item + (int64_t)row * run.parts.all) * DC))[unit] = ((const f32x4*)lds)[row * UNITS + (unit ^ (row & 31))];
    }
    if (threadIdx.x < M && row0 + (int)threadIdx.x < rows)
        run.parts.ml[item + (int64_t)threadIdx.x * run.parts.all] = make_float2(fmaxf(sm_ref[0][threadIdx.x], sm_ref[1][threadIdx.x]), sm_sum[0][threadIdx.x] + sm_sum[1][threadIdx.x]);
}

int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

// Tiles of 32 rows of a workgroup that has `rows` of them to share.
int wide(int64_t rows) { return rows <= 32 ? 1 : 2; }

// When `n` workgroups of length `l` and then `m` shorter ones of length `k` end that have `places`: those that the last round of the
// long ones leaves free are filled first.
float ends(int64_t n, float l, int64_t m, float k, int64_t places) {
    if (l < k) return ends(m, k, n, l, places);
    const int64_t rounds = (n + places - 1) / places, free = rounds * places - n, fit = free * (int64_t)(l / k), left = m > fit ? m - fit : 0;
    return (float)rounds * l + (float)((left + places - 1) / places) * k;
}

// Ranges of slots of the sequences and of the prefix.
struct Split {
    int own_per, own_ranges, pre_per, pre_ranges;
};

// As many ranges as take least, in slots of one workgroup alone: a workgroup takes its range and 150 slots for its start and its end, a third
// more where two share a compute unit; a part costs finish_kernel 16 where one wavefront adds a row's, 2 where eight do.  Whole calls with every
// sequence as long as its bound: 48 of 8000 slots, 128 heads, in three ranges (288 workgroups for 256 compute units) 329 us, in eight 262; of 30000, 8
// heads, in 11 (528 for 512 places) 365, in ten 275; 5 of 30000 in 103 83, in 43 68; 1 of 701 in three ranges 20 us of attention, in eleven 12.5.
// With a prefix in the same launch the two share the places: 64 sequences of 1 to 501 slots and a prefix of 4096, 32 heads, in launches of their own 42 and
// 17 us of attention, together 54 (49 since); 12 of 27 to 81 and 3967 whole calls of 61 and 51 us.
Split split(int64_t own, int64_t own_groups, int64_t pre, int64_t pre_groups, int mt, bool few) {
    const auto cut = [](int64_t most, int64_t n) { return ((most + n - 1) / n + 63) / 64 * 64; };
    const auto limit = [](int64_t most, int64_t n) { return min((most + 63) / 64, n); };
    const float part = few ? 2.f : 16.f;
    float least = 0.f;
    Split best{};
    for (int64_t a = 1; a <= max(limit(own, pre > 0 ? 32 : 256), (int64_t)1); ++a) {
        const int64_t p = own > 0 ? cut(own, a) : 64;
        if (own > 0 && (own + p - 1) / p != a) continue;
        if (a > 1 && part * (float)a >= least) break;
        for (int64_t b = pre > 0 ? 1 : 0; b <= limit(pre, own > 0 ? 64 : 256); ++b) {
            const int64_t r = b > 0 ? cut(pre, b) : 64;
            if (b > 0 && (pre + r - 1) / r != b) continue;
            const float parts = part * (float)(a + b);
            if (b > 1 && parts >= least) break;
            const int64_t wgs = own_groups * a + pre_groups * b;
            const int64_t places = mt == 2 || wgs <= 256 ? 256 : 512;
            float cost = (places == 512 ? 1.33f : 1.f) * ends(pre_groups * b, (float)r + 150.f, own_groups * a, (float)p + 150.f, places);
            cost += parts;
            if (best.own_ranges == 0 || cost < least) {
                least = cost;
                best = Split{(int)p, (int)a, (int)r, (int)b};
            }
        }
    }
    return best;
}

// How a step is run, from its sizes and bounds.
struct Plan {
    int own_mt, own_tiles, pre_mt, pre_tiles;  // 32-row tiles of a workgroup, workgroups' tiles: of a sequence, of all rows over the prefix
    int own_ranges, pre_ranges;
    Parts parts;
    int64_t own_groups, pre_groups;
    int64_t o_ml, o_a, bytes;
};

Plan plan(const Cache& c, const Step& s, const Heads& h) {
    Plan p{};
    if (s.n_rows == 0) return p;
    const int64_t most = min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len);
    const int64_t rows = (int64_t)s.max_new * h.n, all = (int64_t)s.n_rows * h.n;
    const bool few = finish_few(h, s.n_rows);
    p.own_mt = p.pre_mt = wide(rows);
    if (c.prefix_len > 0) {
        p.pre_mt = wide(all);
        // Few rows over few slots go with the prefix's, though half of a workgroup's rows are empty then: a launch of their own costs 8 us and more.
        if (c.n_seq * most <= 1 << 17) p.own_mt = p.pre_mt;
        p.pre_tiles = (int)((all + p.pre_mt * 32 - 1) / (p.pre_mt * 32));
    }
    p.own_tiles = (int)((rows + p.own_mt * 32 - 1) / (p.own_mt * 32));
    const int64_t groups = (int64_t)c.n_seq * p.own_tiles;
    Split cut;
    if (p.own_mt == p.pre_mt) {
        cut = split(most, groups, c.prefix_len, p.pre_tiles, p.own_mt, few);
    } else {
        cut = split(most, groups, 0, 0, p.own_mt, few);
        const Split pre = split(0, 0, c.prefix_len, p.pre_tiles, p.pre_mt, few);
        cut.pre_per = pre.pre_per;
        cut.pre_ranges = pre.pre_ranges;
    }
    p.parts.per = cut.own_per;
    p.parts.pre_per = cut.pre_per;
    p.own_ranges = p.parts.own = cut.own_ranges;
    p.pre_ranges = cut.pre_ranges;
    p.parts.all = p.own_ranges + p.pre_ranges;
    p.own_groups = groups * p.own_ranges;
    p.pre_groups = (int64_t)p.pre_tiles * p.pre_ranges;
    const int64_t items = all * p.parts.all;
    int64_t o = up256(items * c.latent * 4);
    p.o_ml = o;
    o += up256(items * 8);
    p.o_a = o;
    o += up256(all * (2 * c.latent + c.rope) * 2);
    p.bytes = o;
    return p;
}

template <int DC, int DR>
void launch_run(hipStream_t st, const Cache& c, const Step& s, Both both, int mt, int64_t pre_groups, int64_t own_groups) {
    const dim3 grid((unsigned)(pre_groups + own_groups));
    both.before = (int)pre_groups;
    if (mt == 2) {
        hipLaunchKernelGGL((absorbed_kernel<DC, DR, 2, false>), grid, dim3(512), 0, st, c, s, both);
        return;
    }
    // Caches beyond the last-level cache of 256 MiB, read once by every call, are read past it: 512 sequences of 513 slots (302 MB) 74 us with ordinary
    // copies, 66 so.
    const int64_t bytes = (int64_t)c.n_seq * min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len) * (DC + DR) * 2;
    if (own_groups > 0 && both.own.row_tiles == 1 && bytes > (int64_t)256 << 20) hipLaunchKernelGGL((absorbed_kernel<DC, DR, 1, true>), grid, dim3(256), 0, st, c, s, both);
    else hipLaunchKernelGGL((absorbed_kernel<DC, DR, 1, false>), grid, dim3(256), 0, st, c, s, both);
}

template <int DC, int DR>
void launch_sizes(hipStream_t st, const Cache& c, const Step& s, const Plan& p, const Both& both) {
    if (p.own_mt == p.pre_mt) {
        launch_run<DC, DR>(st, c, s, both, p.own_mt, p.pre_groups, p.own_groups);
    } else {
        launch_run<DC, DR>(st, c, s, both, p.pre_mt, p.pre_groups, 0);
        launch_run<DC, DR>(st, c, s, both, p.own_mt, 0, p.own_groups);
    }
}

}  // namespace

bool absorbed_fits(const Cache& c, const Step& s, const Heads& h) {
    const Plan p = plan(c, s, h);
    const bool attention = p.own_mt == p.pre_mt ? launchable(p.own_groups + p.pre_groups, 256 * p.own_mt)
                                                : launchable(p.own_groups, 256 * p.own_mt) && launchable(p.pre_groups, 256 * p.pre_mt);
    return attention && absorb_fits(c, h, s.n_rows) && finish_fits(h, s.n_rows);
}

int64_t absorbed_workspace(const Cache& c, const Step& s, const Heads& h) { return plan(c, s, h).bytes; }

void launch_absorbed(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const Attend& a) {
    Plan p = plan(c, s, h);
    p.parts.acc = (float*)a.ws;
    p.parts.ml = (float2*)(a.ws + p.o_ml);
    uint16_t* rows = (uint16_t*)(a.ws + p.o_a);
    launch_absorb(st, c, h, a.q, s.n_rows, rows);
    Run run{};
    run.H = h.n;
    run.qscale = a.qscale;
    run.a = rows;
    run.parts = p.parts;
    Both both{run, run, 0};
    both.pre.row_tiles = p.pre_tiles;
    both.pre.per = p.parts.pre_per;
    both.pre.ranges = max(p.pre_ranges, 1);
    both.pre.part0 = p.parts.own;
    both.own.row_tiles = p.own_tiles;
    both.own.per = p.parts.per;
    both.own.ranges = p.own_ranges;
    both.own.packed = p.own_ranges > 1 && c.n_seq <= 256;
    if (c.latent == 128 && c.rope == 32) launch_sizes<128, 32>(st, c, s, p, both);
    if (c.latent == 128 && c.rope == 64) launch_sizes<128, 64>(st, c, s, p, both);
    if (c.latent == 256 && c.rope == 32) launch_sizes<256, 32>(st, c, s, p, both);
    if (c.latent == 256 && c.rope == 64) launch_sizes<256, 64>(st, c, s, p, both);
    if (c.latent == 512 && c.rope == 32) launch_sizes<512, 32>(st, c, s, p, both);
    if (c.latent == 512 && c.rope == 64) launch_sizes<512, 64>(st, c, s, p, both);
    launch_finish(st, c, s, h, a.out, p.parts);
}

}  // namespace klat
