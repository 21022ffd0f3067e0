// Attention over the latent cache in its absorbed form: all heads of all new tokens of a sequence are rows of one matrix
// A [rows, latent + rope], and z = A C^T, u = softmax(z) C[:, :latent] with the cache's rows C as keys and as values.
//
// A row of C has 1152 bytes (512 + 64) and takes part in 2 * (2 * 512 + 64) operations per row of A: bound by the bytes of
// the cache up to about 60 rows of A, by the matrix cores and the LDS that feeds them beyond.
#include "latent_device.h"

namespace klat {
namespace {

// How C lies in LDS: tiles of 32 slots, cut into groups of 64 elements (128 bytes), a group being 32 slots x 8 units of 16 bytes.
// Unit u of slot r is at place u ^ twist(r): then neither the reads by slots (32 lanes, one unit each; keys) nor the transposed ones
// (8 slots, 64 bytes each; values) meet in a bank.  Rows whose width is half a group more than whole groups fill the last one twice.
template <int DC, int DR>
struct Tile {
    static constexpr int kWidth = DC + DR, kGroups = (kWidth + 63) / 64, kBytes = kGroups * 4096;
    static constexpr bool kHalf = kWidth % 64 != 0;
};
__device__ __forceinline__ int twist(int slot) { return (slot >> 1 & 1) << 2 | (slot >> 2 & 3); }

struct Run {  // one launch
    int H, row_tiles;  // tiles of MW * 32 rows of a sequence (of the prefix: of all)
    int per, ranges;   // slots of a range, ranges at most
    int part0;         // where the launch's parts are among a row's
    float qscale;
    const uint16_t* a;  // [row, head, latent + rope]
    Parts parts;
};

// A workgroup of four wavefronts takes MW * 32 rows of A and a range of slots: MW wavefronts side by side with 32 rows each
// (in registers), and 4 / MW such teams that take the tiles of the range in turn and add up at the end.  Scores are formed
// transposed, z^T = C A^T, so that a lane has one row of A: its softmax needs no exchange but one between two lanes, and the weights
// are the second operand of u^T = C^T w as they stand.  LDS holds four tiles; a team's tiles come in a ring of MW, copied without
// registers.  With MW = 1 nothing is shared: every wavefront copies, waits and computes by itself, the other three cover its waits.
template <int DC, int DR, int MW, bool PREFIX>
__global__ __launch_bounds__(256, 1) void absorbed_kernel(Cache c, Step s, Run run) {
    typedef Tile<DC, DR> T;
    constexpr int KW = 4 / MW, STEPS = T::kWidth / 16, BLOCKS = DC / 32;
    constexpr int AT_ONCE = BLOCKS > 8 ? 8 : 4;          // blocks of 32 elements that meet in LDS at a time
    constexpr int RING = 4 * T::kBytes, SUMS = AT_ONCE * 4 * 4096;
    __shared__ __attribute__((aligned(16))) uint8_t lds[RING > SUMS || KW == 1 ? RING : SUMS];
    __shared__ float2 sm_ml[4][32];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5;
    const int mw = wave % MW, team = wave / MW;
    int seq = 0, rest = blockIdx.x;
    if (!PREFIX) {
        seq = blockIdx.x % c.n_seq;
        rest = blockIdx.x / c.n_seq;
    }
    const int range = rest % run.ranges, tile = run.row_tiles - 1 - rest / run.ranges;  // those that see the most slots first
    Seq q;
    if (PREFIX) q = Seq{0, s.n_rows, 0};
    else q = kkv8::sequence(c.max_len, s, seq);
    const int rows = q.n_new * run.H, row0 = tile * MW * 32;
    if (row0 >= rows) return;
    const int last_row = min(row0 + MW * 32, rows) - 1;
    const int first = range * run.per;
    const int sees = PREFIX ? c.prefix_len : q.cached + last_row / run.H + 1;  // slots that the last row sees
    const int end = min(first + run.per, sees);
    if (first >= end) return;
    const uint16_t* C = PREFIX ? c.prefix : c.rows + (int64_t)seq * c.max_len * T::kWidth;
    const int r = row0 + mw * 32 + col, mine = min(r, rows - 1);
    const int limit = PREFIX ? c.prefix_len : q.cached + mine / run.H + 1;  // slots that the lane's row sees
    const int wave_least = PREFIX ? c.prefix_len : q.cached + min(row0 + mw * 32, rows - 1) / run.H + 1;  // that all its rows see
    const int64_t row_head = (int64_t)q.row0 * run.H;

    // copies: a wavefront brings 8 slots x 8 units at a time, of 4 / MW of the tile's four quarters
    const uint32_t lds_at = lds_address(lds);
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_at + team * MW * T::kBytes);
    const int in8 = lane >> 3;
    uint32_t unit_at[2];  // byte of the row that the lane brings, in even and odd quarters
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) unit_at[odd] = (uint32_t)(((lane & 7) ^ twist(odd * 8 + in8)) * 16);
    auto copy = [&](int buf, int j0) {
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            const int quarter = mw * KW + i;
            const uint32_t slot = (uint32_t)min(j0 + quarter * 8 + in8, end - 1);  // past the end the last one again
            const uint32_t at = slot * (T::kWidth * 2) + (quarter & 1 ? unit_at[1] : unit_at[0]);
            const uint32_t to = ring_at + buf * T::kBytes + quarter * 1024;
#pragma unroll
            for (int g = 0; g < T::kGroups; ++g) {
                if (T::kHalf && g == T::kGroups - 1) {  // the row ends within the group
                    const uint32_t u = (quarter & 1 ? unit_at[1] : unit_at[0]) & 63;
                    copy_to_lds((const uint8_t*)C + g * 128, slot * (T::kWidth * 2) + u, __builtin_amdgcn_readfirstlane(to + g * 4096));
                } else {
                    copy_to_lds((const uint8_t*)C + g * 128, at, __builtin_amdgcn_readfirstlane(to + g * 4096));
                }
            }
        }
    };
    constexpr int COPIES = KW * T::kGroups;  // of a wavefront for a tile

    u32x4 af[STEPS];
    {
        const uint16_t* p = run.a + (row_head + mine) * T::kWidth + grp * 8;
#pragma unroll
        for (int f = 0; f < STEPS; ++f) af[f] = *(const u32x4*)(p + f * 16);
#pragma unroll
        for (int f = 0; f < STEPS; ++f) asm volatile("" : "+v"(af[f]));  // waited for here, not in the loop
    }
    f32x16 acc[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
    float ref = kEmpty, sum = 0.f;

    // the lane's places in a tile: units 2 * (f % 4) + grp of its slot; four slots of 16 elements for the transposed reads
    uint32_t key_at[4], value_at[2][2];
#pragma unroll
    for (int f = 0; f < 4; ++f) key_at[f] = (uint32_t)(col * 128 + ((2 * f + grp) ^ twist(col)) * 16);
#pragma unroll
    for (int odd = 0; odd < 2; ++odd)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int slot = 8 * j + 4 * grp + ((lane & 15) >> 2), unit = odd * 4 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
            value_at[odd][j] = (uint32_t)(slot * 128 + (unit ^ twist(slot)) * 16 + (lane & 1) * 8);
        }

    // The sums stay in the accumulation registers: 256 of the lane's 512 with 512 latents, the rows of A 144 of the others.
    auto pin = [&](int b) { asm volatile("" : "+a"(acc[b])); };
    auto compute = [&](uint32_t at, int j0) {
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
        for (int f = 0; f < STEPS; ++f) z = mfma32(read_lds(at + key_at[f & 3] + (f >> 2) * 4096), af[f], z);
        if (j0 + 32 > wave_least || j0 + 32 > end) {
            const int within = min(limit, end) - j0 - 4 * grp;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (row_of(i, 0) >= within) z[i] = -__builtin_inff();
        }
        float top = z[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, z[i]);
        top *= run.qscale;
        if (__any(top > ref + kRise)) {
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float now = top > ref + kRise ? reference_of(top) : ref;
            const float f = __builtin_amdgcn_exp2f(ref - now);
            ref = now;
            sum *= f;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                pin(b);
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[b][i] *= f;
                pin(b);
            }
        }
        exponents(ref, kAbove, run.qscale, [&](auto&& of) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = of(z[i]);
        });
        u32x4 w[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(z[t * 8 + i]);
                sum += p[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) w[t][i] = pack_bf16(p[2 * i], p[2 * i + 1]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const uint32_t v = at + (b >> 1) * 4096 + t * 2048;
                acc[b] = mfma32(join(read_transposed(v + value_at[b & 1][0]), read_transposed(v + value_at[b & 1][1])), w[t], acc[b]);
            }
    };
    // A latent that is not finite, in a slot that some row of the workgroup does not see, would reach that row as 0 times it.
    // In tiles where that can be, such slots give up their latents and get NaN in the part that only the scores read:
    // the rows that see them become NaN, as they have to, and no others.  Done by the wavefront that brought the slots.
    const int all_see = PREFIX ? c.prefix_len : q.cached + row0 / run.H + 1;
    auto mend = [&](uint32_t at) {
        for (int i = 0; i < KW * 8; ++i) {
            const int slot = mw * KW * 8 + i;
            const uint32_t to = at + (lane >> 3) * 4096 + slot * 128 + ((lane & 7) ^ twist(slot)) * 16;
            bool bad = false;
            if (lane * 8 < DC) {
                const u32x4 x = read_lds(to);
#pragma unroll
                for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
            }
            if (__any(bad)) {
                if (lane * 8 < DC) write_lds(to, u32x4{0u, 0u, 0u, 0u});
                if (lane == 0)
                    write_lds(at + (DC / 64) * 4096 + slot * 128 + twist(slot) * 16, u32x4{0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu});
            }
        }
    };

    const int tiles = (end - first + 31) / 32;
    if constexpr (MW == 1) {
        for (int t = team; t < tiles; t += KW) {
            const int j0 = first + t * 32;
            copy(0, j0);
            wait_copies<0>();
            if (!PREFIX && all_see < sees && j0 + 32 > all_see) mend(ring_at);
            compute(ring_at, j0);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile has been read
        }
    } else {
        const int steps = (tiles + KW - 1) / KW;  // the same for both teams, which wait for one another
        auto slot_at = [&](int step) { return first + min(step * KW + team, tiles - 1) * 32; };
#pragma unroll
        for (int i = 0; i < MW - 1; ++i)
            if (i < steps) copy(i, slot_at(i));
        int buf = 0;
        for (int t = 0; t < steps; ++t) {
            if (t + MW - 2 < steps) wait_copies<(MW - 2) * COPIES>();  // all but the youngest MW - 2 tiles
            else wait_copies<0>();
            __syncthreads();  // the tile is there, and nobody reads the one before it any more
            if (t + MW - 1 < steps) copy(buf == 0 ? MW - 1 : buf - 1, slot_at(t + MW - 1));
            // Every wavefront takes every tile, though some see nothing of it: a branch around the products would have the sums
            // copied between registers.  A team's tile past the last one is the last one again, and its slots count as hidden.
            if (!PREFIX && all_see < sees && first + (t + 1) * KW * 32 > all_see) {  // the same for both teams
                mend(ring_at + buf * T::kBytes);
                __syncthreads();
            }
            compute(ring_at + buf * T::kBytes, first + (t * KW + team) * 32);
            buf = buf == MW - 1 ? 0 : buf + 1;
        }
    }
    sum += __shfl_xor(sum, 32, 64);

    const int64_t item = (row_head + r) * run.parts.all + run.part0 + range;
    float* to = run.parts.acc + item * DC;
    if constexpr (KW == 1) {
        if (r < rows) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(f32x4*)(to + b * 32 + row_of(4 * i, grp)) = f32x4{acc[b][4 * i], acc[b][4 * i + 1], acc[b][4 * i + 2], acc[b][4 * i + 3]};
            if (grp == 0) run.parts.ml[item] = make_float2(ref, sum);
        }
    } else {
        // the teams' sums meet in LDS, AT_ONCE blocks at a time, each team adding its share of them
        if (grp == 0) sm_ml[wave][col] = make_float2(ref, sum);
        __syncthreads();  // the tiles are done with, too
        float most = kEmpty, all = 0.f;
#pragma unroll
        for (int k = 0; k < KW; ++k) most = fmaxf(most, sm_ml[k * MW + mw][col].x);
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            const float2 ml = sm_ml[k * MW + mw][col];
            all = __builtin_fmaf(ml.y, __builtin_amdgcn_exp2f(ml.x - most), all);
        }
        const float f = __builtin_amdgcn_exp2f(ref - most);
        constexpr int SHARE = AT_ONCE / KW;
        f32x4* sums = (f32x4*)lds;
#pragma unroll
        for (int b0 = 0; b0 < BLOCKS; b0 += AT_ONCE) {
            if (b0 > 0) __syncthreads();
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sums[((wave * AT_ONCE + b) * 4 + i) * 64 + lane] =
                        f32x4{acc[b0 + b][4 * i] * f, acc[b0 + b][4 * i + 1] * f, acc[b0 + b][4 * i + 2] * f, acc[b0 + b][4 * i + 3] * f};
            __syncthreads();
#pragma unroll
            for (int b = 0; b < SHARE; ++b) {
                const int block = team * SHARE + b;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 x = sums[((mw * AT_ONCE + block) * 4 + i) * 64 + lane];
#pragma unroll
                    for (int k = 1; k < KW; ++k) x += sums[(((k * MW + mw) * AT_ONCE + block) * 4 + i) * 64 + lane];
                    if (r < rows) *(f32x4*)(to + (b0 + block) * 32 + row_of(4 * i, grp)) = x;
                }
            }
        }
        if (r < rows && team == 0 && grp == 0) run.parts.ml[item] = make_float2(most, all);
    }
}

int64_t up256(int64_t v) { return (v + 255) & ~(int64_t)255; }

// Wavefronts side by side over `rows` rows.
int wide(int64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// Ranges of `most` slots for `groups` workgroups each.
void split(int64_t most, int64_t groups, int* per, int* ranges) {
    int64_t n = groups > 0 ? (512 + groups - 1) / groups : 1;
    const int64_t least = 256;
    if (n > (most + least - 1) / least) n = (most + least - 1) / least;
    if (n < 1) n = 1;
    int64_t p = ((most + n - 1) / n + 127) / 128 * 128;
    if (p < 128) p = 128;
    *per = (int)p;
    *ranges = (int)(most > p ? (most + p - 1) / p : 1);
}

}  // namespace

// How a step is run, from its sizes and bounds.
struct Plan {
    int own_mw, own_tiles, pre_mw, pre_tiles;  // wavefronts side by side, row tiles: of a sequence, of all rows over the prefix
    int own_ranges, pre_ranges;
    Parts parts;
    int64_t own_groups, pre_groups;
    int64_t o_ml, o_a, bytes;
};

namespace {

Plan plan(const Cache& c, const Step& s, const Heads& h) {
    Plan p{};
    if (s.n_rows == 0) return p;
    const int64_t most = min((int64_t)s.max_cached + s.max_new, (int64_t)c.max_len);
    const int64_t rows = (int64_t)s.max_new * h.n, all = (int64_t)s.n_rows * h.n;
    p.own_mw = wide(rows);
    p.own_tiles = (int)((rows + p.own_mw * 32 - 1) / (p.own_mw * 32));
    split(most, (int64_t)c.n_seq * p.own_tiles, &p.parts.per, &p.own_ranges);
    p.own_groups = (int64_t)c.n_seq * p.own_tiles * p.own_ranges;
    p.parts.own = p.parts.all = p.own_ranges;
    p.parts.pre_per = 1;
    if (c.prefix_len > 0) {
        p.pre_mw = wide(all);
        p.pre_tiles = (int)((all + p.pre_mw * 32 - 1) / (p.pre_mw * 32));
        split(c.prefix_len, p.pre_tiles, &p.parts.pre_per, &p.pre_ranges);
        p.pre_groups = (int64_t)p.pre_tiles * p.pre_ranges;
        p.parts.all += p.pre_ranges;
    }
    const int64_t items = all * p.parts.all;
    int64_t o = up256(items * c.latent * 4);
    p.o_ml = o;
    o += up256(items * 8);
    p.o_a = o;
    o += up256(all * (c.latent + c.rope) * 2);
    p.bytes = o;
    return p;
}

template <int DC, int DR, bool PREFIX>
void launch_run(hipStream_t st, const Cache& c, const Step& s, const Run& run, int mw, int64_t groups) {
    const dim3 grid((unsigned)groups), block(256);
    if (mw == 1) hipLaunchKernelGGL((absorbed_kernel<DC, DR, 1, PREFIX>), grid, block, 0, st, c, s, run);
    if (mw == 2) hipLaunchKernelGGL((absorbed_kernel<DC, DR, 2, PREFIX>), grid, block, 0, st, c, s, run);
    if (mw == 4) hipLaunchKernelGGL((absorbed_kernel<DC, DR, 4, PREFIX>), grid, block, 0, st, c, s, run);
}

template <int DC, int DR>
void launch_sizes(hipStream_t st, const Cache& c, const Step& s, const Plan& p, Run run) {
    if (p.pre_groups > 0) {
        run.row_tiles = p.pre_tiles;
        run.per = p.parts.pre_per;
        run.ranges = p.pre_ranges;
        run.part0 = p.parts.own;
        launch_run<DC, DR, true>(st, c, s, run, p.pre_mw, p.pre_groups);
    }
    run.row_tiles = p.own_tiles;
    run.per = p.parts.per;
    run.ranges = p.own_ranges;
    run.part0 = 0;
    launch_run<DC, DR, false>(st, c, s, run, p.own_mw, p.own_groups);
}

}  // namespace

int choose_form(const Cache&, const Step&, const Heads&, int) { return MOE_LATENT_ABSORBED; }

bool attend_fits(const Cache& c, const Step& s, const Heads& h, int) {
    const Plan p = plan(c, s, h);
    return p.own_groups <= kMostGroups && p.pre_groups <= kMostGroups && absorb_groups(c, h, s.n_rows) <= kMostGroups &&
           finish_groups(h, s.n_rows) <= kMostGroups;
}

int64_t attend_workspace(const Cache& c, const Step& s, const Heads& h, int) { return plan(c, s, h).bytes; }

void launch_attend(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const Attend& a, int) {
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
    if (c.latent == 128 && c.rope == 32) launch_sizes<128, 32>(st, c, s, p, run);
    if (c.latent == 128 && c.rope == 64) launch_sizes<128, 64>(st, c, s, p, run);
    if (c.latent == 256 && c.rope == 32) launch_sizes<256, 32>(st, c, s, p, run);
    if (c.latent == 256 && c.rope == 64) launch_sizes<256, 64>(st, c, s, p, run);
    if (c.latent == 512 && c.rope == 32) launch_sizes<512, 32>(st, c, s, p, run);
    if (c.latent == 512 && c.rope == 64) launch_sizes<512, 64>(st, c, s, p, run);
    launch_finish(st, c, s, h, a.out, p.parts);
}

}  // namespace klat
