// The latent cache: filling it; bringing queries into the latent space and sums out of it (the absorbed form's products around
// the attention itself, which is in k_latent_attn.hip).
#include "latent_device.h"

namespace klat {
namespace {

// One wavefront per row: 8 latents a lane, the mean of squares over the lanes, then one element of the part that turns a lane (its
// partner is read again, from the first-level cache).  Bound by latency (512 rows: 3.7 us), then by
// the rows read and written once (16600 rows of 576: 38 MB in 10.9 us, 3.5 TB/s).
__global__ __launch_bounds__(256) void append_kernel(Cache c, Step s, Append a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + wave_number();
    if (row >= s.n_rows) return;
    Seq q;
    int token;
    const int seq = seq_of_row(c, s, row, &token, &q);
    if (seq < 0) return;
    const uint16_t* x = a.x + (int64_t)row * a.x_row;
    uint16_t* to = c.rows + ((int64_t)seq * c.max_len + q.cached + token) * (c.latent + c.rope);
    const bool mine = lane * 8 < c.latent;
    u32x4 v = {0u, 0u, 0u, 0u}, g = v;
    if (mine) v = *(const u32x4*)(x + lane * 8);
    uint32_t e = 0, partner = 0;
    const int at = lane - a.first, half = a.rot / 2;
    const bool turns = lane < c.rope && at >= 0 && at < a.rot;
    // the element's pair, whether it is the pair's second, where its partner is
    const bool second = a.interleaved ? (at & 1) != 0 : at >= half;
    const int pair = a.interleaved ? at >> 1 : second ? at - half : at;
    const int partner_at = a.interleaved ? at ^ 1 : second ? at - half : at + half;
    if (lane < c.rope) e = x[c.latent + lane];
    if (turns) partner = x[c.latent + a.first + partner_at];
    if (a.norm != nullptr) {
        if (mine) g = *(const u32x4*)(a.norm + lane * 8);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += bf_lo(v[i]) * bf_lo(v[i]) + bf_hi(v[i]) * bf_hi(v[i]);
#pragma unroll
        for (int m = 32; m > 0; m /= 2) sum += __shfl_xor(sum, m, 64);
        const float square = sum / (float)c.latent + a.eps;
        if (square >= 0x1p-80f && sum <= 3.40282347e38f) {
            const float inv = 1.f / sqrtf(square);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pack_bf16(bf_lo(v[i]) * inv * bf_lo(g[i]), bf_hi(v[i]) * inv * bf_hi(g[i]));
        } else {  // squares beyond the range of 32 bits, or below it, from which eps does not keep them
            double all = 0.;
#pragma unroll
            for (int i = 0; i < 4; ++i) all += (double)bf_lo(v[i]) * bf_lo(v[i]) + (double)bf_hi(v[i]) * bf_hi(v[i]);
#pragma unroll
            for (int m = 32; m > 0; m /= 2) all += __shfl_xor(all, m, 64);
            const double inv = 1. / sqrt(all / c.latent + a.eps);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pack_bf16((float)(bf_lo(v[i]) * inv * bf_lo(g[i])), (float)(bf_hi(v[i]) * inv * bf_hi(g[i])));
        }
    }
    if (mine) *(u32x4*)(to + lane * 8) = v;
    if (turns) {
        const int position = (s.next_position != nullptr ? s.next_position[seq] : c.prefix_len + q.cached) + token;
        const float2 cs = krope::turn(a.turns, pair, position);
        const float cosine = cs.x * a.turns.magnitude, sine = cs.y * a.turns.magnitude;
        e = pack_bf16(krope::turned(bf_lo(e), bf_lo(partner), cosine, second ? sine : -sine), 0.f);
    }
    if (lane < c.rope) to[c.latent + lane] = (uint16_t)e;
}

// a[row][head] = w_k[head]^T n in bf16, then the part that carries the position, then what rounding a left over, in bf16, too:
// rows of 2 * latent + rope elements, in the caller's order of rows and heads.  (a counts with 16 bits: rounded to 8 it would move
// the scores, and with them the outputs, by more than the outputs' own rounding: 2.8e-3 over 3000 slots, where that is 1.7e-3.)
//
// A workgroup of WAVES wavefronts per (head, 128 latents, `each` tiles of 32 rows for each of them): its piece of w_k lies in LDS (nope_dim x
// 256 bytes) and is read transposed by the LDS, four latents of four rows at a time, as the first operand: a^T = w_k^T n^T, so that a lane
// has one row and four latents side by side.  The result goes through LDS to leave in pieces of 256 bytes.  Bound by the bytes written (four
// for every latent) where there are many rows, by latency where there are few: then one wavefront a workgroup.
// 512 rows of 32 heads, latents of 512: 42 MB in 15 us; 1 row 4.1 us.
template <int NOPE, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void absorb_kernel(Cache c, Heads h, Rows q, int n_rows, int each, uint16_t* out) {
    __shared__ u32x4 w[NOPE * 16], stage[WAVES][32 * 16];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5;
    const int chunks = c.latent / 128, head = blockIdx.x % h.n, rest = blockIdx.x / h.n, chunk = rest % chunks;
    const int tile0 = rest / chunks * each * WAVES + wave, tiles = (n_rows + 31) / 32, width = 2 * c.latent + c.rope;
    u32x4* o = stage[wave];
    // rows of w_k four at a time; 16-byte units of a row lie at an xor of its number, which spreads the transposed reads over the banks
    const uint16_t* from = h.w_k + head * h.w_k_head + chunk * 128 + (lane >> 4) * c.latent + ((lane & 15) ^ (lane >> 4 & 3) << 2) * 8;
    const uint32_t w_at = lds_address(w);
#pragma unroll
    for (int i = 0; i < NOPE / 4 / WAVES; ++i) {
        const int four = i * WAVES + wave;
        copy_to_lds(from + (int64_t)four * 4 * c.latent, __builtin_amdgcn_readfirstlane(w_at + four * 1024));
    }
    u32x4 n[NOPE / 16];
    const uint16_t* rows = q.p + (int64_t)head * q.head + grp * 8;
    auto load = [&](int tile) {
        const uint16_t* p = rows + (int64_t)min(tile * 32 + col, n_rows - 1) * q.row;
#pragma unroll
        for (int f = 0; f < NOPE / 16; ++f) n[f] = *(const u32x4*)(p + f * 16);
    };
    load(tile0);
    wait_copies<0>();
    __syncthreads();
    // transposed reads: a lane points at row (lane % 16) / 4 of four and four latents, and gets one latent of the four rows
    const int rr = (lane & 15) >> 2;
    const uint32_t at = w_at + (8 * grp + rr) * 256 + (lane & 1) * 8;
    const int unit = (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
    for (int t = 0; t < each; ++t) {
        const int tile = tile0 + t * WAVES;
        if (tile >= tiles) break;
        f32x16 acc[4];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
#pragma unroll
        for (int f = 0; f < NOPE / 16; ++f)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const uint32_t p = at + f * 4096 + ((b * 4 + unit) ^ rr << 2) * 16;
                acc[b] = mfma32(join(read_transposed(p), read_transposed(p + 1024)), n[f], acc[b]);
            }
        const int row0 = tile * 32;
        if (t + 1 < each) load(tile + WAVES);
        uint16_t* to = out + ((int64_t)row0 * h.n + head) * width + chunk * 128 + (lane & 15) * 8;
#pragma unroll
        for (int second = 0; second < 2; ++second) {  // what is left over goes where the values themselves went before: only this wavefront's
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    u32x2 x;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int e = 4 * i + 2 * j;
                        x[j] = pack_bf16(acc[b][e], acc[b][e + 1]);
                        acc[b][e] -= bf_lo(x[j]);
                        acc[b][e + 1] -= bf_hi(x[j]);
                    }
                    ((u32x2*)&o[col * 16 + ((b * 4 + i) ^ (col & 15))])[grp] = x;
                }
            wave_sync();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int in = i * 4 + (lane >> 4);
                if (row0 + in < n_rows)
                    *(u32x4*)(to + (int64_t)in * h.n * width + second * (c.latent + c.rope)) = o[in * 16 + ((lane & 15) ^ (in & 15))];
            }
            wave_sync();
        }
        if (chunk == 0) {
            const int units = c.rope / 8;
            for (int i = lane; i < 32 * units; i += 64) {
                const int row = row0 + i / units, u = i % units;
                if (row < n_rows)
                    *(u32x4*)(out + ((int64_t)row * h.n + head) * width + c.latent + u * 8) =
                        *(const u32x4*)(q.p + (int64_t)row * q.row + (int64_t)head * q.head + NOPE + u * 8);
            }
        }
    }
}

// o = w_v u / sum for up to 32 rows of one head: the parts of a row's sums are brought to the largest reference and added (a wavefront
// per row; FEW: one row, which all eight share), the result goes into LDS as two bf16 (value and what rounding it left over) in the
// order of the matrix instructions, and the wavefronts take 32 of the value's elements and a share of the latents each, which then meet
// in LDS.  w_v is asked for before the parts are read.  Bound by latency where there are few rows (1 row of 32 heads in
// eleven parts 8 us), then by the parts' bytes and w_v's from L2 (512 rows of 32 heads in one part, 34 MB and 67 from L2: 19 us).
template <int DC, int DV, bool FEW>
__global__ __launch_bounds__(512, FEW ? 2 : 4) void finish_kernel(Cache c, Step s, Heads h, RowsOut out, Parts parts, int span) {
    constexpr int BLOCKS = DV / 32, SHARES = 8 / BLOCKS, F = DC / 16 / SHARES, Q = DC / 4 > 64 ? DC / 256 : 1;  // pieces of four elements that a lane has
    __shared__ u32x4 u[2][DC / 8 * 32];
    __shared__ int own_parts[32];                    // of a row's slots; 0: no row
    __shared__ f32x4 shared_sums[FEW ? 8 : 1][FEW ? (DC / 4 < 64 ? 64 : DC / 4) : 1];
    constexpr bool FITS = sizeof u >= 8 * 4096 + 32 * DV * 2;  // the shares of the product and the rows that leave
    __shared__ f32x4 shares_apart[FITS ? 1 : 8 * 256 + 32 * DV / 8];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5;
    const int head = blockIdx.x % h.n, row0 = blockIdx.x / h.n * span, rows = min(span, s.n_rows - row0);
    if (threadIdx.x < 32) {
        int own = 0;
        if ((int)threadIdx.x < rows) {
            Seq q;
            int token;
            if (lane_seq_of_row(c, s, row0 + threadIdx.x, &token, &q) >= 0) own = (q.cached + token + parts.per) / parts.per;
        }
        own_parts[threadIdx.x] = own;
    }
    const int block = wave % BLOCKS, share = wave / BLOCKS;
    u32x4 wf[F];
    {
        const uint16_t* p = h.w_v + head * h.w_v_head + (int64_t)(block * 32 + col) * DC + share * F * 16 + grp * 8;
#pragma unroll
        for (int f = 0; f < F; ++f) wf[f] = *(const u32x4*)(p + f * 16);
    }
    __syncthreads();
    // the wavefront's rows two by two, so that their reads are on the way together
    constexpr int R = FEW ? 1 : 2;
    for (int i0 = 0; i0 < (FEW ? 1 : (span + 8 * R - 1) / (8 * R)); ++i0) {
        const auto row_of_wave = [&](int r) { return FEW ? 0 : wave + 8 * (R * i0 + r); };
        int own[R], n[R], most = 0;
        int64_t item[R];
        float ref[R], sum[R];
        f32x4 x[R][Q];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            own[r] = __builtin_amdgcn_readfirstlane(own_parts[row_of_wave(r)]);
            n[r] = own[r] > 0 ? own[r] + parts.all - parts.own : 0;
            most = max(most, n[r]);
            item[r] = ((int64_t)(row0 + row_of_wave(r)) * h.n + head) * parts.all;
            ref[r] = kEmpty;
            sum[r] = 0.f;
#pragma unroll
            for (int j = 0; j < Q; ++j) x[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const auto at = [&](int r, int k) { return item[r] + (k < own[r] ? k : parts.own + k - own[r]); };
        for (int k = lane; k < (most + 63 & ~63); k += 64)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (k < n[r]) ref[r] = fmaxf(ref[r], parts.ml[at(r, k)].x);
#pragma unroll
        for (int m = 32; m > 0; m /= 2)
#pragma unroll
            for (int r = 0; r < R; ++r) ref[r] = fmaxf(ref[r], __shfl_xor(ref[r], m, 64));
        for (int k0 = 0; k0 < most; k0 += 64) {
            float f[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                f[r] = 0.f;
                if (k0 + lane < n[r]) {
                    const float2 ml = parts.ml[at(r, k0 + lane)];
                    f[r] = __builtin_amdgcn_exp2f(ml.x - ref[r]);
                    sum[r] = __builtin_fmaf(ml.y, f[r], sum[r]);
                }
            }
            for (int k = FEW ? wave : 0; k < min(64, most - k0); k += FEW ? 8 : 1) {
                f32x4 y[R][Q];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    // past a row's last part the last one again, which then counts 0 times
                    const f32x4* p = (const f32x4*)(parts.acc + at(r, max(0, min(k0 + k, n[r] - 1))) * DC) + lane;
#pragma unroll
                    for (int j = 0; j < Q; ++j) y[r][j] = n[r] > 0 && (DC / 4 >= 64 || lane < DC / 4) ? p[j * 64] : f32x4{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (k0 + k >= n[r]) continue;
                    const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f[r]), k));
#pragma unroll
                    for (int j = 0; j < Q; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[r][j][e] = __builtin_fmaf(y[r][j][e], by, x[r][j][e]);
                }
            }
        }
#pragma unroll
        for (int m = 32; m > 0; m /= 2)
#pragma unroll
            for (int r = 0; r < R; ++r) sum[r] += __shfl_xor(sum[r], m, 64);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float inv = n[r] > 0 ? 1.f / sum[r] : 0.f;
#pragma unroll
            for (int j = 0; j < Q; ++j) x[r][j] *= inv;
        }
        if constexpr (FEW) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < Q; ++j) shared_sums[wave][j * 64 + lane] = x[0][j];
            __syncthreads();
            if (wave != 0) continue;
#pragma unroll
            for (int j = 0; j < Q; ++j)
#pragma unroll
                for (int w = 1; w < 8; ++w) x[0][j] += shared_sums[w][j * 64 + lane];
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                const int piece = j * 64 + lane, unit = piece >> 1;  // of four elements, of eight
                if (piece * 4 >= DC) continue;
                u32x2 hi, lo;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    hi[e] = pack_bf16(x[r][j][2 * e], x[r][j][2 * e + 1]);
                    lo[e] = pack_bf16(x[r][j][2 * e] - bf_lo(hi[e]), x[r][j][2 * e + 1] - bf_hi(hi[e]));
                }
                ((u32x2*)&u[0][unit * 32 + (row_of_wave(r) ^ (unit & 31))])[piece & 1] = hi;
                ((u32x2*)&u[1][unit * 32 + (row_of_wave(r) ^ (unit & 31))])[piece & 1] = lo;
            }
    }
    __syncthreads();
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int unit = 2 * (share * F + f) + grp;
        acc = mfma32(wf[f], u[0][unit * 32 + (col ^ (unit & 31))], acc);
        acc = mfma32(wf[f], u[1][unit * 32 + (col ^ (unit & 31))], acc);
    }
    f32x4* shares = FITS ? (f32x4*)&u[0][0] : shares_apart;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) shares[(wave * 4 + i) * 64 + lane] = f32x4{acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
    __syncthreads();
    // four elements of a row a piece: wavefront w takes pieces w, w + 8 ... of BLOCKS * 4; through LDS, so that a row leaves in one piece
    u32x2* rows_out = (u32x2*)(shares + 8 * 256);
#pragma unroll
    for (int n = 0; n < (BLOCKS * 4 + 7) / 8; ++n) {
        const int piece = n * 8 + wave;
        if (piece >= BLOCKS * 4) break;
        f32x4 y = shares[piece * 64 + lane];  // share 0 of block piece / 4
#pragma unroll
        for (int k = 1; k < SHARES; ++k) y += shares[(k * BLOCKS * 4 + piece) * 64 + lane];
        u32x2 x;
        x.x = pack_bf16(y[0], y[1]);
        x.y = pack_bf16(y[2], y[3]);
        rows_out[(col * (DV / 8) + (piece ^ (col & (DV / 8 - 1)))) * 2 + grp] = x;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * (DV / 8); i += 512) {
        const int row = i / (DV / 8), piece = i % (DV / 8);
        if (own_parts[row] != 0)
            *(u32x4*)(out.p + (int64_t)(row0 + row) * out.row + (int64_t)head * out.head + piece * 8) = ((const u32x4*)rows_out)[row * (DV / 8) + (piece ^ (row & (DV / 8 - 1)))];
    }
}

}  // namespace

void launch_append(hipStream_t st, const Cache& c, const Step& s, const Append& a) {
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)((s.n_rows + 3) / 4)), dim3(256), 0, st, c, s, a);
}

// Wavefronts of a workgroup, and tiles of 32 rows of each: about 2048 wavefronts, two for each SIMD.  With nope 128 (198 registers and 64 for the
// products) a SIMD holds one at a time, otherwise both.
static int absorb_waves(int n_rows) { return n_rows > 64 ? 4 : 1; }
static int absorb_each(const Cache& c, const Heads& h, int n_rows) {
    const int64_t all = (int64_t)h.n * (c.latent / 128) * ((n_rows + 31) / 32);
    return all > 2048 ? (int)((all + 2047) / 2048) : 1;
}

static int64_t absorb_groups(const Cache& c, const Heads& h, int n_rows) {
    const int64_t tiles = (n_rows + 31) / 32, of = absorb_each(c, h, n_rows) * absorb_waves(n_rows);
    return h.n * (c.latent / 128) * ((tiles + of - 1) / of);
}

bool absorb_fits(const Cache& c, const Heads& h, int n_rows) { return launchable(absorb_groups(c, h, n_rows), 64 * absorb_waves(n_rows)); }

template <int NOPE>
static void launch_absorb_nope(hipStream_t st, const Cache& c, const Heads& h, const Rows& q, int n_rows, uint16_t* out) {
    const dim3 grid((unsigned)absorb_groups(c, h, n_rows));
    const int each = absorb_each(c, h, n_rows);
    if (absorb_waves(n_rows) == 4) hipLaunchKernelGGL((absorb_kernel<NOPE, 4>), grid, dim3(256), 0, st, c, h, q, n_rows, each, out);
    else hipLaunchKernelGGL((absorb_kernel<NOPE, 1>), grid, dim3(64), 0, st, c, h, q, n_rows, each, out);
}

void launch_absorb(hipStream_t st, const Cache& c, const Heads& h, const Rows& q, int n_rows, uint16_t* out) {
    if (h.nope == 32) launch_absorb_nope<32>(st, c, h, q, n_rows, out);
    if (h.nope == 64) launch_absorb_nope<64>(st, c, h, q, n_rows, out);
    if (h.nope == 128) launch_absorb_nope<128>(st, c, h, q, n_rows, out);
}

// Up to one row and head per compute unit.  1 sequence of 30000 slots with 8 heads, whole call: a wavefront for a row 64 us, all eight 37; 8 of 4000 with
// 32 heads 42 and 34; with 512 rows and heads they are slower, 16 of 700 with 32 heads 33 and 40.
bool finish_few(const Heads& h, int n_rows) { return (int64_t)h.n * n_rows <= 256; }

// Rows of a workgroup: 32 of them share w_v, fewer where compute units would be left alone (64 rows of 32 heads in 9 to 16 parts: 64 workgroups 24
// us, 256 of eight rows 15; 48 rows of 128 heads: 256 workgroups 17 us, 768 of eight rows 24).
static int finish_span(const Heads& h, int n_rows) {
    if (finish_few(h, n_rows)) return 1;
    int span = 32;
    while (span > 8 && (int64_t)h.n * ((n_rows + span - 1) / span) < 256) span /= 2;
    return span;
}

static int64_t finish_groups(const Heads& h, int n_rows) {
    const int span = finish_span(h, n_rows);
    return (int64_t)h.n * ((n_rows + span - 1) / span);
}

bool finish_fits(const Heads& h, int n_rows) { return launchable(finish_groups(h, n_rows), 512); }

namespace {
template <int DC, int DV>
void launch_finish_sizes(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const RowsOut& out, const Parts& parts) {
    const int span = finish_span(h, s.n_rows);
    const dim3 grid((unsigned)finish_groups(h, s.n_rows)), block(512);
    if (finish_few(h, s.n_rows)) hipLaunchKernelGGL((finish_kernel<DC, DV, true>), grid, block, 0, st, c, s, h, out, parts, span);
    else hipLaunchKernelGGL((finish_kernel<DC, DV, false>), grid, block, 0, st, c, s, h, out, parts, span);
}
template <int DC>
void launch_finish_latent(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const RowsOut& out, const Parts& parts) {
    if (h.v == 32) launch_finish_sizes<DC, 32>(st, c, s, h, out, parts);
    if (h.v == 64) launch_finish_sizes<DC, 64>(st, c, s, h, out, parts);
    if (h.v == 128) launch_finish_sizes<DC, 128>(st, c, s, h, out, parts);
}
}  // namespace

void launch_finish(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const RowsOut& out, const Parts& parts) {
    if (c.latent == 128) launch_finish_latent<128>(st, c, s, h, out, parts);
    if (c.latent == 256) launch_finish_latent<256>(st, c, s, h, out, parts);
    if (c.latent == 512) launch_finish_latent<512>(st, c, s, h, out, parts);
}

}  // namespace klat
