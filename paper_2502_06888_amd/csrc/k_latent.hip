// The latent cache: filling it; bringing queries into the latent space and sums out of it (the absorbed form's products around
// the attention itself, which is in k_latent_attn.hip).
#include "latent_device.h"

namespace klat {
namespace {

// One wavefront per row: 8 latents a lane, the mean of squares over the lanes, then one element of the part that turns a lane (its
// partner is read again, from the first-level cache).  Bound by latency, then by the rows read and written once.
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
        const float inv = 1.f / sqrtf(sum / (float)c.latent + a.eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack_bf16(bf_lo(v[i]) * inv * bf_lo(g[i]), bf_hi(v[i]) * inv * bf_hi(g[i]));
    }
    if (mine) *(u32x4*)(to + lane * 8) = v;
    if (turns) {
        const int position = (s.next_position != nullptr ? s.next_position[seq] : c.prefix_len + q.cached) + token;
        const float2 cs = krope::turn(a.turns.per_position[pair], position);
        const float cosine = cs.x * a.turns.magnitude, sine = cs.y * a.turns.magnitude;
        e = pack_bf16(krope::turned(bf_lo(e), bf_lo(partner), cosine, second ? sine : -sine), 0.f);
    }
    if (lane < c.rope) to[c.latent + lane] = (uint16_t)e;
}

// a[row][head] = w_k[head]^T n in bf16, then the part that carries the position, then what rounding a left over, in bf16, too:
// rows of 2 * latent + rope elements, in the caller's order of rows and heads.  (a counts with 16 bits: rounded to 8 it would move
// the scores, and with them the outputs, by more than the outputs' own rounding: 2.8e-3 over 3000 slots, where that is 1.7e-3.)
//
// One wavefront per (head, 128 latents, `each` tiles of 32 rows): its piece of w_k lies in LDS (nope_dim x 256 bytes) and is read
// transposed by the LDS, four latents of four rows at a time, as the first operand: a^T = w_k^T n^T, so that a lane has one row and
// four latents side by side.  The result goes through LDS to leave in pieces of 256 bytes.
template <int NOPE>
__global__ __launch_bounds__(64) void absorb_kernel(Cache c, Heads h, Rows q, int n_rows, int each, uint16_t* out) {
    __shared__ u32x4 w[NOPE * 16], o[2][32 * 16];
    const int lane = threadIdx.x, col = lane & 31, grp = lane >> 5;
    const int chunks = c.latent / 128, head = blockIdx.x % h.n, rest = blockIdx.x / h.n, chunk = rest % chunks;
    const int tile0 = rest / chunks * each, tiles = (n_rows + 31) / 32, width = 2 * c.latent + c.rope;
    // rows of w_k four at a time; 16-byte units of a row lie at an xor of its number, which spreads the transposed reads over the banks
    const uint16_t* from = h.w_k + head * h.w_k_head + chunk * 128 + (lane >> 4) * c.latent + ((lane & 15) ^ (lane >> 4 & 3) << 2) * 8;
    const uint32_t w_at = lds_address(w);
#pragma unroll
    for (int i = 0; i < NOPE / 4; ++i) copy_to_lds(from + (int64_t)i * 4 * c.latent, __builtin_amdgcn_readfirstlane(w_at + i * 1024));
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
    for (int t = 0; t < each && tile0 + t < tiles; ++t) {
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
        const int row0 = (tile0 + t) * 32;
        if (t + 1 < each && tile0 + t + 1 < tiles) load(tile0 + t + 1);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x2 x, y;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float e = acc[b][4 * i + 2 * j], e2 = acc[b][4 * i + 2 * j + 1];
                    x[j] = pack_bf16(e, e2);
                    y[j] = pack_bf16(e - bf_lo(x[j]), e2 - bf_hi(x[j]));
                }
                const int at = col * 16 + ((b * 4 + i) ^ (col & 15));
                ((u32x2*)&o[0][at])[grp] = x;
                ((u32x2*)&o[1][at])[grp] = y;
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int in = i * 4 + (lane >> 4), row = row0 + in;
            if (row < n_rows) {
                uint16_t* to = out + ((int64_t)row * h.n + head) * width + chunk * 128 + (lane & 15) * 8;
                *(u32x4*)to = o[0][in * 16 + ((lane & 15) ^ (in & 15))];
                *(u32x4*)(to + c.latent + c.rope) = o[1][in * 16 + ((lane & 15) ^ (in & 15))];
            }
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
        __syncthreads();
    }
}

// o = w_v u / sum for 32 rows of one head: the parts of a row's sums are brought to the largest reference and added,
// the result goes into LDS as two bf16 (value and what rounding it left over) in the order of the matrix instructions, and every
// wavefront takes 32 of the value's elements.  w_v is asked for before the parts are read.
template <int DC>
__global__ __launch_bounds__(256) void finish_kernel(Cache c, Step s, Heads h, RowsOut out, Parts parts) {
    constexpr int F = DC / 16;
    __shared__ u32x4 u[2][DC / 8 * 32];
    __shared__ int there[32];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, grp = lane >> 5;
    const int head = blockIdx.x % h.n, row0 = blockIdx.x / h.n * 32;
    const bool busy = wave * 32 < h.v;
    u32x4 wf[F];
    if (busy) {
        const uint16_t* p = h.w_v + head * h.w_v_head + (int64_t)(wave * 32 + col) * DC + grp * 8;
#pragma unroll
        for (int f = 0; f < F; ++f) wf[f] = *(const u32x4*)(p + f * 16);
    }
    for (int i = wave * 8; i < wave * 8 + 8; ++i) {
        const int row = row0 + i;
        Seq q;
        int token = 0;
        const int seq = row < s.n_rows ? seq_of_row(c, s, row, &token, &q) : -1;
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
        if (seq >= 0) {
            const int own = (q.cached + token + parts.per) / parts.per;  // parts of the slots that the row sees
            const int64_t item = ((int64_t)row * h.n + head) * parts.all;
            const int n = own + parts.all - parts.own;
            float ref = kEmpty, sum = 0.f;
            for (int k = 0; k < n; ++k) ref = fmaxf(ref, parts.ml[item + (k < own ? k : parts.own + k - own)].x);
            for (int k = 0; k < n; ++k) {
                const int64_t at = item + (k < own ? k : parts.own + k - own);
                const float2 ml = parts.ml[at];
                const float f = __builtin_amdgcn_exp2f(ml.x - ref);
                sum = __builtin_fmaf(ml.y, f, sum);
                if (lane * 8 < DC) {
                    const f32x4* p = (const f32x4*)(parts.acc + at * DC + lane * 8);
                    const f32x4 a = p[0], b = p[1];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[j] = __builtin_fmaf(a[j], f, x[j]);
                        x[4 + j] = __builtin_fmaf(b[j], f, x[4 + j]);
                    }
                }
            }
            const float inv = 1.f / sum;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= inv;
        }
        if (lane == 0) there[i] = seq >= 0;
        if (lane * 8 < DC) {
            u32x4 hi, lo;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                hi[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
                lo[j] = pack_bf16(x[2 * j] - bf_lo(hi[j]), x[2 * j + 1] - bf_hi(hi[j]));
            }
            u[0][lane * 32 + (i ^ (lane & 31))] = hi;
            u[1][lane * 32 + (i ^ (lane & 31))] = lo;
        }
    }
    __syncthreads();
    if (!busy) return;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int unit = 2 * f + grp;
        acc = mfma32(wf[f], u[0][unit * 32 + (col ^ (unit & 31))], acc);
        acc = mfma32(wf[f], u[1][unit * 32 + (col ^ (unit & 31))], acc);
    }
    if (!there[col]) return;
    uint16_t* o = out.p + (int64_t)(row0 + col) * out.row + (int64_t)head * out.head + wave * 32 + 4 * grp;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u32x2 x;
        x.x = pack_bf16(acc[4 * i], acc[4 * i + 1]);
        x.y = pack_bf16(acc[4 * i + 2], acc[4 * i + 3]);
        *(u32x2*)(o + 8 * i) = x;
    }
}

}  // namespace

void launch_append(hipStream_t st, const Cache& c, const Step& s, const Append& a) {
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)((s.n_rows + 3) / 4)), dim3(256), 0, st, c, s, a);
}

// Tiles of 32 rows of a wavefront: about 2048 wavefronts, which are eight per compute unit.
static int absorb_each(const Cache& c, const Heads& h, int n_rows) {
    const int64_t all = (int64_t)h.n * (c.latent / 128) * ((n_rows + 31) / 32);
    return all > 2048 ? (int)((all + 2047) / 2048) : 1;
}

int64_t absorb_groups(const Cache& c, const Heads& h, int n_rows) {
    const int64_t tiles = (n_rows + 31) / 32, each = absorb_each(c, h, n_rows);
    return h.n * (c.latent / 128) * ((tiles + each - 1) / each);
}

void launch_absorb(hipStream_t st, const Cache& c, const Heads& h, const Rows& q, int n_rows, uint16_t* out) {
    const dim3 grid((unsigned)absorb_groups(c, h, n_rows)), block(64);
    const int each = absorb_each(c, h, n_rows);
    if (h.nope == 32) hipLaunchKernelGGL(absorb_kernel<32>, grid, block, 0, st, c, h, q, n_rows, each, out);
    if (h.nope == 64) hipLaunchKernelGGL(absorb_kernel<64>, grid, block, 0, st, c, h, q, n_rows, each, out);
    if (h.nope == 128) hipLaunchKernelGGL(absorb_kernel<128>, grid, block, 0, st, c, h, q, n_rows, each, out);
}

int64_t finish_groups(const Heads& h, int n_rows) { return (int64_t)h.n * ((n_rows + 31) / 32); }

void launch_finish(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const RowsOut& out, const Parts& parts) {
    const dim3 grid((unsigned)finish_groups(h, s.n_rows)), block(256);
    if (c.latent == 128) hipLaunchKernelGGL(finish_kernel<128>, grid, block, 0, st, c, s, h, out, parts);
    if (c.latent == 256) hipLaunchKernelGGL(finish_kernel<256>, grid, block, 0, st, c, s, h, out, parts);
    if (c.latent == 512) hipLaunchKernelGGL(finish_kernel<512>, grid, block, 0, st, c, s, h, out, parts);
}

}  // namespace klat
