// Rotary positions over rows of queries and keys.
//
// (a, b) -> (a cos - b sin, b cos + a sin) for every pair of a head, with an angle that all heads of a row share: a workgroup
// forms the cosines and sines of its rows once, in LDS, and then turns q's and k's heads of those rows.  Bound by the bytes of
// the rows, read and written once.
#include "attn_device.h"
#include "rope.h"

namespace krope {
namespace {

using namespace kattn;

template <class T>
constexpr int kPiece = 16 / sizeof(T);

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void narrow(float x, float* to) { *to = x; }
__device__ __forceinline__ void narrow(float x, uint16_t* to) { *to = (uint16_t)pack_bf16(x, x); }

// V elements side by side: one load, one store.
template <class T, int V>
struct alignas(V * sizeof(T)) Part {
    T e[V];
};

// V = 1: an item is a pair, or an element that does not turn.  Else it is two pieces of 16 bytes (halves as pairs) or one (pairs side by
// side, or elements that do not turn).
template <class T, bool INTERLEAVED, int V>
__global__ __launch_bounds__(256) void rotate_kernel(Rotate r, int rows_each) {
    extern __shared__ float2 table[];  // [row of the workgroup][pair]
    const int pairs = r.rot / 2, row0 = blockIdx.x * rows_each, rows = min(rows_each, r.n_rows - row0);
    for (int i = threadIdx.x; i < rows * pairs; i += 256) {
        const float2 cs = turn(r.turns, i % pairs, r.positions[row0 + i / pairs]);
        table[i] = make_float2(cs.x * r.turns.magnitude, cs.y * r.turns.magnitude);
    }
    __syncthreads();
    constexpr bool APART = !INTERLEAVED && V > 1;
    const int turning = V == 1 ? pairs : APART ? pairs / V : r.rot / V;  // items of a head that turn
    const int items = turning + (r.head_dim - r.rot) / V, heads = r.x[0].heads + r.x[1].heads;
    for (int i = threadIdx.x; i < rows * heads * items; i += 256) {
        const int at = i % items, rest = i / items, h = rest % heads, row = rest / heads;
        const bool second = h >= r.x[0].heads;
        const Rows& x = r.x[second];
        const int head = second ? h - r.x[0].heads : h;
        const T* in = (const T*)x.in + (int64_t)(row0 + row) * x.in_row + (int64_t)head * x.in_head;
        T* out = (T*)x.out + (int64_t)(row0 + row) * x.out_row + (int64_t)head * x.out_head;
        typedef Part<T, V> P;
        if (at >= turning) {
            if (in == out) continue;
            int e = (at - turning) * V;
            if (e >= r.first) e += r.rot;
            *(P*)(out + e) = *(const P*)(in + e);
        } else if constexpr (INTERLEAVED && V > 1) {
            const P p = *(const P*)(in + r.first + at * V);
            P o;
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const float2 cs = table[row * pairs + (at * V + j) / 2];
                const float a = widen(p.e[j]), b = widen(p.e[j + 1]);
                narrow(turned(a, b, cs.x, -cs.y), &o.e[j]);
                narrow(turned(b, a, cs.x, cs.y), &o.e[j + 1]);
            }
            *(P*)(out + r.first + at * V) = o;
        } else {
            const int lo = r.first + (INTERLEAVED ? 2 * at : at * V), hi = lo + (INTERLEAVED ? 1 : pairs);
            const P p = *(const P*)(in + lo), q = *(const P*)(in + hi);
            P o, s;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float2 cs = table[row * pairs + at * V + j];
                const float a = widen(p.e[j]), b = widen(q.e[j]);
                narrow(turned(a, b, cs.x, -cs.y), &o.e[j]);
                narrow(turned(b, a, cs.x, cs.y), &s.e[j]);
            }
            *(P*)(out + lo) = o;
            *(P*)(out + hi) = s;
        }
    }
}

template <class T>
void launch(hipStream_t st, const Rotate& r, bool f32) {
    const bool pieces = by_pieces(r, f32);
    // As many rows to a workgroup as give each thread an item.  Several items each leave too few wavefronts at once to hide the reads: 2051 rows
    // of 21 heads of 192 floats, 64 of them turned, with four rows to a workgroup 22 us, with one 16; 8192 rows of 40 heads of 128 bf16 27.2 and
    // 26.  (A launch has less than 2^32 threads.)
    const int v = pieces ? kPiece<T> : 1, of_head = (r.head_dim - (r.interleaved && pieces ? 0 : r.rot / 2)) / v;
    const int64_t items = (int64_t)(r.x[0].heads + r.x[1].heads) * of_head;
    const int each = max((int)min(max(256 / items, (int64_t)1), (int64_t)8), (r.n_rows >> 23) + 1);
    const dim3 grid((unsigned)((r.n_rows + each - 1) / each)), block(256);
    const unsigned lds = (unsigned)(each * (r.rot / 2) * sizeof(float2));
    if (r.interleaved) {
        if (pieces) hipLaunchKernelGGL((rotate_kernel<T, true, kPiece<T>>), grid, block, lds, st, r, each);
        else hipLaunchKernelGGL((rotate_kernel<T, true, 1>), grid, block, lds, st, r, each);
    } else {
        if (pieces) hipLaunchKernelGGL((rotate_kernel<T, false, kPiece<T>>), grid, block, lds, st, r, each);
        else hipLaunchKernelGGL((rotate_kernel<T, false, 1>), grid, block, lds, st, r, each);
    }
}

}  // namespace

bool by_pieces(const Rotate& r, bool f32) {
    const int v = f32 ? 4 : 8;
    if (r.head_dim % v != 0 || r.first % v != 0 || (r.interleaved ? r.rot : r.rot / 2) % v != 0) return false;
    for (const Rows& x : r.x) {
        if (x.heads == 0) continue;
        if (((uintptr_t)x.in | (uintptr_t)x.out) % 16 != 0) return false;
        if (x.in_row % v != 0 || x.in_head % v != 0 || x.out_row % v != 0 || x.out_head % v != 0) return false;
    }
    return true;
}

void launch_rotate(hipStream_t st, const Rotate& r, bool f32) {
    if (f32) launch<float>(st, r, true);
    else launch<uint16_t>(st, r, false);
}

}  // namespace krope
