// Shared by the kernels of the latent cache: transposed reads of LDS, the parts of a row's sums.
#pragma once
#include "latent_kernels.h"

namespace klat {

typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T>
__device__ __forceinline__ uint32_t lds_address(T* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) T*)p;
}
__device__ __forceinline__ u32x4 read_lds(uint32_t at) { return *(__attribute__((address_space(3))) const u32x4*)(uintptr_t)at; }
__device__ __forceinline__ uint32_t read_lds_word(uint32_t at) { return *(__attribute__((address_space(3))) const uint32_t*)(uintptr_t)at; }
__device__ __forceinline__ void write_lds_word(uint32_t at, uint32_t v) { *(__attribute__((address_space(3))) uint32_t*)(uintptr_t)at = v; }
__device__ __forceinline__ void write_lds2(uint32_t at, const u32x2 v) { *(__attribute__((address_space(3))) u32x2*)(uintptr_t)at = v; }
// LDS accesses of a wavefront before it are done before those behind it: they run in order, the compiler has to keep them so.
__device__ __forceinline__ void wave_sync() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// Four rows of 16 elements of 16 bits, transposed: lane l of 16 points at four elements of row l / 4, 4 * (l % 4) on, and gets element l
// of the four rows.
__device__ __forceinline__ u32x2 read_transposed(uint32_t at) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)at));
}
__device__ __forceinline__ u32x4 join(const u32x2 a, const u32x2 b) { return u32x4{a.x, a.y, b.x, b.y}; }

// Where the eight 16-byte units of a slot's 128 bytes lie in LDS: unit u at place u ^ twist(slot).  A read of 16 bytes a lane takes lanes
// 0-3, 12-15, 20-23 and 24-27 together, then the others of 32: by the slot's bits 0 and 1 (half of the banks, and their half) and the
// permutation 0, 2, 3, 1 of bits 2 and 3 none of them meet, whether lanes 16-31 read the same unit of other slots or the next one of the
// same; and neither do transposed reads, of four units of four slots each.
__device__ __forceinline__ int twist(int slot) {
    const int q = slot >> 2 & 3;
    return (slot >> 1 & 1) << 2 | ((q ^ q >> 1) & 1) << 1 | q >> 1;
}

// Scores to exponents of the weights (attn_device.h), each lane's by its own reference: over a prefix rows of several sequences share a
// wavefront, and one with huge scores, or with none, must not change how the others' are rounded.
template <class T>
__device__ __forceinline__ void exponents_of_rows(float reference, float above, float factor, T&& each) {
    const float less = reference + above;
    const bool far = fabsf(reference) > kFar;
    if (!__any(far)) {
        each([&](float score) { return __builtin_fmaf(score, factor, -less); });
    } else {
        each([&](float score) {
            const float near = __builtin_fmaf(score, factor, -less);
            return far ? apart(score, factor, reference) - above : near;
        });
    }
}

// Sums, cut into parts: a row's slots into ranges of `per`, the prefix into ranges of its own, behind them.
struct Parts {
    int per, pre_per;  // slots of a range: of a sequence, of the prefix
    int own, all;      // parts of a row at most: of its sequence, with the prefix's
    float* acc;        // [row, head, part, element] sums of weight * latent, or means of the values
    float2* ml;        // [row, head, part] reference, sum of weights
};

// Whether finish_kernel has all wavefronts of a workgroup share a row's parts.
bool finish_few(const Heads& h, int n_rows);
bool absorb_fits(const Cache& c, const Heads& h, int n_rows);
void launch_absorb(hipStream_t st, const Cache& c, const Heads& h, const Rows& q, int n_rows, uint16_t* out);
bool finish_fits(const Heads& h, int n_rows);
void launch_finish(hipStream_t st, const Cache& c, const Step& s, const Heads& h, const RowsOut& out, const Parts& parts);

}  // namespace klat
