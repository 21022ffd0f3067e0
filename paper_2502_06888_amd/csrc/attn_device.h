// Device helpers of the attention kernels: the running softmax, matrix instructions, copies into LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kattn {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // to nearest even
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

constexpr float kEmpty = -3.40282347e38f;  // finite stand-in for "no slot seen yet": the lowest number, not above any finite score
// The reference of a running softmax is the largest score at the time it was set, and is set anew once a score exceeds it by
// more than kRise: the sums are not rescaled for every new maximum.  Weights are 2^(score - reference - kAbove): the largest
// one is a power of two at first, so that rounding it to bf16 takes nothing, and none is over 2^-20, so that the sums of 2^20
// slots of any finite values stay finite.
constexpr float kAbove = 28.f, kRise = 8.f, kBelow = 0x1p-28f;  // kBelow = 2^-kAbove
// score * factor - (reference + kAbove) is one fused operation; but the reference comes from a rounded product, where this
// one is exact.  That is half a step of the score, as any of its roundings; but from where a step is no longer
// small beside 1 the largest score itself would be put far above or below its reference, and from 2^29 on kAbove would be
// lost beside it.  Beyond kFar the product is rounded first, by itself, and reference and kAbove are taken off one after the other.
constexpr float kFar = 0x1p18f;
// The reference for a largest score: up to kFar one to which kAbove can be added without rounding, half a step of the sum off.
__device__ __forceinline__ float reference_of(float top) { return fabsf(top) > kFar ? top : (top + kAbove) - kAbove; }
__device__ __forceinline__ float apart(float score, float factor, float reference) {
#pragma clang fp contract(off)
    const float z = score * factor;
    return z - reference;
}
// Scores to exponents of the weights: score * factor - reference - above.  `each` takes what to make of every score of a lane.
template <class T>
__device__ __forceinline__ void exponents(float reference, float above, float factor, T&& each) {
    if (!__any(fabsf(reference) > kFar)) {
        const float less = reference + above;
        each([&](float score) { return __builtin_fmaf(score, factor, -less); });
    } else {
        each([&](float score) { return apart(score, factor, reference) - above; });
    }
}

// The wavefront's number in its workgroup, in a scalar register.
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ bf16x8 as_bf16x8(const u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ f32x4 mfma16(const u32x4 a, const u32x4 b, const f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
// 16 bytes per lane from `from` (the lane's own address) to LDS at `to` + 16 * lane, without registers; the wavefront waits
// for it with wait_copies().  The instruction takes the LDS address from m0, which is named as overwritten; the compiler
// keeps that register for itself and says so, though nothing else in these kernels uses it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(const void* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory", "m0");
}
// The same from `base` (uniform) + `offset` bytes (the lane's): the addresses then cost no vector instructions.
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(to) : "memory", "m0");
}
// The same past the caches, for what is read once.
__device__ __forceinline__ void stream_to_lds(const void* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(offset), "s"(base), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void copy_word_to_lds(const void* from, uint32_t to) {  // 4 bytes per lane, to `to` + 4 * lane
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(to) : "memory", "m0");
}
#pragma clang diagnostic pop
// Until at most N of the wavefront's copies (and other accesses) are on their way.
template <int N>
__device__ __forceinline__ void wait_copies() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mfma32(const u32x4 a, const u32x4 b, const f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
// Row of a 32x32 result that register r of a lane in half g holds.
__device__ __forceinline__ int row_of(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

}  // namespace kattn
