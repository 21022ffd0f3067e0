// Rotary positions: the frequencies of a configuration (host) and the turn of a pair (device).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/moe_rope.h"
#include "call_checks.h"

namespace krope {

constexpr int kMostPairs = 128;

// Turns per position of each pair, w_i / (2 pi): 53 bits and the next 11, without which positions near 2^31 would be 2^-22 of a quarter turn off.
// Passed by value: 1.5 KiB of kernel arguments, nothing to own or to free.
struct Turns {
    double per_position[kMostPairs];
    float rest[kMostPairs];
    float magnitude;
};

// The powers of the frequency base one after the other with 64 bits of fraction: 127 products are 2^-57 off at most, and the call
// pays for one power, not for 128.
inline Turns turns_of(const moe_rope_config& c) {
    Turns t{};
    t.magnitude = (float)c.magnitude;
    const long double two_pi = 6.283185307179586476925286766559L;
    const long double ratio = powl((long double)c.theta, -2.0L / c.rot_dim);
    long double w = 1.0L;
    for (int i = 0; i < c.rot_dim / 2; ++i, w *= ratio) {
        long double keep = 0.0L;
        if (c.original_len > 0) {
            keep = (c.original_len * w / two_pi - c.low_turns) / ((long double)c.high_turns - c.low_turns);
            keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
        }
        const long double turns = w * (keep + (1.0L - keep) / c.factor) / two_pi;
        t.per_position[i] = (double)turns;
        t.rest[i] = (float)(turns - (long double)t.per_position[i]);
    }
    return t;
}

inline moe_status check_config(const moe_rope_config* c, kcall::CallError& e) {
    if (!c) return e.fail(MOE_ERR_INVALID_ARG, "the rotation's configuration is null");
    if (c->rot_dim < 2 || c->rot_dim > 2 * kMostPairs || c->rot_dim % 2 != 0) return e.fail(MOE_ERR_SHAPE, "rot_dim must be even, 2..256");
    if (c->first < 0) return e.fail(MOE_ERR_INVALID_ARG, "first is negative");
    if (c->interleaved != 0 && c->interleaved != 1) return e.fail(MOE_ERR_INVALID_ARG, "interleaved must be 0 or 1");
    if (c->original_len < 0 || c->original_len > (1 << 30)) return e.fail(MOE_ERR_INVALID_ARG, "original_len outside 0..2^30");
    if (!(c->theta > 0) || std::isinf(c->theta)) return e.fail(MOE_ERR_INVALID_ARG, "theta must be finite and > 0");
    if (!(c->factor > 0) || std::isinf(c->factor)) return e.fail(MOE_ERR_INVALID_ARG, "factor must be finite and > 0");
    if (!std::isfinite((float)c->magnitude)) return e.fail(MOE_ERR_INVALID_ARG, "magnitude must be finite in 32 bits");
    if (c->original_len > 0 && (!(c->low_turns >= 0) || !(c->high_turns > c->low_turns) || std::isinf(c->high_turns)))
        return e.fail(MOE_ERR_INVALID_ARG, "low_turns must be >= 0 and less than high_turns, both finite");
    return MOE_OK;
}

// Cosine and sine of `position` times a pair's turns.  Whole turns are taken off the exact product, the turns' last bits are added, and the rest is
// reduced to quarters, so that in 32 bits it is at most half of one: an angle is off by less than 2^-25 of a quarter turn at any position
// where w_i is at most 1 (of less than 2^31 radians where it is not).
__device__ __forceinline__ float2 turn(const Turns& turns, int pair, int position) {
    const double at = (double)position, per = turns.per_position[pair];
    const double part = __builtin_fma(at, (double)turns.rest[pair], __builtin_fma(at, per, -rint(at * per)));
    const double quarters = part * 4.0, whole = rint(quarters);
    float s, c;
    sincospif((float)(quarters - whole) * 0.5f, &s, &c);
    const int q = (int)whole & 3;
    const float a = q & 1 ? s : c, b = q & 1 ? c : s;
    return make_float2(q == 1 || q == 2 ? -a : a, q & 2 ? -b : b);
}

// What an element of a pair becomes, from itself and the other one; `sine` negated for the pair's first.  Which product is rounded by
// itself is written down, so that every kernel gives the same bits.
__device__ __forceinline__ float turned(float own, float other, float cosine, float sine) { return __builtin_fmaf(own, cosine, other * sine); }

struct Rows {
    const void* in;
    void* out;
    int32_t heads;
    int64_t in_row, in_head, out_row, out_head;
};

struct Rotate {
    Turns turns;
    Rows x[2];  // q, k
    int32_t n_rows, head_dim, rot, first, interleaved;
    const int32_t* positions;
};

// Whether rows move 16 bytes at a time.
bool by_pieces(const Rotate& r, bool f32);
void launch_rotate(hipStream_t st, const Rotate& r, bool f32);

}  // namespace krope
