// The 8-bit format of kept activations: groups of 32 columns of a row share a power of two.
#pragma once

#include "train.cuh"

namespace ss {

inline int64_t act8_groups(int64_t cols) { return (cols + SS_ACT8_GROUP - 1) / SS_ACT8_GROUP; }

// A checkpoint: values first, `pitch` bytes a row, then one exponent byte for each group.
struct Ckpt {
    uint8_t* values;
    uint8_t* exps;
    int64_t groups;  // of one row; pitch = 32 * groups
};

inline Ckpt ckpt_of(uint8_t* p, int64_t rows, int64_t cols) {
    const int64_t groups = act8_groups(cols);
    return Ckpt{p, p == nullptr ? nullptr : p + rows * groups * SS_ACT8_GROUP, groups};
}

// Exponent byte e + 127 of a group from the largest magnitude's bits (as an integer: infinities
// and NaNs order above every number). With a = 1.m * 2^k, 127 * 2^e = 1.984375 * 2^(e+6) >= a
// gives e = k - 6 where 1.m <= 1.984375, else k - 5.
__device__ __forceinline__ uint32_t act8_exp_byte(uint32_t abs_bits) {
    if (abs_bits >= (253u << 23)) return 255u;  // not below 2^126
    const int b = static_cast<int>(abs_bits >> 23) - 6 + ((abs_bits & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
    return b < 1 ? 1u : static_cast<uint32_t>(b);
}

// 2^-e, for bytes 1 .. 247; a marked group's values are never used, any factor will do.
__device__ __forceinline__ float act8_inverse(uint32_t exp_byte) {
    return exp_byte == 255u ? 0.0f : __uint_as_float((254u - exp_byte) << 23);
}

// Sign and magnitude of x * 2^-e rounded to the nearest integer, ties to even: the product is
// exact (a power of two), and adding 2^23 rounds it at the unit.
__device__ __forceinline__ uint32_t act8_code(float x, float inverse) {
    const float t = __fmaf_rn(fabsf(x), inverse, 8388608.0f);
    return (__float_as_uint(t) & 0x7Fu) | ((__float_as_uint(x) >> 24) & 0x80u);
}

// 2^e, or NaN for a marked group.
__device__ __forceinline__ float act8_unit(uint32_t exp_byte) {
    return __uint_as_float(exp_byte == 255u ? 0x7FC00000u : exp_byte << 23);
}

// Value of a code: exact. `code` may carry other bits above its eight.
__device__ __forceinline__ float act8_value(uint32_t code, float unit) {
    const float m = __uint_as_float(0x4B000000u | (code & 0x7Fu)) - 8388608.0f;
    return (code & 0x80u) ? -(m * unit) : m * unit;
}

}  // namespace ss
