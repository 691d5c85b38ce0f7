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

// Magnitude of x * 2^-e rounded to the nearest integer, ties to even, in the low byte (bit 7 is 0):
// the product is exact (a power of two), and adding 2^23 rounds it at the unit.
__device__ __forceinline__ uint32_t act8_magnitude(float x, float inverse) {
    return __float_as_uint(__fmaf_rn(fabsf(x), inverse, 8388608.0f));
}

// The same for two bf16 (|x| given): numbers from 128 to 255 have their unit in the last place of
// a bf16, so one fused multiply-add rounds both where they belong.
__device__ __forceinline__ uint32_t act8_magnitude_pair(uint32_t abs_pair, uint32_t inverse_pair) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(abs_pair), "r"(inverse_pair), "r"(0x43004300u));
    return r;
}

// The exponent field of 2^(e+7), twice, for act8_value_pair; all ones for a marked group.
__device__ __forceinline__ uint32_t act8_exponent_pair(uint32_t exp_byte) {
    const uint32_t e = exp_byte == 255u ? 255u : exp_byte + 7u;
    return (e << 7) | (e << 23);
}

// Codes 2 PAIR and 2 PAIR + 1 of a word's four as two bf16, exactly. With E the exponent field of
// 2^(e+7), E | magnitude is 2^e (128 + magnitude) and E alone 2^e 128, both with the code's sign;
// their difference is exact. A marked group has the E of an infinity: inf - inf and NaN - inf are NaN.
template <int PAIR>
__device__ __forceinline__ uint32_t act8_value_pair(uint32_t codes, uint32_t exponent_pair) {
    const uint32_t r = __byte_perm(codes, 0, PAIR == 0 ? 0x1100 : 0x3322);
    const uint32_t a = (r & 0x807F807Fu) | exponent_pair, b = (r & 0x80008000u) | exponent_pair;
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

}  // namespace ss
