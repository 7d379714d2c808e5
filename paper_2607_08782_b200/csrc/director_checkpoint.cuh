// The 8-bit activation checkpoint: gate and up values of the expert FFNs, kept by the forward pass of training for the
// backward pass: 2 + 2/16 bytes a (row, feature) pair, where the bf16 values would take 4.
//
// Sixteen consecutive features of a row form a block; its gate values and its up values have a power-of-two scale each:
//   e = biased exponent of the block's largest magnitude - 6, at least 1;    code = clamp(rint(v 2^(127 - e)), -127, 127);
//   v is kept as code * 2^(e - 127).
// The largest magnitude gets a code of 64 to 127, so the error of a value is at most 2^-7 of the largest of its block (half a
// step of 2^-6; a magnitude above 127.5 steps is held at 127, which adds less than another half step).  A power of two makes
// both conversions exact up to the one rounding.  Why 16: in the gate|up GEMM's accumulator a warp holds exactly 16 features
// of both, so the maxima stay inside a warp.  Why gate and up apart: their magnitudes differ by layer, and the smaller of the
// two would lose its bits to the other's scale.  A block that holds a NaN or an infinity has e = 255 and codes of zero, and its
// values read as NaN: the gradient then shows that the activations were not finite.
#pragma once

#include <stdint.h>

namespace director {

constexpr int kCheckpointBlock = 16;

// codes: [rows][F][2] (gate, up);  exps: [F/16][rows] with the gate's exponent in the low and the up's in the high byte, so that
// the exponents of a block for consecutive rows are contiguous (a warp's lanes hold consecutive rows).
struct Checkpoint {
    int8_t* codes;
    uint16_t* exps;
    int rows;
};

#ifdef __CUDACC__
// The code in the low byte, two's complement; scale = 2^(127 - e).  Adding 1.5 * 2^23 rounds to the nearest integer, ties to
// even, and leaves it in the low bits (the product is exact, so there is the one rounding).
__device__ __forceinline__ uint32_t checkpoint_code(float v, float scale) {
    constexpr float magic = 12582912.0f;
    return __float_as_uint(fminf(fmaxf(fmaf(v, scale, magic), magic - 127.0f), magic + 127.0f));
}
// Magnitudes order as their bit patterns do, NaN above infinity, and so do their upper halves, which hold the exponents.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// 2^(e - 127), NaN for e = 255
__device__ __forceinline__ float checkpoint_scale(uint32_t e) {
    return __uint_as_float(e == 255u ? 0x7FC00000u : e << 23);
}
// The value of byte `byte` of four codes, given as codes ^ 0x80808080 (each plus 128): the byte in the low end of 2^23 is that
// integer as a float.  (An integer conversion instruction has a quarter of the rate of these.)
__device__ __forceinline__ float checkpoint_value(uint32_t biased_codes, int byte, float scale) {
    return (__uint_as_float(__byte_perm(biased_codes, 0x4B000000u, 0x7440u + byte)) - 8388736.0f) * scale;
}
#endif

}  // namespace director
