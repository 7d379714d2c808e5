// The 8-bit activation checkpoint: gate and up values of the expert FFNs, kept by the forward pass of training for the
// backward pass: 2 + 2/16 bytes a (row, feature) pair, where the bf16 values would take 4.
//
// Sixteen consecutive features of a row form a block; its gate values and its up values have a power-of-two scale each:
//   e = biased exponent of the block's largest magnitude - 6, at least 1;    code = clamp(rint(v 2^(127 - e)), -127, 127);
//   v is kept as code * 2^(e - 127).
// The largest magnitude gets a code of 64 to 127, so the error of a value is at most 2^-7 of the largest of its block (half a
// step of 2^-6; a magnitude above 127.5 steps is held at 127, which adds less than another half step).  A power of two makes
// both conversions exact up to the one rounding.  Why 16: in the gate|up GEMM's accumulator a warp holds exactly 16 features
// of both, so the maxima are warp reductions.  Why gate and up apart: their magnitudes differ by layer, and the smaller of the
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
// from the bit pattern of the block's largest magnitude (magnitudes order as their bit patterns do; NaN above infinity)
__device__ __forceinline__ uint32_t checkpoint_exponent(uint32_t max_bits) {
    const uint32_t biased = max_bits >> 23;
    return biased == 255u ? 255u : (biased > 7u ? biased - 6u : 1u);
}
__device__ __forceinline__ int checkpoint_code(float v, uint32_t e) {
    const float scaled = v * __uint_as_float((254u - e) << 23);       // 2^(127 - e)
    const int code = __float2int_rn(fminf(fmaxf(scaled, -127.0f), 127.0f));
    return e == 255u ? 0 : code;
}
// 2^(e - 127), NaN for e = 255
__device__ __forceinline__ float checkpoint_scale(uint32_t e) {
    return __uint_as_float(e == 255u ? 0x7FC00000u : e << 23);
}
#endif

}  // namespace director
