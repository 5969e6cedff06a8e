// Activations in 8 bits: blocks of 32 features of a row share a step, a power
// of two: the smallest that leaves the block's largest magnitude below 127.5
// steps. A value is its nearest multiple of the step (ties to even), so the error
// is at most half a step: 1 / 127.5 of the block's largest magnitude at most, or 2^-127
// where the step is the smallest.
// Everything is exact but that one rounding: x / step is a change of exponent,
// and code * step has 7 significant bits, so it is a bf16 value too, which
// lets the gradient's product take the codes to the matrix cores unrounded.
//
// A step is kept as its fp32 exponent field (1 .. 249); 255 marks a block that held
// an infinity or NaN, all of which come back as NaN.
#pragma once

#include "common.hpp"

namespace pyg {
namespace eight {

constexpr int kBlockLen = 32;
constexpr uint32_t kNotFinite = 255;

// The exponent field of the step for a block whose largest magnitude has these bits
// (as integers, magnitudes of floats keep their order, NaN above infinity).
__device__ __forceinline__ uint32_t step_of(uint32_t top) {
    const uint32_t ex = top >> 23;
    if (ex == 255) return kNotFinite;
    const int e = static_cast<int>(ex) - 6 + ((top & 0x7FFFFFu) >= 0x7F0000u ? 1 : 0);  // 127.5 / 64 = 1.9921875
    return e < 1 ? 1u : static_cast<uint32_t>(e);
}
__device__ __forceinline__ float step_value(uint32_t e) {
    return e == kNotFinite ? __uint_as_float(0x7FC00000u) : __uint_as_float(e << 23);
}
__device__ __forceinline__ float step_inverse(uint32_t e) {
    return e == kNotFinite ? 0.f : __uint_as_float((254u - e) << 23);
}
__device__ __forceinline__ uint32_t code(float x, float inverse, uint32_t e) {
    return e == kNotFinite ? 0u : static_cast<uint32_t>(static_cast<int>(rintf(x * inverse))) & 0xFFu;
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The four codes of a word as floats.
__device__ __forceinline__ void unpack(uint32_t w, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(static_cast<int>(w << (24 - 8 * i)) >> 24);
}

}  // namespace eight
}  // namespace pyg
