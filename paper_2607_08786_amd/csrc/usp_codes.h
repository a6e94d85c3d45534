// usp_codes.h -- tokens in 8 bits: the scale of a token and the code of a value, as
// usp_quantize defines them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace usp {
namespace {

// fp16 magnitudes order as their bits do, NaN above infinity above all others.
__device__ inline uint32_t magnitude_bits(_Float16 h) { return __builtin_bit_cast(uint16_t, h) & 0x7FFFu; }

// Scale and reciprocal of a token's codes from the bits of its largest magnitude.
__device__ inline void code_scale(uint32_t top, float &scale, float &inv) {
    const float a = (float)__builtin_bit_cast(_Float16, (uint16_t)top);
    const bool finite = top < 0x7C00u;
    scale = finite ? a / 127.f : __builtin_nanf("");
    inv = finite && top ? 127.f / a : 0.f;
}

// A value's code as a byte; inv is 0 for tokens whose codes are all 0 (it may then meet
// a NaN or an infinity, whose product must not be converted).
__device__ inline uint32_t code_bits(_Float16 h, float inv) {
    return inv == 0.f ? 0u : (uint32_t)(uint8_t)(int)rintf((float)h * inv);
}

}  // namespace
}  // namespace usp
