// Rows of 4-bit floats with a scale for every 32 dimensions (include/hdc.h, hdc_quantize): what the kernels that make and
// read them share.
//
// Block w of a row is the 32 dimensions of word w of a hypervector.  Nibble j of its word r is dimension 4 j + r, so that the
// bits of a hypervector's word that go with word r are (word << (3 - r)) & 0x88888888: signs, in the place that signs have.
#pragma once

#include "hdc_internal.h"

namespace hdc {

constexpr int kQuantNone = 255;   // the scale of a block that is no number
constexpr int kQuantZero = 127;   // the scale byte of 1

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// Magnitude of a code in halves.
__device__ __forceinline__ int code_halves(uint32_t code) { return (int)(0x0C08060403020100ull >> 8 * (code & 7) & 255); }
__device__ __forceinline__ int code_signed_halves(uint32_t code) { return code & 8 ? -code_halves(code) : code_halves(code); }

// The same number, of which the compiler does not know that it is: what is computed from it is computed here, and not kept in registers
// from before a loop.
template <typename T>
__device__ __forceinline__ T anew(T v) {
    asm volatile("" : "+v"(v));
    return v;
}

// 2^(s - 127) in 64 bits; a quiet NaN for a block that is no number.
__device__ __forceinline__ double scale_value(int s) {
    return s == kQuantNone ? __longlong_as_double(0x7FF8000000000000ll) : __longlong_as_double((long long)(s + 896) << 52);
}

}  // namespace hdc
