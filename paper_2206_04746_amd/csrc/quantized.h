// Rows of 4-bit floats with a scale for every 32 dimensions (include/hdc.h, hdc_quantize): what the kernels that make and
// read them share.
//
// Block w of a row is the 32 dimensions of word w of a hypervector.  Nibble j of its word r is dimension 4 j + r, so that the
// bits of a hypervector's word that go with word r are (word << (3 - r)) & 0x88888888: signs, in the place that signs have.
#pragma once

#include "hdc_internal.h"
#include "online_weight.h"

namespace hdc {

constexpr int kQuantNone = 255;   // the scale of a block that is no number
constexpr int kQuantZero = 127;   // the scale byte of 1

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// Products of 32 rows by 32 over 64 dimensions, or 16 by 16 over 128, on the matrix cores: a lane has the codes of a block of a row of either
// side, its scales in byte B of a register.
template <int BA, int BB>
__device__ __forceinline__ v16f mfma_codes(v4u a, v4u b, v16f c, uint32_t sa, uint32_t sb) {
    const v8i a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, b8 = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, c, 4, 4, BA, (int)sa, BB, (int)sb);
}
template <int BA, int BB>
__device__ __forceinline__ v4f mfma_codes(v4u a, v4u b, v4f c, uint32_t sa, uint32_t sb) {
    const v8i a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, b8 = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, BA, (int)sa, BB, (int)sb);
}
template <int B, typename Sums>
__device__ __forceinline__ Sums mfma(v4u a, v4u b, Sums c, uint32_t sa, uint32_t sb) {
    return mfma_codes<B, B>(a, b, c, sa, sb);
}
template <int B, typename Sums>   // with samples, whose scale is 1
__device__ __forceinline__ Sums mfma(v4u a, v4u b, Sums c, uint32_t sa) {
    return mfma_codes<B, 0>(a, b, c, sa, 0x7F7F7F7Fu);
}

// +-1 of a word's 32 dimensions in the order of the codes: 2 is the code of 1, 10 that of -1.
__device__ __forceinline__ v4u signs_of(uint32_t word) {
    v4u out;
#pragma unroll
    for (int r = 0; r < 4; ++r) out[r] = ((word << (3 - r)) & 0x88888888u) ^ 0xAAAAAAAAu;
    return out;
}

// The largest difference of scales of so many blocks whose sums with samples are without rounding in fp32.
constexpr int range_of(int blocks) {
    int r = 0;
    while ((int64_t)blocks * 192 * 2 << (r + 1) <= 1 << 24) ++r;
    return r;
}

// The nearest class so far; of equals the lowest.
constexpr int kNoClass = 0x7FFFFFFF;
struct Best {
    double cos;
    int c;
};
__device__ __forceinline__ Best better(Best a, Best b) { return b.cos > a.cos || (b.cos == a.cos && b.c < a.c) ? b : a; }

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

// Loads straight into LDS, 16 bytes a lane: lane i's go to `to` + 16 i.  By inline assembly, for a wave that has several on their way: around the
// builtin the compiler waits for all of them before every read of LDS.  The kernel waits for them itself (all loads return in order; a
// barrier alone does not wait), and keeps what it reads in between from places that are being loaded.
struct LdsSource {
    v4u words;   // a buffer's description
};
__device__ __forceinline__ LdsSource lds_source(const void *from, uint32_t bytes) {
    const uint64_t at = reinterpret_cast<uint64_t>(from);
    return {v4u{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32) & 0xFFFF),
                (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u}};
}
__device__ __forceinline__ void load_lds(LdsSource from, uint32_t lane_offset, uint32_t offset, uint32_t *to) {
    const uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t *)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(at), "v"(lane_offset), "s"(from.words), "s"((uint32_t)__builtin_amdgcn_readfirstlane((int)offset))
                 : "memory", "m0");
}

// 2^(s - 127) in 64 bits; a quiet NaN for a block that is no number.
__device__ __forceinline__ double scale_value(int s) {
    return s == kQuantNone ? __longlong_as_double(0x7FF8000000000000ll) : __longlong_as_double((long long)(s + 896) << 52);
}

// Lane exchanges within a row of 16: with the neighbour, with the neighbour's neighbour, and from the other end of eight lanes and of all.
template <int kSel>
__device__ __forceinline__ uint32_t lanes(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kSel, 0xF, 0xF, true);
}
constexpr int kNext = 0xB1, kNextPair = 0x4E, kMirrorEight = 0x141, kMirrorRow = 0x140;

// The scale byte of a block whose largest magnitude has these bits (of a number), and its value.
__device__ __forceinline__ int scale_of(uint32_t most) { return max((int)(most >> 23) - 2, 0); }   // floor(log2) less 2; what is below 2^-126: 2^-127
__device__ __forceinline__ float scale_float(int s) { return __uint_as_float(s ? (uint32_t)s << 23 : 0x00400000u); }
// A quarter of the square of a scale: what the square of a code's halves counts for.
__device__ __forceinline__ double scale_square(int s) {
    return s == kQuantNone ? scale_value(kQuantNone) : __longlong_as_double((long long)(2 * s + 1023 - 2 * kQuantZero - 2) << 52);
}

// Rows that are quantised as they are trained (online_batched.hip).
struct QuantRows {
    uint32_t *codes;
    uint8_t *scales;
};

// What online_weights_kernel makes of a batch's dot products, made where these are formed: the samples' weight records and, for few classes,
// their dense rows of signed weights (coef, width cb), and the transposed bits by blocks of their own.
struct QuantWeights {
    const int32_t *labels;
    const double *normpart;   // [C][G]
    OnlineWeight *records;
    double *coef;
    uint64_t *colmask;
    uint32_t *reset;          // a counter to be zero afterwards, or null
    int64_t ld;               // samples, up to a multiple of 64
    float lr;
    int G, cb, gw, tblocks;   // blocks for the transposed bits
};
bool quantized_weights_takes(int C);
int launch_quantized_weights(hdc_ctx_impl *c, const uint32_t *hv, int64_t nb, const uint32_t *codes, const uint8_t *scales, const QuantWeights &out,
                             hipStream_t s);

// Two blocks of a row, w and w + 1 (if there is one), an element a lane: their codes by ballots of the codes' bits, their scales, and, in
// every lane, what they add to the squared norm is to be summed from.
__device__ __forceinline__ double quantise_pair(QuantRows to, int64_t c, int w, int W, float x, int lane) {
    uint32_t most = __float_as_uint(x) & 0x7FFFFFFFu;
    most = max(most, lanes<kNext>(most));
    most = max(most, lanes<kNextPair>(most));
    most = max(most, lanes<kMirrorEight>(most));
    most = max(most, lanes<kMirrorRow>(most));
    most = max(most, (uint32_t)__shfl_xor((int)most, 16, kWave));
    const bool none = most >= 0x7F800000u;
    const int s = none ? kQuantNone : scale_of(most);
    const uint32_t code = none ? 0u : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x, 0.0f, scale_float(s), 0) & 15u;
    uint64_t bits[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) bits[k] = __ballot(code >> k & 1);
    const int block = lane >> 2 & 1;
    uint32_t word = 0;   // lane 4 b + r: word r of block b
#pragma unroll
    for (int k = 0; k < 4; ++k) word |= ((uint32_t)(bits[k] >> 32 * block) >> (lane & 3) & 0x11111111u) << k;
    if (lane < 8 && w + block < W) to.codes[(c * W + w) * 4 + lane] = word;
    if ((lane & 31) == 0 && w + (lane >> 5) < W) to.scales[c * W + w + (lane >> 5)] = (uint8_t)s;
    const int halves = code_halves(code);
    return (double)(halves * halves) * scale_square(s);
}

}  // namespace hdc
