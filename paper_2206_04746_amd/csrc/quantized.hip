// Class rows in 4-bit floats: quantisation and its way back (arXiv 2206.04746, Sec. III, with rows between
// the bits of hdc_binarize_online and the 32-bit floats of hdc_search_cosine).
#include <algorithm>

#include "quantized.h"

namespace hdc {

namespace {

__device__ __forceinline__ double wave_sum(double v) {
    for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// Squares of the magnitudes in halves, by code: 0 1 4 9 16 36 64 144.
__device__ __forceinline__ int squares(uint32_t four) {
    return (int)__builtin_amdgcn_udot4(__builtin_amdgcn_perm(0x90402410u, 0x09040100u, four & 0x07070707u), 0x01010101u, 0u, false);
}

// Eight lanes a block of 32 dimensions, four adjacent ones a lane; a wave eight blocks at a time, twice.  Four elements become four codes
// in the bytes of a register (v_cvt_scalef32_pk_fp4_f32: nearest, ties to even, beyond 6 it is 6), and the eight lanes' registers the
// block's four words by two byte permutes: so rows are read in order and words written in order.  Bound by memory:
// 6238 rows of 9999 (249 MB in, 33 MB out) take 55.8 us, 5.07 TB/s.
// A block of threads a row (or, with norms by groups of 64 dimensions, `chunks` blocks); norm: the row's, or part: [row][group].
__global__ __launch_bounds__(1024) void quantize_rows_kernel(const float *__restrict__ rows, int64_t N, int D, int W, uint32_t *__restrict__ codes,
                                                             uint8_t *__restrict__ scales, double *__restrict__ norm, double *__restrict__ part, int G) {
    __shared__ double sums[16];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, waves = blockDim.x >> 6;
    const int j = lane & 7, pair = j >> 1;
    // A lane of pair q takes byte r of its own register and of pair q ^ 1's for its word's half, then halves from pair q ^ 2.
    const uint32_t pick = pair & 1 ? 0x03070105u : 0x06020400u, half = pair & 2 ? 0x03020706u : 0x05040100u;
    for (int64_t n = blockIdx.y; n < N; n += gridDim.y) {
        const float *const row = rows + n * D;
        double mine = 0.0;
        for (int w0 = (blockIdx.x * waves + wave) * 16; w0 < W; w0 += gridDim.x * waves * 16) {   // uniform
            uint32_t x[2][4], word[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int d = (w0 + 8 * k) * 32 + lane * 4;
                if (d + 4 <= D) {
                    __builtin_memcpy(x[k], row + d, 16);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[k][r] = d + r < D ? __float_as_uint(row[d + r]) : 0u;
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int w = w0 + 8 * k + (lane >> 3);
                uint32_t most = 0;   // of the magnitudes' bits, which are ordered like the numbers
#pragma unroll
                for (int r = 0; r < 4; ++r) most = max(most, x[k][r] & 0x7FFFFFFFu);
                most = max(most, lanes<kNext>(most));
                most = max(most, lanes<kNextPair>(most));
                most = max(most, lanes<kMirrorEight>(most));
                const bool none = most >= 0x7F800000u;
                const int s = none ? kQuantNone : scale_of(most);
                const float unit = scale_float(s);
                uint32_t four = 0;
                if (!none) {
                    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, __uint_as_float(x[k][0]), 0.0f, unit, 0);
                    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, __uint_as_float(x[k][1]), 0.0f, unit, 1);
                    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, __uint_as_float(x[k][2]), 0.0f, unit, 2);
                    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, __uint_as_float(x[k][3]), 0.0f, unit, 3);
                }
                mine = fma((double)squares(four), scale_square(s), mine);
                if (part) {   // sixteen lanes a group
                    for (int off = 1; off < 16; off <<= 1) mine += __shfl_xor(mine, off, kWave);
                    if ((lane & 15) == 0 && w < W) part[n * G + w / 2] = mine;
                    mine = 0.0;
                }
                four <<= 4 * (j & 1);
                four |= lanes<kNext>(four);
                const uint32_t two = __builtin_amdgcn_perm(lanes<kNextPair>(four), four, pick);
                word[k] = __builtin_amdgcn_perm(lanes<kNextPair>(lanes<kMirrorEight>(two)), two, half);
                if (j == 0 && w < W) scales[n * W + w] = (uint8_t)s;
            }
            const int w = w0 + 8 * (j & 1) + (lane >> 3);
            if (w < W) codes[(n * W + w) * 4 + pair] = word[j & 1];
        }
        if (norm) {
            const double sum = wave_sum(mine);
            if (lane == 0) sums[wave] = sum;
            __syncthreads();
            if (tid == 0) {
                double all = sums[0];
                for (int i = 1; i < waves; ++i) all += sums[i];
                norm[n] = all;
            }
            __syncthreads();
        }
    }
}

// The four codes of dimensions 4 g to 4 g + 3 of a row, one a byte: nibble g & 7 of each of a block's words.
__device__ __forceinline__ uint32_t four_codes(const uint32_t *__restrict__ codes, int64_t block, int g) {
    const v4u word = *reinterpret_cast<const v4u *>(codes + block * 4);
    uint32_t four = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) four |= (word[r] >> 4 * (g & 7) & 15) << 8 * r;
    return four;
}

constexpr int kLine = 32;   // floats of a cache line

// Four floats a lane, so that a wave stores whole cache lines: in a row that starts `ahead` floats before sixteen aligned bytes these are
// of two fours of codes, and the first lanes of a row, those before it in its first line, have nothing to do.  The stores leave the caches
// alone.  Bound by memory: 6238 rows of 9999 (33 MB in, 249 MB out) take 47 us, 6.0 TB/s, where stores that follow the codes take 75 us,
// those that also leave the caches alone 63; 60000 rows of 1001 take 59, for a line that two rows share is written twice.
__global__ __launch_bounds__(256) void dequantize_rows_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t N, int D,
                                                              int W, float *__restrict__ rows) {
    for (int64_t n = blockIdx.y; n < N; n += gridDim.y) {
        float *const row = rows + n * D;
        const int before = (int)((uintptr_t)row >> 2 & (kLine - 1)), ahead = -before & 3;   // uniform
        for (int d = (int)(blockIdx.x * blockDim.x + threadIdx.x) * 4 - before; d < D; d += gridDim.x * blockDim.x * 4) {
            if (d <= -4) continue;
            const int g = (d - ahead) >> 2;
            uint32_t four = 0, next = 0;
            int s = kQuantZero, t = kQuantZero;
            if (g >= 0) {
                const int64_t block = n * W + (g >> 3);
                four = four_codes(codes, block, g);
                s = scales[block];
            }
            if (ahead && 4 * g + 4 < D) {
                const int64_t block = n * W + ((g + 1) >> 3);
                next = four_codes(codes, block, g + 1);
                t = scales[block];
            }
            four = __builtin_amdgcn_alignbyte(next, four, ahead);
            const uint32_t halves = __builtin_amdgcn_perm(0x0C080604u, 0x03020100u, four & 0x07070707u);
            v4u x;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int scale = r + ahead < 4 ? s : t;
                const uint32_t v = __float_as_uint(ldexpf((float)(halves >> 8 * r & 255), scale - kQuantZero - 1));
                x[r] = scale == kQuantNone ? 0x7FC00000u : v | (four >> 8 * r & 8) << 28;
            }
            if (d >= 0 && d + 4 <= D) {
                __builtin_nontemporal_store(x, reinterpret_cast<v4u *>(row + d));
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (d + r >= 0 && d + r < D) row[d + r] = __uint_as_float(x[r]);
            }
        }
    }
}

}  // namespace

// Rows beyond a launch's 65535 are taken by the same blocks.
int launch_quantize(hdc_ctx_impl *c, const float *rows, int64_t N, uint32_t *codes, uint8_t *scales, double *norm, double *part, hipStream_t s) {
    ProfScope prof(c, HDC_K_QUANTIZE_ROWS, s);
    // A wave takes 512 dimensions at a time, a block of up to four waves a row; up to sixteen where there are fewer rows than compute units
    // (a row of 100000: 14 us a call, with four 31; 2000 rows of 9999: 21, with four 17).  Without norms to be summed over a row, several
    // blocks of four where there are few rows instead (a row of 100000 6.5 us, in one block 30; 6238 rows of 9999 46, in one 44).
    const int steps = (c->W + 15) / 16, waves = std::min(steps, norm && N < (int64_t)c->num_cus ? 16 : 4);
    const int chunks = norm ? 1 : (int)std::min<int64_t>((steps + waves - 1) / waves, std::max<int64_t>(1, 8 * (int64_t)c->num_cus / N));
    hipLaunchKernelGGL(quantize_rows_kernel, dim3((unsigned)chunks, (unsigned)std::min<int64_t>(N, 65535)), dim3((unsigned)waves * kWave), 0, s, rows, N,
                       c->p.D, c->W, codes, scales, norm, part, (c->p.D + kWave - 1) / kWave);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

int launch_dequantize(hdc_ctx_impl *c, const uint32_t *codes, const uint8_t *scales, int64_t N, float *rows, hipStream_t s) {
    // A wave writes 1 KiB at a time, twice where there are rows enough (6238 rows of 9999: once 57 us, twice 47, three times 56, five times 48;
    // 60000 of 1000: 46, 41, 45 and 50).
    const int64_t steps = (c->p.D + kLine - 1 + 255) / 256, each = N * steps >= 128 * (int64_t)c->num_cus ? 2 : 1;
    const int64_t waves = (steps + each - 1) / each, chunks = (waves + 3) / 4;
    hipLaunchKernelGGL(dequantize_rows_kernel, dim3((unsigned)chunks, (unsigned)std::min<int64_t>(N, 65535)),
                       dim3((unsigned)std::min<int64_t>(waves, 4) * kWave), 0, s, codes, scales, N, c->p.D, c->W, rows);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

}  // namespace hdc
