// Class rows in 4-bit floats: quantisation and its way back, and products (arXiv 2206.04746, Sec. III, with rows between
// the bits of hdc_binarize_online and the 32-bit floats of hdc_search_cosine).
#include <algorithm>

#include "quantized.h"

namespace hdc {

namespace {

__device__ __forceinline__ double wave_sum(double v) {
    for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// A block of threads a row, a thread a block of 32 dimensions at a time.
__global__ __launch_bounds__(256) void quantize_rows_kernel(const float *__restrict__ rows, int64_t N, int D, int W, uint32_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales, double *__restrict__ norm, double *__restrict__ part, int G) {
    __shared__ double sums[4];
    const int tid = threadIdx.x;
    for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
        double mine = 0.0;
        for (int w = tid; w < W; w += 256) {
            const float *x = rows + n * D + (int64_t)w * 32;
            const int count = min(32, D - w * 32);
            uint32_t most = 0;   // of the magnitudes' bits, which are ordered like the numbers
            for (int i = 0; i < count; ++i) most = max(most, __float_as_uint(x[i]) & 0x7FFFFFFFu);
            int s = kQuantNone;
            uint32_t word[4] = {0, 0, 0, 0};
            if (most < 0x7F800000u) {
                s = max((int)(most >> 23) - 2, 0);   // floor(log2) less 2; what is below 2^-126 has 2^-127
                const double unit = scale_value(254 - s);
                for (int i = 0; i < count; ++i) {
                    const double v = fabs((double)x[i]) * unit;
                    uint32_t code = (v > 0.25) + (v >= 0.75) + (v > 1.25) + (v >= 1.75) + (v > 2.5) + (v >= 3.5) + (v > 5.0);
                    code |= __float_as_uint(x[i]) >> 31 << 3;
                    word[i & 3] |= code << (i & ~3);
                }
            }
            int q = 0;
            for (int i = 0; i < 32; ++i) {
                const int h = code_halves(word[i & 3] >> (i & ~3));
                q += h * h;
            }
            mine += (double)q * (0.25 * scale_value(s)) * scale_value(s);
            for (int i = 0; i < 4; ++i) codes[((int64_t)n * W + w) * 4 + i] = word[i];
            scales[(int64_t)n * W + w] = (uint8_t)s;
            if (part) {
                const double other = __shfl_xor(mine, 1, kWave);
                if ((w & 1) == 0) part[n * G + w / 2] = w + 1 < W ? mine + other : mine;
                mine = 0.0;
            }
        }
        if (norm) {
            const double sum = wave_sum(mine);
            if ((tid & 63) == 0) sums[tid >> 6] = sum;
            __syncthreads();
            if (tid == 0) norm[n] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
            __syncthreads();
        }
    }
}

// A thread four adjacent dimensions.
__global__ __launch_bounds__(256) void dequantize_rows_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t N, int D,
                                                              int W, float *__restrict__ rows) {
    for (int64_t n = blockIdx.x; n < N; n += gridDim.x)
        for (int d = threadIdx.x * 4; d < D; d += 1024) {
            const int w = d / 32, j = d % 32;
            const double unit = 0.5 * scale_value(scales[n * W + w]);
            for (int r = 0; r < 4 && d + r < D; ++r) {
                const uint32_t code = codes[(n * W + w) * 4 + r] >> j & 15;
                const float v = (float)(code_halves(code) * unit);
                rows[n * D + d + r] = code & 8 ? -v : v;
            }
        }
}

// A wave a product of two rows.
__global__ __launch_bounds__(256) void product_quantized_kernel(const uint32_t *__restrict__ a, const uint8_t *__restrict__ sa, int64_t M,
                                                                const uint32_t *__restrict__ b, const uint8_t *__restrict__ sb, int64_t N, int W,
                                                                float *__restrict__ out) {
    const int lane = threadIdx.x & 63;
    for (int64_t m = blockIdx.y; m < M; m += gridDim.y)
        for (int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); n < N; n += (int64_t)gridDim.x * 4) {
            double dot = 0.0;
            for (int w = lane; w < W; w += kWave) {
                int sum = 0;
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = a[(m * W + w) * 4 + i], y = b[(n * W + w) * 4 + i];
                    for (int j = 0; j < 32; j += 4) sum += code_signed_halves(x >> j) * code_signed_halves(y >> j);
                }
                dot += sum * (0.5 * scale_value(sa[m * W + w])) * (0.5 * scale_value(sb[n * W + w]));
            }
            dot = wave_sum(dot);
            if (lane == 0) out[m * N + n] = (float)dot;
        }
}

}  // namespace

int launch_quantize(hdc_ctx_impl *c, const float *rows, int64_t N, uint32_t *codes, uint8_t *scales, double *norm, double *part, hipStream_t s) {
    ProfScope prof(c, HDC_K_QUANTIZE_ROWS, s);
    hipLaunchKernelGGL(quantize_rows_kernel, dim3((unsigned)std::min<int64_t>(N, 1 << 20)), dim3(256), 0, s, rows, N, c->p.D, c->W, codes, scales, norm, part,
                       (c->p.D + kWave - 1) / kWave);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

int launch_dequantize(hdc_ctx_impl *c, const uint32_t *codes, const uint8_t *scales, int64_t N, float *rows, hipStream_t s) {
    hipLaunchKernelGGL(dequantize_rows_kernel, dim3((unsigned)std::min<int64_t>(N, 1 << 20)), dim3(256), 0, s, codes, scales, N, c->p.D, c->W, rows);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

int launch_product_quantized(hdc_ctx_impl *c, const uint32_t *a, const uint8_t *sa, int64_t M, const uint32_t *b, const uint8_t *sb, int64_t N, float *out,
                             hipStream_t s) {
    ProfScope prof(c, HDC_K_PRODUCT_QUANTIZED, s);
    const dim3 grid((unsigned)std::min<int64_t>((N + 3) / 4, 1 << 20), (unsigned)std::min<int64_t>(M, 65535));
    hipLaunchKernelGGL(product_quantized_kernel, grid, dim3(256), 0, s, a, sa, M, b, sb, N, c->W, out);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

}  // namespace hdc
