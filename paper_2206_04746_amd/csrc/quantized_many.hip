// Cosine inference with class rows of 4-bit floats, for many samples and many classes (arXiv 2206.04746, Sec. III): a block takes
// 128 classes and 256 samples, 256 dimensions at a time.  The codes go through LDS, with room for three steps; a wave's samples are 64 of
// the 256, whose words it turns into +-1 itself (7 instructions for 32 dimensions, for 128 classes), so that of both sides together a step
// loads 24 KB for 17 MFLOP.  16001 samples of 8191 dimensions by 1024 classes take 103 us, 2.6 PFLOP/s, 64000 of 10000 366 us, 3.6.
// Matrix instructions are 29 of the 103 us (28 % of the active cycles, at 2.3 GHz).  What bounds it is a step's latency: scales come by
// ordinary loads, and before it takes or asks for them the compiler waits for all that the two waves that bring them have on their
// way, the latest loads into LDS too, for which the other two waves then wait at the barrier.  After the loop 53 registers a lane are spilled (216
// bytes of scratch; 28 MB of the 95 that such a call writes).
//
// The sums are of fp32, over the whole row, and without rounding: whole multiples of half the row's smallest scale, at most 192
// of its largest for a block.  scan_kernel finds out whether every row's scales lie near enough to one another for that; if
// one's do not, this kernel leaves the call to the one that takes them in passes (quantized_search.hip).
#include <algorithm>
#include <type_traits>

#include "quantized.h"

namespace hdc {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave, kTile = 32;
constexpr int kA = 4, kB = 2;                        // tiles of classes of a wave, and of samples
constexpr int kClasses = kA * kTile, kSamples = kWaves * kB * kTile;
constexpr int kStep = 8, kUnit = 16;                 // blocks of 32 dimensions a step, bytes of one's codes
constexpr int kBuffers = 3;                          // steps in LDS


// limits[c]: the largest scale of row c (-1: a row of zeros); limits[kMost + c]: whether its scales lie further apart than 2^range.
constexpr int kMost = HDC_MAX_C;
__global__ __launch_bounds__(256) void scan_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, int W, int range,
                                                   int *__restrict__ limits) {
    __shared__ int of[2][4];
    const int c = blockIdx.x, tid = threadIdx.x;
    int most = -1, least = 256;
    for (int w = tid; w < W; w += 256) {
        const int64_t at = (int64_t)c * W + w;
        const int s = scales[at];
        if (s == 0) {   // a block of zeros counts for nothing
            const v4u code = *reinterpret_cast<const v4u *>(codes + at * 4);
            if (((code[0] | code[1] | code[2] | code[3]) & 0x77777777u) == 0) continue;
        }
        most = max(most, s), least = min(least, s);
    }
    for (int off = 1; off < kWave; off <<= 1) most = max(most, __shfl_xor(most, off, kWave)), least = min(least, __shfl_xor(least, off, kWave));
    if ((tid & 63) == 0) of[0][tid >> 6] = most, of[1][tid >> 6] = least;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < 4; ++w) most = max(most, of[0][w]), least = min(least, of[1][w]);
        limits[c] = most;
        limits[kMost + c] = most >= 0 && most != kQuantNone && most - least > range;
    }
}

// grid: classes' tiles of eight samples' tiles at a time, a die's together.  pred_out, or best_cos and best_c [classes' tile][N].
__global__ __launch_bounds__(kThreads, 2) void search_many_kernel(const uint32_t *__restrict__ hv, int64_t N, int W, int C,
                                                                  const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                                  const double *__restrict__ norm, double root_d, const int *__restrict__ limits, int range,
                                                                  float *__restrict__ cos_out, int32_t *__restrict__ pred_out,
                                                                  double *__restrict__ best_cos, int *__restrict__ best_c) {
    // Codes: block k of a row's eight is at place k ^ (row / 2 % 8) of the row, so that sixteen rows' blocks lie in different banks.
    __shared__ __align__(16) uint32_t unit[kBuffers][kClasses * kStep * 4];
    __shared__ __align__(16) uint32_t words[kBuffers][kSamples * kStep];   // of the samples
    __shared__ uint32_t scale[2][4][kClasses];   // of two steps, and of the next two; relative to the row's largest, 127
    __shared__ double value[kClasses], size[kClasses];   // the largest scale; the row's norm times a sample's
    __shared__ double ratio[kClasses];                   // value / size
    __shared__ __align__(16) float about[kClasses];      // ... in fp32
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    const int tiles_c = (C + kClasses - 1) / kClasses, steps = (W + kStep - 1) / kStep;
    const int die = blockIdx.x % 8, in = blockIdx.x / 8;
    const int tc = __builtin_amdgcn_readfirstlane(in % tiles_c);
    const int64_t n0 = ((int64_t)(in / tiles_c) * 8 + die) * kSamples;
    const int c0 = tc * kClasses, rows = min(kClasses, C - c0);
    int wide = 0;
    for (int c = tid; c < C; c += kThreads) wide |= limits[kMost + c];
    if (__syncthreads_or(wide) || n0 >= N) return;

    // This thread's class, where it has one: scales are brought to LDS by the threads of the first two waves.
    const int own = min(c0 + tid, C - 1);
    int top = 0;
    if (tid < kClasses) {
        const int most = limits[own];
        top = (most < 0 ? kQuantZero : most) - kQuantZero;
        const double v = scale_value(most < 0 ? kQuantZero : most), z = c0 + tid < C ? sqrt(norm[own]) * root_d : scale_value(kQuantNone);
        value[tid] = v, size[tid] = z;
        ratio[tid] = z == 0.0 ? 0.0 : v / z;
        about[tid] = (float)(z == 0.0 ? 0.0 : v / z);
    }

    // A step's blocks, or the row's last eight: those that the step before has had are zeros then.
    auto begin_of = [&](int step) { return min(step * kStep, W - kStep); };
    const uint32_t pitch = (uint32_t)W * kUnit;
    const int rows_n = (int)min((int64_t)kSamples, N - n0);
    const LdsSource from_codes = lds_source(codes + (int64_t)c0 * W * 4, (uint32_t)rows * pitch), from_words = lds_source(hv + n0 * W, (uint32_t)rows_n * pitch / 4);
    auto load = [&](int step) {   // rows past the last are taken from it
        const uint32_t begin = (uint32_t)begin_of(step), at = (begin + ((lane & 7) ^ ((wave & 1) * 4 + (lane >> 4)))) * kUnit;
        const int l = anew(lane);
#pragma unroll
        for (int i = 0; i < kClasses / 32; ++i)   // eight rows a wave
            load_lds(from_codes, (uint32_t)min(i * 32 + wave * 8 + (l >> 3), rows - 1) * pitch + at, 0, unit[step % kBuffers] + (i * 32 + wave * 8) * kStep * 4);
#pragma unroll
        for (int j = 0; j < kB; ++j)   // a wave's own samples, half a step's words a lane
            load_lds(from_words, (uint32_t)min((wave * kB + j) * kTile + (l >> 1), rows_n - 1) * (pitch / 4) + (begin + 4 * (l & 1)) * 4, 0,
                     words[step % kBuffers] + (wave * kB + j) * kTile * kStep);
    };
    uint32_t piece[4];
    auto ask_scales = [&](int step) {   // of two steps
        __builtin_memcpy(piece, scales + (int64_t)own * W + begin_of(step), 8);
        __builtin_memcpy(piece + 2, scales + (int64_t)own * W + begin_of(step + 1), 8);
    };
    auto put_scales = [&](int step) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t to = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {   // (further away than `range` is none but a block of zeros)
                const int rel = (int)(piece[i] >> 8 * k & 255) - top;
                to |= (uint32_t)(rel <= kQuantZero && rel >= kQuantZero - range ? rel : kQuantZero) << 8 * k;
            }
            scale[step / 2 & 1][i][tid] = to;
        }
    };
    int64_t n_of[kB];
#pragma unroll
    for (int j = 0; j < kB; ++j) n_of[j] = n0 + (wave * kB + j) * kTile + col;
    v4u word[kB];
    v16f acc[kA][kB] = {};
    v4u x[2][kA];
    uint32_t sx[kA];
    auto take = [&](int step, int t) {
        const uint32_t *const from = unit[step % kBuffers] + (col * kStep + ((4 * half + t) ^ (col >> 1 & 7))) * 4;
#pragma unroll
        for (int i = 0; i < kA; ++i) x[t & 1][i] = *reinterpret_cast<const v4u *>(from + i * kTile * kStep * 4);
    };
    auto take_words = [&](int step) {
#pragma unroll
        for (int j = 0; j < kB; ++j) word[j] = *reinterpret_cast<const v4u *>(words[step % kBuffers] + ((wave * kB + j) * kTile + col) * kStep + 4 * half);
    };
    auto take_scales = [&](int step) {
#pragma unroll
        for (int i = 0; i < kA; ++i) sx[i] = scale[step / 2 & 1][(step & 1) * 2 + half][i * kTile + col];
    };
    auto multiply = [&](auto t_of) {
        constexpr int t = decltype(t_of)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < kB; ++j) {
            const v4u sign = signs_of(word[j][t]);
#pragma unroll
            for (int i = 0; i < kA; ++i) acc[i][j] = mfma<t>(x[t & 1][i], sign, acc[i][j], sx[i]);
        }
#pragma unroll
        for (int i = 0; i < kA; ++i)   // here, and not past the next barrier
#pragma unroll
            for (int j = 0; j < kB; ++j) acc[i][j] = anew(acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // Blocks that the step before has had.
    auto clear = [&](int step) {
        const int again = step * kStep - begin_of(step);   // (of the last step only)
        if (again > 0) {
            for (int u = tid; u < kClasses * kStep; u += kThreads)
                if (((u & 7) ^ (u >> 4 & 7)) < again) *reinterpret_cast<v4u *>(unit[step % kBuffers] + u * 4) = v4u{0, 0, 0, 0};
            __syncthreads();
        }
    };

    // At the end of a step its buffer takes the third step from it (past the row, the last ones again), and no more than these loads are on their
    // way when the next step begins (of the waves that bring scales none).
    constexpr int kLoads = kClasses / 32 + kB;
    static_assert(kLoads == 6, "what is waited for");
    auto meet = [&]() {
        asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
        __syncthreads();
    };
    if (tid < kClasses) ask_scales(0);
    load(0);
    load(1);
    if (tid < kClasses) put_scales(0);
    load(2);
    meet();
    for (int k = 0;; ++k) {
        clear(k);
        take_words(k);
        take_scales(k);
        take(k, 0);
        take(k, 1);
        multiply(std::integral_constant<int, 0>{});
        take(k, 2);
        multiply(std::integral_constant<int, 1>{});
        take(k, 3);
        multiply(std::integral_constant<int, 2>{});
        multiply(std::integral_constant<int, 3>{});
        if (k + 1 == steps) break;
        if (tid < kClasses && (k & 1)) put_scales(k + 1);
        meet();
        if (tid < kClasses && !(k & 1)) ask_scales(k + 2);
        load(k + 3);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing may be on its way into LDS when the block's is given to another)

    // Register r of lane 32 h + col: class 8 (r / 4) + 4 h + r % 4 of a tile, the column's sample.
#pragma unroll
    for (int j = 0; j < kB; ++j) {
        float best = -__builtin_inff(), second = -__builtin_inff(), sum = 0.0f;   // of the cosines in fp32, and the best's sum
        int at = kNoClass;
#pragma unroll
        for (int i = 0; i < kA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int first = i * kTile + 8 * q + 4 * half;
                const v4f by = *reinterpret_cast<const v4f *>(about + first);
                if (cos_out && n_of[j] < N) {
                    float out[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[r] = (float)((double)acc[i][j][4 * q + r] * ratio[first + r]);
                    float *const to = cos_out + n_of[j] * C + c0 + first;
                    if (c0 + first + 4 <= C) {
                        __builtin_memcpy(to, out, 16);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (c0 + first + r < C) to[r] = out[r];
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {   // (what is no number is neither above nor below)
                    const float v = acc[i][j][4 * q + r] * by[r];
                    const bool above = v > best;
                    second = above ? best : fmaxf(second, v);
                    best = above ? v : best, at = above ? first + r : at, sum = above ? acc[i][j][4 * q + r] : sum;
                }
            }
        const float other = __shfl_xor(best, 32, kWave);
        const bool near_it = fmaxf(fminf(best, other), fmaxf(second, __shfl_xor(second, 32, kWave))) >= fmaxf(best, other) * (1.0f - copysignf(0x1p-19f, fmaxf(best, other)));
        Best nearest = {at == kNoClass ? -__builtin_inf() : size[at & (kClasses - 1)] == 0.0 ? 0.0 : (double)sum * value[at & (kClasses - 1)] / size[at & (kClasses - 1)], at};
        if (__ballot(near_it) != 0) {   // cosines that fp32 does not tell apart
            nearest = {-__builtin_inf(), kNoClass};
#pragma unroll
            for (int i = 0; i < kA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = i * kTile + 8 * (r / 4) + 4 * half + r % 4;
                    nearest = better(nearest, Best{size[c] == 0.0 ? 0.0 : (double)acc[i][j][r] * value[c] / size[c], c});
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
        nearest = better(nearest, Best{__shfl_xor(nearest.cos, 32, kWave), __shfl_xor(nearest.c, 32, kWave)});
        if (half == 0 && n_of[j] < N) {
            const int c = nearest.c == kNoClass ? kNoClass : c0 + nearest.c;
            if (pred_out) {
                pred_out[n_of[j]] = c == kNoClass ? 0 : c;
            } else {
                best_cos[(int64_t)tc * N + n_of[j]] = nearest.cos;
                best_c[(int64_t)tc * N + n_of[j]] = c;
            }
        }
    }
}

}  // namespace

int64_t search_many_limits() { return 2 * kMost; }

// Whether a call goes this way, unless its rows' scales lie far apart: where the classes fill more than half of a block's (of its first: the
// rule does not look at how many are left for the last) and there are blocks for three of eight compute units.  us, so and by
// search_quantized_kernel; classes by samples of 10000 dimensions: 64 by 64000 (250 blocks) 67 47, 96 68 72, 128 67 91; 128 by 16000 (63) 60 41;
// 256 by 4000 (32) 59 36, by 16000 (126) 67 78; 1024 by 4000 (128) 66 124, by 64000 366 627.  Of 1000: 64 by 64000 28 19, 96 22 29, 128 29 36;
// 256 by 4000 21 20, by 16000 29 40, 1024 by 16000 37 147.
// Just past 128 the second block's classes are few, and the rule is wrong by up to a fifth, of calls of 16000 by a quarter: of 10000, 129 by
// 16000 63 49, by 64000 95 105, by 200000 309 260; 160 63 51, 97 107, 319 266; 192 63 60, 101 128, 321 313; 257 by 16000 67 84, by 200000 498
// 465; 320 507 526.  Of 1000, 129 by 400000 153 142, 192 152 178, 257 216 256.  96 by 200000 of 10000 179 173.
bool search_many_takes(const hdc_ctx_impl *c, int64_t N) {
    static_assert((int64_t)HDC_MAX_D / 32 * kUnit * kClasses < (int64_t)1 << 31, "places in a block's codes are of 32 bits");
    return c->p.C > kClasses / 2 && c->W >= kStep &&
           (N + kSamples - 1) / kSamples * ((c->p.C + kClasses - 1) / kClasses) >= c->num_cus * 3 / 8;
}

// One launch for samples that the scratch of the nearest classes has room for; *splits: classes' tiles, 1 if pred is written already.
int launch_search_many(hdc_ctx_impl *c, const uint32_t *hv, int64_t N, const uint32_t *codes, const uint8_t *scales, const double *norm, float *cos_out,
                       int32_t *pred, bool scan, int *splits, hipStream_t s) {
    const int tiles_c = (c->p.C + kClasses - 1) / kClasses, range = range_of(c->W);
    if (scan) hipLaunchKernelGGL(scan_kernel, dim3((unsigned)c->p.C), dim3(256), 0, s, codes, scales, c->W, range, c->qs_limits_d);
    const int64_t tiles_n = (N + kSamples - 1) / kSamples;
    *splits = tiles_c;
    hipLaunchKernelGGL(search_many_kernel, dim3((unsigned)((tiles_n + 7) / 8 * 8 * tiles_c)), dim3(kThreads), 0, s, hv, N, c->W, c->p.C, codes, scales, norm,
                       sqrt((double)c->p.D), c->qs_limits_d, range, cos_out, tiles_c == 1 ? pred : nullptr, c->qs_cos_d, c->qs_class_d);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

}  // namespace hdc
