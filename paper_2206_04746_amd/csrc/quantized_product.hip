// Products of rows of 4-bit floats with one another: out[m][n] = <a[m], b[n]>, on v_mfma_scale_f32_32x32x64_f8f6f4, which takes the
// codes and the scales as they are stored and sums in fp32.
//
// Many rows: tiles of a's rows by b's rows through LDS, 256 dimensions at a time (128 bytes a row, loaded straight into LDS), the next step's
// while a step's are multiplied; within a step a wave takes the operands of its next matrix instructions while it issues these.
// 8191 by 4093 rows of 9999: 219 us, 3.06 PFLOP/s.  Matrix instructions are 82 us of that (38 % of the active cycles, at the 2.1 GHz that they leave
// the chip): a step waits for its loads and reads of LDS, with which they overlap in part only.  Where a row is no whole number of
// cache lines loads take longer (8192 by 4096: of 9999 245, of 9984 187; without loads 175 and, without scales, too, 154).
// Few rows: a block takes 32 by 32 rows, or 16 by 16 (v_mfma_scale_f32_16x16x128_f8f6f4), its waves a share of the dimensions each, without LDS
// but for the sum over the waves.
#include <algorithm>
#include <type_traits>

#include "quantized.h"

namespace hdc {

namespace {

// Bytes [at, at + kBytes) of a row's scales as words; past the row's end those of 1.
template <int kBytes>
__device__ __forceinline__ void scale_bytes(const uint8_t *row, int at, int W, uint32_t (&out)[kBytes / 4]) {
    if (at + kBytes <= W) {
        __builtin_memcpy(out, row + at, kBytes);
    } else {
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) {
            uint32_t s[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] = row[min(at + 4 * i + k, W - 1)];
            out[i] = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) out[i] |= (at + 4 * i + k < W ? s[k] : kQuantZero) << 8 * k;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// ---- few rows: kSize of a by kSize of b a block, 32 or 16, a share of the dimensions to each of its waves
constexpr int kFewWaves = 8;

// A wave takes the blocks of 32 dimensions of four matrix instructions at a time, four adjacent ones a lane, and then those that are as many
// further on as the waves have.  Bound by the latency of its loads, 64 bytes of a row each.
template <int kSize>
__global__ __launch_bounds__(kFewWaves * kWave) void product_few_kernel(const uint32_t *__restrict__ a, const uint8_t *__restrict__ sa, int64_t M,
                                                                        const uint32_t *__restrict__ b, const uint8_t *__restrict__ sb, int64_t N, int W,
                                                                        float *__restrict__ out, int64_t pitch) {
    constexpr int kGroups = kWave / kSize, kPerUnit = 4 * kGroups;   // lanes to a row, blocks of four instructions
    __shared__ float sums[kFewWaves][kSize][kSize + 1];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, waves = blockDim.x >> 6, col = lane % kSize, group = lane / kSize;
    const int64_t m0 = (int64_t)blockIdx.y * kSize, n0 = (int64_t)blockIdx.x * kSize;
    const int64_t ra = min(m0 + col, M - 1) * W, rb = min(n0 + col, N - 1) * W;
    const v4u *const ca = reinterpret_cast<const v4u *>(a) + ra, *const cb = reinterpret_cast<const v4u *>(b) + rb;
    typename std::conditional<kSize == 32, v16f, v4f>::type acc = {};
    for (int u = wave * kPerUnit; u < W; u += waves * kPerUnit) {   // uniform
        const int first = u + 4 * group;
        v4u x[4], y[4];
        uint32_t sx[1], sy[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = first + i, in = min(w, W - 1);
            x[i] = ca[in], y[i] = cb[in];
            if (w >= W) x[i] = v4u{0, 0, 0, 0}, y[i] = v4u{0, 0, 0, 0};
        }
        scale_bytes<4>(sa + ra, first, W, sx);
        scale_bytes<4>(sb + rb, first, W, sy);
        acc = mfma<0>(x[0], y[0], acc, sx[0], sy[0]);
        acc = mfma<1>(x[1], y[1], acc, sx[0], sy[0]);
        acc = mfma<2>(x[2], y[2], acc, sx[0], sy[0]);
        acc = mfma<3>(x[3], y[3], acc, sx[0], sy[0]);
    }
#pragma unroll
    for (int j = 0; j < kSize * kSize / kWave; ++j) sums[wave][4 * kGroups * (j / 4) + 4 * group + j % 4][col] = acc[j];
    __syncthreads();
    for (int at = tid; at < kSize * kSize; at += blockDim.x) {
        const int r = at / kSize, k = at % kSize;
        double sum = 0.0;   // of the waves' fp32 sums, rounded once
        for (int w = 0; w < waves; ++w) sum += (double)sums[w][r][k];
        if (m0 + r < M && n0 + k < N) out[(m0 + r) * pitch + n0 + k] = (float)sum;
    }
}

// ---- many rows: a tile of 64 kA rows of a by 64 kB of b a block, or each of its groups, of two by two waves
constexpr int kThreads = 256, kStep = 8, kUnit = 16;   // blocks of 32 dimensions a step, bytes of one

// The sums of a tile are computed here, and not past the next barrier: operands take the registers of those that have been multiplied.
// (Sixteen tiles a wave take all of the accumulation registers.)
template <bool kAccumulators>
__device__ __forceinline__ v16f settled(v16f v) {
    if constexpr (kAccumulators)
        asm volatile("" : "+a"(v));
    else
        asm volatile("" : "+v"(v));
    return v;
}

// Steps of 256 dimensions.  While a step's matrix instructions are issued, four groups of kA kB, the operands of each next group are read
// from LDS and, once all of the step's are in registers, the step after next is asked for in its place: all of it a piece to a
// matrix instruction, so that these follow one another without a pause.  W >= 2 kStep.
//
// kSplit > 1: the dimensions are shared out to as many groups of four waves, whose sums meet in LDS.
template <int kA, int kB, int kSplit>
__global__ __launch_bounds__(kThreads *kSplit, kA * kB > 4 ? 1 : 2) void product_tiles_kernel(const uint32_t *__restrict__ a, const uint8_t *__restrict__ sa, int64_t M,
                                                                                      const uint32_t *__restrict__ b, const uint8_t *__restrict__ sb,
                                                                                      int64_t N, int W, int tiles_m, int tiles_n, float *__restrict__ out) {
    constexpr int kRowsA = 64 * kA, kRowsB = 64 * kB, kRows = kRowsA + kRowsB;
    constexpr int kOwn = (kRows + kThreads - 1) / kThreads, kLoads = kRows / 32, kPer = kLoads / (kA * kB);   // rows whose scales a thread brings; loads of a step, and to a matrix instruction
    static_assert(kLoads % (kA * kB) == 0 && kA + kB <= 2 * kA * kB, "pieces to a matrix instruction");
    // Codes of a step and of the next: block k of a row's eight is at place k ^ (row / 2 % 8) of the row, so that sixteen rows' blocks lie in
    // different banks.  Scales of two steps and of the next two.
    __shared__ __align__(16) uint32_t units[kSplit][2][kRows * kStep * 4];
    __shared__ uint32_t scales[kSplit][2][4][kRows];
    const int part = kSplit > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads) : 0;
    uint32_t(*const unit)[kRows * kStep * 4] = units[part];
    uint32_t(*const scale)[4][kRows] = scales[part];
    const int tid = kSplit > 1 ? threadIdx.x % kThreads : threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;

    // Blocks of consecutive numbers go to the eight dies in turn: a die takes tiles that lie together, eight rows of tiles wide.
    int tm, tn;
    {
        const int all = tiles_m * tiles_n, die = blockIdx.x % 8, per = all / 8, more = all % 8;
        const int at = die * per + min(die, more) + blockIdx.x / 8;
        const int band = at / (8 * tiles_n), high = min(8, tiles_m - band * 8), in = at - band * 8 * tiles_n;
        tm = __builtin_amdgcn_readfirstlane(band * 8 + in % high), tn = __builtin_amdgcn_readfirstlane(in / high);
    }
    const int64_t m0 = (int64_t)tm * kRowsA, n0 = (int64_t)tn * kRowsB;
    const int rows_a = (int)min((int64_t)kRowsA, M - m0), rows_b = (int)min((int64_t)kRowsB, N - n0);
    const uint32_t pitch = (uint32_t)W * kUnit;
    // A group's steps: an even number if there are several groups, so that none begins between two steps whose scales come together.
    const int all = (W + kStep - 1) / kStep, steps = kSplit > 1 ? (all + 2 * kSplit - 1) / (2 * kSplit) * 2 : all, first = part * steps;
    const LdsSource from_a = lds_source(a + m0 * W * 4, (uint32_t)rows_a * pitch), from_b = lds_source(b + n0 * W * 4, (uint32_t)rows_b * pitch);

    // A step's blocks, or the row's last eight: those that the step before has had are zeros then.
    auto begin_of = [&](int step) { return min(step * kStep, W - kStep); };
    // A wave's load fills eight rows of 128 bytes; rows past the last are taken from it.
    uint32_t offset[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = i * 32 + wave * 8 + (lane >> 3);
        offset[i] = (uint32_t)(i * 32 < kRowsA ? min(r, rows_a - 1) : min(r - kRowsA, rows_b - 1)) * pitch + ((lane & 7) ^ ((wave & 1) * 4 + (lane >> 4))) * kUnit;
    }
    auto load = [&](int i, uint32_t *to, uint32_t begin) {
        load_lds(i * 32 < kRowsA ? from_a : from_b, offset[i], begin * kUnit, to + (i * 32 + wave * 8) * kStep * 4);
    };
    const uint8_t *own[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int r = tid + i * kThreads;
        own[i] = r < kRowsA ? sa + (m0 + min(r, rows_a - 1)) * W : sb + (n0 + min(r - kRowsA, rows_b - 1)) * W;
    }
    // The scales of two steps are sixteen bytes, or the row's last sixteen.
    auto pair_of = [&](int step) { return min(step * kStep, W - 2 * kStep); };
    uint32_t piece[kOwn][4];
    auto ask_scales = [&](int step) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) __builtin_memcpy(piece[i], own[i] + pair_of(step), 16);
    };
    auto put_scales = [&](int to) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (kRows % kThreads == 0 || tid + i * kThreads < kRows) scale[to][j][tid + i * kThreads] = piece[i][j];
    };

    const int wm = (wave >> 1) * 32 * kA, wn = kRowsA + (wave & 1) * 32 * kB;   // this wave's rows
    v16f acc[kA][kB] = {};
    v4u x[2][kA], y[2][kB];           // operands of a group of matrix instructions, and of the next
    uint32_t sx[2][kA], sy[2][kB];    // scales of a step, and of the next
    const uint32_t *const codes_x = unit[0] + (wm + col) * kStep * 4, *const codes_y = unit[0] + (wn + col) * kStep * 4;
    auto take = [&](int buffer, int t, int i) {   // the i-th operand of group t
        const int place = buffer * kRows * kStep * 4 + ((4 * half + t) ^ (col >> 1 & 7)) * 4;
        if (i < kA) x[t & 1][i] = *reinterpret_cast<const v4u *>(codes_x + place + i * 32 * kStep * 4);
        else if (i < kA + kB) y[t & 1][i - kA] = *reinterpret_cast<const v4u *>(codes_y + place + (i - kA) * 32 * kStep * 4);
    };
    auto take_scales = [&](int step, int to) {
        const int at = begin_of(step) - pair_of(step & ~1) + 4 * half;   // the first of this lane's four bytes among the sixteen
        const uint32_t(*const from)[kRows] = &scale[step / 2 & 1][at >> 2];
#pragma unroll
        for (int i = 0; i < kA; ++i) sx[to][i] = from[0][wm + i * 32 + col];
#pragma unroll
        for (int i = 0; i < kB; ++i) sy[to][i] = from[0][wn + i * 32 + col];
        if (at & 3) {   // (of the last steps, by the same for all lanes: the next word is one of the four)
#pragma unroll
            for (int i = 0; i < kA; ++i) sx[to][i] = __builtin_amdgcn_alignbyte(from[1][wm + i * 32 + col], sx[to][i], at & 3);
#pragma unroll
            for (int i = 0; i < kB; ++i) sy[to][i] = __builtin_amdgcn_alignbyte(from[1][wn + i * 32 + col], sy[to][i], at & 3);
        }
    };
    // A group of matrix instructions, with meanwhile(i) after the i-th.
    auto multiply = [&](auto t_of, int step, auto meanwhile) {
        constexpr int t = decltype(t_of)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kA; ++i)
#pragma unroll
            for (int j = 0; j < kB; ++j) {
                acc[i][j] = mfma<t>(x[t & 1][i], y[t & 1][j], acc[i][j], sx[step][i], sy[step][j]);
                meanwhile(i * kB + j);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
        for (int i = 0; i < kA; ++i)
#pragma unroll
            for (int j = 0; j < kB; ++j) acc[i][j] = settled<(kA * kB > 8)>(acc[i][j]);
    };
    // What a wave has asked for in LDS is there, for every wave, and what was there has been read by all.  (A barrier by itself does not wait for
    // loads into LDS.)
    auto meet = [&](int step) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int again = step * kStep - begin_of(step);   // blocks that the step before has had: of the last step, and past it
        const int latest = step + (kSplit - 1 - part) * steps;
        if (latest * kStep > begin_of(latest)) {           // for all of the block's threads or none, the last group's
            for (int u = tid; u < kRows * kStep; u += kThreads)
                if (((u & 7) ^ (u >> 4 & 7)) < again) *reinterpret_cast<v4u *>(unit[step & 1] + u * 4) = v4u{0, 0, 0, 0};
            __syncthreads();
        }
    };
    // Step k, in buffer `odd`; what follows the row's last step is asked for and read as well, and not used.
    auto go = [&](int k, auto odd_of) {
        constexpr int odd = decltype(odd_of)::value;
        const int chunk = k / 2 & 1;
        if (!odd) ask_scales(k + 2);
        multiply(std::integral_constant<int, 0>{}, odd, [&](int i) { take(odd, 1, i), i + kA * kB < kA + kB ? take(odd, 1, i + kA * kB) : (void)0; });
        multiply(std::integral_constant<int, 1>{}, odd, [&](int i) { take(odd, 2, i), i + kA * kB < kA + kB ? take(odd, 2, i + kA * kB) : (void)0; });
        multiply(std::integral_constant<int, 2>{}, odd, [&](int i) { take(odd, 3, i), i + kA * kB < kA + kB ? take(odd, 3, i + kA * kB) : (void)0; });
        if (odd) put_scales(chunk ^ 1);
        meet(k + 1);
        const uint32_t begin = (uint32_t)begin_of(k + 2);
        take_scales(k + 1, odd ^ 1);
        multiply(std::integral_constant<int, 3>{}, odd, [&](int i) {
            take(odd ^ 1, 0, i), i + kA * kB < kA + kB ? take(odd ^ 1, 0, i + kA * kB) : (void)0;
#pragma unroll
            for (int l = 0; l < kPer; ++l) load(i * kPer + l, unit[odd], begin);
        });
    };

    ask_scales(first);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(i, unit[0], (uint32_t)begin_of(first));
    put_scales(first / 2 & 1);
    meet(first);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(i, unit[1], (uint32_t)begin_of(first + 1));
    take_scales(first, 0);
#pragma unroll
    for (int i = 0; i < kA + kB; ++i) take(0, 0, i);
    for (int k = first; k < first + steps; k += 2) {   // (a step past the last is one of zeros)
        go(k, std::integral_constant<int, 0>{});
        go(k + 1, std::integral_constant<int, 1>{});
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing may be on its way into LDS when the block's is given to another)
    if constexpr (kSplit > 1) {
        constexpr int kRow = 64 * kB;
        static_assert(kRowsA * kRow <= 2 * kRows * kStep * 4, "a group's sums take its codes' place");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kA; ++i)
#pragma unroll
            for (int j = 0; j < kB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    reinterpret_cast<float *>(unit[0])[(wm + i * 32 + 8 * (r / 4) + 4 * half + r % 4) * kRow + wn - kRowsA + j * 32 + col] = acc[i][j][r];
        __syncthreads();
        for (int at = threadIdx.x; at < kRowsA * kRow; at += kThreads * kSplit) {
            const int row = at / kRow, n = at % kRow;
            double sum = 0.0;   // of the groups' fp32 sums, rounded once
#pragma unroll
            for (int q = 0; q < kSplit; ++q) sum += (double)reinterpret_cast<const float *>(units[q])[at];
            if (row < rows_a && n < rows_b) out[(m0 + row) * N + n0 + n] = (float)sum;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kA; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = wm + i * 32 + 8 * (r / 4) + 4 * half + r % 4;
            if (row >= rows_a) continue;
            float *const to = out + (m0 + row) * N + n0;
#pragma unroll
            for (int j = 0; j < kB; ++j) {
                const int n = wn - kRowsA + j * 32 + col;
                if (n < rows_b) to[n] = acc[i][j][r];
            }
        }
}

}  // namespace

int launch_product_quantized(hdc_ctx_impl *c, const uint32_t *a, const uint8_t *sa, int64_t M, const uint32_t *b, const uint8_t *sb, int64_t N, float *out,
                             hipStream_t s) {
    ProfScope prof(c, HDC_K_PRODUCT_QUANTIZED, s);
    const int W = c->W;
    auto blocks = [&](int64_t size) { return ((M + size - 1) / size) * ((N + size - 1) / size); };
    // Few rows up to as many blocks as compute units, in 16 by 16 up to as many blocks of these; then tiles of 64 rows, two shares of the
    // dimensions a block, up to two blocks a unit (its LDS), tiles of 128 up to two, tiles of 256 beyond.  us a call:
    //   16 by 16 / 32 by 32: 64 by 64 rows of 9999 6.6 9.9, 1559 by 26 6.8 9.8 (196 blocks of 16 by 16), 96 by 1000 14.2 10.5 (378), 512 by 512
    //   21 13.5 (1024), of 16384 40 23
    //   32 by 32 / 64: 512 by 512 rows of 9999 13.7 17.7 (256 blocks of 32 by 32), 600 by 600 30 19 (361), 1000 by 1000 54 25, of 4096 22 10.4, of 1000
    //   9.1 7.1
    //   64 / 128: 1000 by 1000 rows of 9999 25 45 (256 blocks of 64), 1300 by 1300 35 45 (441), 1500 by 1500 58 46 (576), of 4096 22 17.6, of 1000
    //   11.9 9.8; in four shares 1000 by 1000 of 9999 24, 1300 by 1300 45
    //   128 / 256: 2000 by 2000 rows of 9999 50 86 (256 blocks of 128), 3000 by 3000 109 90 (576), of 1000 19.8 23.2, 4096 by 4096 of 9999 135 104
    if (blocks(32) <= c->num_cus || W < 2 * kStep) {
        auto launch = [&](auto kernel, int size) {
            const int per = 4 * kWave / size, waves = std::min((W + per - 1) / per, kFewWaves);
            const int64_t most = (int64_t)size << 22;   // rows of b a launch, whose threads along x are fewer than 2^32 then
            for (int64_t m = 0; m < M; m += (int64_t)size * 65535)
                for (int64_t n = 0; n < N; n += most) {
                    const int64_t rows = std::min<int64_t>(M - m, (int64_t)size * 65535), cols = std::min(N - n, most);
                    hipLaunchKernelGGL(kernel, dim3((unsigned)((cols + size - 1) / size), (unsigned)((rows + size - 1) / size)), dim3((unsigned)waves * kWave), 0, s,
                                       a + m * W * 4, sa + m * W, rows, b + n * W * 4, sb + n * W, cols, W, out + m * N + n, N);
                }
        };
        if (blocks(16) <= c->num_cus)
            launch(product_few_kernel<16>, 16);
        else
            launch(product_few_kernel<32>, 32);
    } else {
        auto launch = [&](auto kernel, int size, int split) {
            const int64_t tiles_m = (M + size - 1) / size, tiles_n = (N + size - 1) / size;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles_m * tiles_n)), dim3(kThreads * split), 0, s, a, sa, M, b, sb, N, W, (int)tiles_m, (int)tiles_n, out);
        };
        if (blocks(64) <= 2 * (int64_t)c->num_cus)
            launch(product_tiles_kernel<1, 1, 2>, 64, 2);
        else if (blocks(128) <= 2 * (int64_t)c->num_cus)
            launch(product_tiles_kernel<2, 2, 1>, 128, 1);
        else
            launch(product_tiles_kernel<4, 4, 1>, 256, 1);
    }
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

}  // namespace hdc
