// Cosine inference with class rows of 4-bit floats (arXiv 2206.04746, Sec. III), and the dot products of online training with them.
//
// The matrix cores take such rows as they are, with their scales (v_mfma_scale_f32_32x32x64_f8f6f4), and a sample's bits as +-1 in the
// same format.  A block of eight waves takes 32 classes, or the model's up to 16, and walks over the samples, 32 at a time; each wave has
// an eighth of the dimensions and holds the codes of its classes there in registers, so that all there is to read on the way is the
// samples, once.  The waves' parts of the dot products meet in LDS.  Where a row is short and samples are many, four, two or one of
// the waves hold it, and the block takes two, four or eight times 32 samples at once, for one barrier and with fewer lanes a sample at the end.
// 200000 samples of 10000 dimensions, 26 classes: 64 us (3.9 TB/s of words), with the launch 67; 1000000 of 1000: 51, with cosines 83.
//
// Sums without rounding: the products of a row are whole multiples of half its smallest scale, and a block of 32 dimensions gives at
// most 192 (32 times 6) of the largest.  Where a row's scales lie no further apart than 2^kRange, sums over it fit the 24 bits of
// fp32, the waves' and theirs together.  Where they lie further apart, the blocks are taken in several passes, each of the scales
// that lie within such a range, and the passes are added in fp64.  (us, rows of
// normal values, and with blocks up to 2^12 and 2^24 smaller: 200000 samples of 10000, 26 classes 61 132 211; 1000000 of 1000 46 125
// 150; 16001 of 8191, 1024 classes, which go by the other kernel only as the first, 86 415 605.)
#include <algorithm>
#include <type_traits>

#include "online_weight.h"
#include "quantized.h"

namespace hdc {

namespace {

constexpr int kWaves = 8, kThreads = kWaves * kWave, kTile = 32;   // samples; most classes of a block
constexpr int kMaxTiles = 32;                                      // of samples a block walks over once for every group of classes



// The best of a row of 16 lanes, in each of them: neighbours, their neighbours, halves of eight, halves of the row.
template <int kSel>
__device__ __forceinline__ Best of_lane(Best b) {
    auto from = [](int v) { return __builtin_amdgcn_update_dpp(0, v, kSel, 0xF, 0xF, true); };
    return {__hiloint2double(from(__double2hiint(b.cos)), from(__double2loint(b.cos))), from(b.c)};
}
__device__ __forceinline__ Best best_of_16(Best b) {
    b = better(b, of_lane<0xB1>(b));
    b = better(b, of_lane<0x4E>(b));
    b = better(b, of_lane<0x141>(b));
    return better(b, of_lane<0x140>(b));
}

__device__ __forceinline__ double sum_of_16(double v) {
    auto from = [](double x, auto sel) {
        constexpr int kSel = decltype(sel)::value;
        return __hiloint2double((int)lanes<kSel>((uint32_t)__double2hiint(x)), (int)lanes<kSel>((uint32_t)__double2loint(x)));
    };
    v += from(v, std::integral_constant<int, kNext>{});
    v += from(v, std::integral_constant<int, kNextPair>{});
    v += from(v, std::integral_constant<int, kMirrorEight>{});
    return v + from(v, std::integral_constant<int, kMirrorRow>{});
}

// kShare waves hold a row.  grid (runs of `tiles` tiles of samples, a multiple of kWaves / kShare; splits of the groups of classes).
//   kNearest  cos_out (or null) takes the cosines, and the nearest class of a block's own goes to pred_out or, if that is null, to best_cos and
//             best_c [split][N]
//   kDots     part[n][C] takes the dot products
//   kWeights  up to 32 classes: the weights of online training (`weigh`); the last weigh.tblocks blocks transpose the samples' bits
enum Mode { kNearest, kDots, kWeights };
template <int kClasses, int kSteps, int kShare, bool kParts, int kMode>
__global__ __launch_bounds__(kThreads, 2) void search_quantized_kernel(const uint32_t *__restrict__ hv, int64_t N, int W, int C,
                                                                       const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                                       const double *__restrict__ norm, double root_d, int tiles, int groups,
                                                                       double *__restrict__ part, float *__restrict__ cos_out,
                                                                       int32_t *__restrict__ pred_out, double *__restrict__ best_cos, int *__restrict__ best_c,
                                                                       QuantWeights weigh, const int *__restrict__ wide) {
    constexpr int kPieces = kWave / kClasses, kCols = kTile / kClasses, kOwn = kClasses / 16;   // lanes to a row; rows of samples to a lane; classes of a thread
    constexpr int kBlocks = kShare * kPieces * kSteps, kRange = range_of(kBlocks);              // of a row at a time
    constexpr int kAtOnce = kWaves / kShare;                                                    // tiles of samples
    static_assert(kShare == kWaves || (!kParts && kMode == kNearest), "shares of short rows");
    typedef typename std::conditional<kClasses == 32, v16f, v4f>::type Sums;
    constexpr int kPitch = kTile + 4;                                          // (sixteen classes by four samples lie in different banks)
    __shared__ float sums[2][kWaves][kTile][kPitch];
    __shared__ int limits[2][kWaves][kTile];                    // largest and smallest scale of a class in a wave's dimensions
    __shared__ double run_cos[kMode == kNearest ? kMaxTiles * kTile : kTile];   // the nearest of the groups before; kWeights: norms of the classes
    __shared__ int run_c[kMode == kNearest ? kMaxTiles * kTile : 1];
    __shared__ double class_unit[kAtOnce > 1 ? kClasses : 1], class_size[kAtOnce > 1 ? kClasses : 1];   // unit and size by class of a group
    __shared__ double ratio[kAtOnce > 1 ? kClasses : 1];        // unit by size, or 0
    __shared__ float about[kAtOnce > 1 ? kClasses : 1];         // ... in fp32, no number for a class past the last
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, col = lane % kClasses, piece = lane / kClasses;
    if constexpr (kMode == kWeights) {
        const int idx = (int)blockIdx.x - ((int)gridDim.x - weigh.tblocks);
        if (blockIdx.x == 0 && tid == 0 && weigh.reset) *weigh.reset = 0;
        if (idx >= 0) {
            static_assert(sizeof(TransposeTile) <= sizeof(sums), "the tile takes the sums' place");
            transpose_tile<kThreads>(reinterpret_cast<TransposeTile &>(sums), idx, hv, N, W, weigh.G, weigh.colmask, weigh.ld, weigh.gw);
            return;
        }
    }
    if constexpr (kMode == kNearest) {   // the call's other kernel has taken it, unless a row's scales lie far apart
        if (wide) {
            int any = 0;
            for (int c = tid; c < C; c += kThreads) any |= wide[c];
            if (!__syncthreads_or(any)) return;
        }
    }
    const int64_t all = kMode == kWeights ? weigh.ld / kTile : (N + kTile - 1) / kTile, tile0 = (int64_t)blockIdx.x * tiles;
    const int count = (int)((min((int64_t)tiles, all - tile0) + kAtOnce - 1) / kAtOnce), parts = kParts ? (W + kBlocks - 1) / kBlocks : 1;
    const int g0 = blockIdx.y * groups, g1 = min(g0 + groups, (C + kClasses - 1) / kClasses);
    const bool several = kMode == kNearest && (g1 - g0 > 1 || !pred_out);   // groups whose nearest classes are compared

    v4u code[kSteps];
    uint32_t scale[kSteps / 4];   // a byte a step, less `top` (modulo 2^32, all four together): 127 for the row's largest
    int top = 0, passes = 1;      // the row's largest scale less 127; passes that the block needs
    double unit[kOwn], size[kOwn];   // of this thread's classes: the largest scale; the row's norm times that of a sample
    const int n_of = tid >> 4, c_of = tid & 15;   // this thread's sample of a tile, and the first of its classes, which are 16 apart
    constexpr int kAhead = !kParts && kSteps <= 20 ? 1 : 0;   // words of the next sample asked for before this one's products, or after them
    uint32_t word[1 + kAhead][kCols][kSteps];

    // This wave's tile of those at once, and its share of the row: of part z its blocks are those from share_of(z) on.  Step t has block kPieces
    // (t & ~3) + 4 piece + t % 4 from there, a load of four words is 16 kPieces bytes of kClasses rows; where the row ends before, the
    // row's last four, so that loads need no limits, with codes of zero for those that are not theirs.  (Rows shorter than that: one by one.)
    const int tile = wave / kShare, share = wave % kShare;
    const bool whole = W >= 4;
    auto share_of = [&](int z) { return z * kBlocks + share * kPieces * kSteps; };
    // Words of sample tile i in part z of the row.
    auto ask = [&](int i, int z, uint32_t(&to)[kCols][kSteps]) {
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
            const int64_t n = min((tile0 + i * kAtOnce + tile) * kTile + kClasses * k + col, N - 1);
            const uint32_t *const from = hv + n * W;
            if (whole) {
                const int w0 = share_of(z) + 4 * piece;
#pragma unroll
                for (int t = 0; t < kSteps; t += 4) __builtin_memcpy(&to[k][t], from + min(w0 + kPieces * t, W - 4), 16);
            } else {
                const int here = anew(share * kPieces * kSteps + 4 * piece);   // (no places in the row are kept)
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    to[k][t] = from[min(here + kPieces * (t & ~3) + t % 4, W - 1)];
                    if (t % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (not all addresses at once)
                }
            }
        }
    };
    // This wave's codes of a group of classes in part z; meanwhile() is done while they are on their way.  (Classes past the last are that one
    // again.)
    auto hold = [&](int group, int z, auto meanwhile) {
        const int w0 = share_of(z);
        const int64_t from = anew((int64_t)min(group * kClasses + col, C - 1) * W);
        const v4u *const here = reinterpret_cast<const v4u *>(codes) + from;
        if (whole) {
            const int first = w0 + 4 * piece;
#pragma unroll
            for (int t = 0; t < kSteps; t += 4) __builtin_memcpy(&scale[t / 4], scales + from + min(first + kPieces * t, W - 4), 4);
#pragma unroll
            for (int t = 0; t < kSteps; ++t) code[t] = here[min(first + kPieces * (t & ~3), W - 4) + t % 4];
            if (w0 + kPieces * kSteps > W) {   // blocks before a step's own are another's
                const int place = anew(first);
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const int own = place + kPieces * (t & ~3);
                    const bool mine = min(own, W - 4) + t % 4 >= own;
#pragma unroll
                    for (int r = 0; r < 4; ++r) code[t][r] = mine ? code[t][r] : 0u;
                    scale[t / 4] &= mine ? ~0u : ~(255u << 8 * (t & 3));
                }
            }
        } else {
            const int begin = anew(w0 + 4 * piece);
            uint32_t s[kSteps];
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                const int w = min(begin + kPieces * (t & ~3) + t % 4, W - 1);
                s[t] = scales[from + w];
                code[t] = here[w];
                if (t % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (not all addresses at once)
            }
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                const bool in = begin + kPieces * (t & ~3) + t % 4 < W;
                scale[t / 4] = (t % 4 ? scale[t / 4] : 0u) | (in ? s[t] : 0u) << 8 * (t % 4);
#pragma unroll
                for (int r = 0; r < 4; ++r) code[t][r] = in ? code[t][r] : 0u;
            }
        }
        meanwhile();
        // Blocks of zeros, whose scale is 0 and may lie far from the others', count for nothing.
        uint32_t zeros = 0;
#pragma unroll
        for (int t = 0; t < kSteps; t += 4) zeros |= (scale[t / 4] - 0x01010101u) & ~scale[t / 4] & 0x80808080u;
        if (__ballot(zeros != 0) != 0) {
            zeros = 0;
#pragma unroll
            for (int t = 0; t < kSteps; ++t)
                if ((scale[t / 4] >> 8 * (t & 3) & 255) == 0 && ((code[t][0] | code[t][1] | code[t][2] | code[t][3]) & 0x77777777u) == 0) zeros |= 1u << t;
        }
        int most = -1, least = 256;
#pragma unroll
        for (int t = 0; t < kSteps; ++t) {
            const int s = scale[t / 4] >> 8 * (t & 3) & 255;
            most = max(most, zeros >> t & 1 ? -1 : s);
            least = min(least, zeros >> t & 1 ? 256 : s);
        }
#pragma unroll
        for (int off = kClasses; off < kWave; off <<= 1) {
            most = max(most, __shfl_xor(most, off, kWave));
            least = min(least, __shfl_xor(least, off, kWave));
        }
        __syncthreads();   // what is written here has been read
        if (piece == 0) limits[0][wave][col] = most, limits[1][wave][col] = least;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kShare; ++w) most = max(most, limits[0][w][col]), least = min(least, limits[1][w][col]);
        passes = most < 0 || most == kQuantNone ? 1 : (most - least) / (kRange + 1) + 1;   // (of a row that is no number, any)
        for (int off = 1; off < kClasses; off <<= 1) passes = max(passes, __shfl_xor(passes, off, kWave));
        passes = __builtin_amdgcn_readfirstlane(passes);
        if (__ballot(zeros != 0) != 0) {   // blocks of zeros as the largest
#pragma unroll
            for (int t = 0; t < kSteps; ++t) scale[t / 4] |= (zeros >> t & 1 ? (uint32_t)max(most, 0) : 0u) << 8 * (t & 3);
        }
        top = most - kQuantZero;
#pragma unroll
        for (int t = 0; t < kSteps; t += 4) scale[t / 4] -= 0x01010101u * (uint32_t)top;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            int largest = -1;
#pragma unroll
            for (int w = 0; w < kShare; ++w) largest = max(largest, limits[0][w][c_of + 16 * j]);
            unit[j] = largest < 0 ? 1.0 : scale_value(largest);
        }
    };

    // This wave's part of a tile's dot products, where the codes need one pass.
    auto multiply = [&](Sums(&acc)[kCols]) {
#pragma unroll
        for (int k = 0; k < kCols; ++k) acc[k] = Sums{};
#pragma unroll
        for (int t = 0; t < kSteps; t += 4) {
#pragma unroll
            for (int k = 0; k < kCols; ++k) {
                acc[k] = mfma<0>(code[t], signs_of(word[0][k][t]), acc[k], scale[t / 4]);
                acc[k] = mfma<1>(code[t + 1], signs_of(word[0][k][t + 1]), acc[k], scale[t / 4]);
                acc[k] = mfma<2>(code[t + 2], signs_of(word[0][k][t + 2]), acc[k], scale[t / 4]);
                acc[k] = mfma<3>(code[t + 3], signs_of(word[0][k][t + 3]), acc[k], scale[t / 4]);
            }
            __builtin_amdgcn_sched_barrier(0);   // (not all signs at once: their registers)
        }
    };
    auto put = [&](int turn, const Sums(&acc)[kCols]) {
        float(*const to)[kPitch] = sums[turn][wave];
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
#pragma unroll
            for (int j = 0; j < kClasses * kClasses / kWave; ++j) to[4 * kPieces * (j / 4) + 4 * piece + j % 4][kClasses * k + col] = acc[k][j];
        }
    };
    auto sum_of = [&](int turn, int q, int j) {   // of tile q
        float sum = 0.0f;   // without rounding
#pragma unroll
        for (int w = 0; w < kShare; ++w) sum += sums[turn][q * kShare + w][c_of + 16 * j][n_of];
        return sum;
    };
    // The nearest of a group of classes for the block's sample `at`, which is n.
    auto keep = [&](int g, int at, int64_t n, Best best) {
        if (g > g0) best = better(Best{run_cos[at], run_c[at]}, best);
        if (g + 1 < g1) {
            run_cos[at] = best.cos, run_c[at] = best.c;
        } else if (n < N) {
            if (pred_out) {
                pred_out[n] = best.c == kNoClass ? 0 : best.c;
            } else {
                best_cos[(int64_t)blockIdx.y * N + n] = best.cos;
                best_c[(int64_t)blockIdx.y * N + n] = best.c;
            }
        }
    };
    auto finish = [&](int g, int i, const double(&total)[kOwn]) {
        const int c = g * kClasses + c_of;
        const int64_t n = (tile0 + i) * kTile + n_of;   // tile i of the block
        if constexpr (kMode == kDots) {
#pragma unroll
            for (int j = 0; j < kOwn; ++j)
                if (n < N && c + 16 * j < C) part[n * C + c + 16 * j] = total[j];
        } else if constexpr (kMode == kWeights) {   // (as finish_cosines and online_weights_kernel, online_batched.hip)
            const int y = n < N ? weigh.labels[n] : -1;
            const bool live = y >= 0 && y < C;
            Best best = {-2.0, kNoClass};   // cosines lie in [-1, 1]
            double mine = 0.0;
#pragma unroll
            for (int j = 0; j < kOwn; ++j)
                if (c + 16 * j < C) {
                    const double cs = size[j] == 0.0 ? 0.0 : total[j] / size[j];
                    best = better(best, Best{cs, c + 16 * j});
                    if (c + 16 * j == y) mine = cs;
                }
            best = best_of_16(best);
            const double cos_y = sum_of_16(mine);
            OnlineWeight r;
            r.y = live ? y : -1;
            r.pred = live && best.c != y ? best.c : -1;
            r.w_y = live ? (float)(1.0 - cos_y) : 0.0f;
            r.w_p = live ? (float)((double)weigh.lr * (1.0 - best.cos)) : 0.0f;
            if (n < N && c_of == 0) weigh.records[n] = r;
            if (weigh.coef)
                for (int j = c_of; j < weigh.cb; j += 16)
                    weigh.coef[n * weigh.cb + j] = j == r.y ? (double)r.w_y : j == r.pred ? -(double)r.w_p : 0.0;
        } else {
            Best best = {-__builtin_inf(), kNoClass};
#pragma unroll
            for (int j = 0; j < kOwn; ++j)
                if (c + 16 * j < C) {
                    const double cs = size[j] == 0.0 ? 0.0 : total[j] / size[j];
                    if (cos_out && n < N) cos_out[n * C + c + 16 * j] = (float)cs;
                    best = better(best, Best{cs, c + 16 * j});
                }
            best = best_of_16(best);
            if (c_of == 0) keep(g, i * kTile + n_of, n, best);
        }
    };
    // All of the tiles at once, for the nearest class with kLanes lanes a sample.  The class is the one that the quotients in fp64 give, which are
    // formed where fp32 does not tell them apart (its cosines are off by 2^-23 of themselves: the factor's rounding and the product's).
    // Cosines in the order in which they lie in memory, but for blocks of 32 classes that take two tiles (us, so and a tile at a time as where a
    // row has all waves: 26 classes, 1000000 samples of 1000 84 98, 300000 of 4096 - two tiles - 56 53; 20 classes, 400000 of 2000 46 51).
    constexpr int kLanes = 16 / kAtOnce;
    constexpr bool kLaidOut = kClasses == 16 || kAtOnce > 2;
    auto finish_all = [&](int g, int i) {
        const int64_t n0 = (tile0 + i * kAtOnce) * kTile;
        auto sum_at = [&](int at, int c) {
            float sum = 0.0f;   // without rounding
#pragma unroll
            for (int w = 0; w < kShare; ++w) sum += sums[i & 1][at / kTile * kShare + w][c][at % kTile];
            return sum;
        };
        auto quotient = [&](float sum, int c) { return class_size[c] == 0.0 ? 0.0 : (double)sum * class_unit[c] / class_size[c]; };
        if (kLaidOut && cos_out) {
            const int width = min(kClasses, C - g * kClasses), down = kThreads / width, right = kThreads % width;
            for (int at = tid / width, c = tid % width; at < kAtOnce * kTile; at += down) {
                if (n0 + at < N) cos_out[(n0 + at) * C + g * kClasses + c] = (float)((double)sum_at(at, c) * ratio[c]);
                c += right;
                if (c >= width) c -= width, ++at;
            }
        }
        const int at = tid / kLanes, lane_of = tid % kLanes;
        float most = -__builtin_inff(), second = -__builtin_inff(), sum_of_most = 0.0f;   // the two largest
        int which = kNoClass;
#pragma unroll 4
        for (int c = lane_of; c < kClasses; c += kLanes) {   // (what is no number is neither above nor below)
            const float sum = sum_at(at, c), v = sum * about[c];
            const bool above = v > most;
            second = above ? most : fmaxf(second, v);
            most = above ? v : most, which = above ? c : which, sum_of_most = above ? sum : sum_of_most;
        }
        auto join = [&](auto sel) {
            constexpr int kSel = decltype(sel)::value;
            const float other = __uint_as_float(lanes<kSel>(__float_as_uint(most)));
            const float sum = __uint_as_float(lanes<kSel>(__float_as_uint(sum_of_most)));
            const int c = (int)lanes<kSel>((uint32_t)which);
            second = fmaxf(fminf(most, other), fmaxf(second, __uint_as_float(lanes<kSel>(__float_as_uint(second)))));
            const bool above = other > most || (other == most && c < which);
            most = above ? other : most, which = above ? c : which, sum_of_most = above ? sum : sum_of_most;
        };
        if constexpr (kLanes > 1) join(std::integral_constant<int, kNext>{});
        if constexpr (kLanes > 2) join(std::integral_constant<int, kNextPair>{});
        if constexpr (kLanes > 4) join(std::integral_constant<int, kMirrorEight>{});
        Best best = {-__builtin_inf(), kNoClass};
        if (__builtin_expect(__ballot(second >= most * (1.0f - copysignf(0x1p-19f, most))) != 0, 0)) {
            for (int c = lane_of; c < kClasses && g * kClasses + c < C; c += kLanes) best = better(best, Best{quotient(sum_at(at, c), c), g * kClasses + c});
            if constexpr (kLanes > 1) best = better(best, of_lane<kNext>(best));
            if constexpr (kLanes > 2) best = better(best, of_lane<kNextPair>(best));
            if constexpr (kLanes > 4) best = better(best, of_lane<kMirrorEight>(best));
        } else if (which != kNoClass) {
            best = {several ? quotient(sum_of_most, which) : (double)most, g * kClasses + which};
        }
        if (lane_of == 0) keep(g, i * kAtOnce * kTile + at, n0 + at, best);
    };

    constexpr int kEarly = kMode == kWeights ? 16 : 1;   // partial norms asked for first
    double early[kEarly];
    if constexpr (kMode == kWeights) {
#pragma unroll
        for (int i = 0; i < kEarly; ++i) early[i] = weigh.normpart[(int64_t)min(n_of, C - 1) * weigh.G + min(c_of + 16 * i, weigh.G - 1)];
    }
    ask(0, 0, word[0]);
    for (int g = g0; g < g1; ++g) {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) size[j] = kMode == kNearest ? norm[min(g * kClasses + c_of + 16 * j, C - 1)] : 0.0;
        auto norms = [&]() {   // of the classes, sixteen lanes each
            if constexpr (kMode == kWeights) {
                double sum = 0.0;
#pragma unroll
                for (int i = 0; i < kEarly; ++i) sum += c_of + 16 * i < weigh.G ? early[i] : 0.0;
                for (int i = c_of + 16 * kEarly; i < weigh.G; i += 16) sum += weigh.normpart[(int64_t)min(n_of, C - 1) * weigh.G + i];
                sum = sum_of_16(sum);
                if (c_of == 0) run_cos[n_of] = sum;
            }
        };
        if constexpr (!kParts) hold(g, 0, norms);
        if constexpr (kMode == kWeights) {
            if constexpr (kParts) {
                norms();
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < kOwn; ++j) size[j] = run_cos[c_of + 16 * j];
        }
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            size[j] = sqrt(size[j]) * root_d;
            if (kAtOnce > 1 && n_of == 0) {
                const int c = c_of + 16 * j;
                class_unit[c] = unit[j], class_size[c] = size[j], ratio[c] = size[j] == 0.0 ? 0.0 : unit[j] / size[j];
                about[c] = g * kClasses + c < C ? (float)ratio[c] : __builtin_nanf("");
            }
        }
        if constexpr (!kParts) {
            if (__builtin_expect(passes == 1, 1)) {
                // A tile is finished while the next one's products are formed, by half of the waves before and by the other half after their own:
                // of the two waves that share a SIMD one multiplies while the other adds.
                const int one = anew(1);   // (no loop of its own for the first tile)
                for (int i = 0; i <= count; ++i) {
                    auto before = [&]() {
                        if (kAtOnce > 1 && (kLaidOut || !cos_out)) {
                            finish_all(g, i - 1);
                            return;
                        }
#pragma unroll 1
                        for (int q = 0; q < kAtOnce; ++q) {
                            double total[kOwn];
#pragma unroll
                            for (int j = 0; j < kOwn; ++j) total[j] = (double)sum_of((i - 1) & 1, q, j) * unit[j];
                            finish(g, (i - 1) * kAtOnce + q, total);
                        }
                    };
                    if (i >= one && wave < kWaves / 2) before();
                    if (i < count) {
                        if constexpr (kAhead) ask(i + 1 < count ? i + 1 : 0, 0, word[kAhead]);
                        Sums acc[kCols];
                        multiply(acc);
                        put(i & 1, acc);
                        if constexpr (kAhead) {
#pragma unroll
                            for (int k = 0; k < kCols; ++k) {
#pragma unroll
                                for (int t = 0; t < kSteps; ++t) word[0][k][t] = word[kAhead][k][t];
                            }
                        } else {
                            ask(i + 1 < count ? i + 1 : 0, 0, word[0]);
                        }
                    }
                    if (i >= one && wave >= kWaves / 2) before();
                    if (i < count) __syncthreads();
                }
                continue;
            }
        }
        int turn = 0;
        for (int i = 0; i < count; ++i) {
            double total[kAtOnce][kOwn] = {};
            for (int z = 0; z < parts; ++z) {
                if constexpr (kParts) hold(g, z, []() {});
                double down = 1.0;
                for (int p = 0; p < passes; ++p) {   // the blocks whose scale is one of this pass's: from 2^-(kRange + 1) p of the largest on downwards
                    Sums acc[kCols] = {};
#pragma unroll
                    for (int k = 0; k < kCols; ++k) {   // (or all signs would be made before the loop)
#pragma unroll
                        for (int t = 0; t < kSteps; ++t) word[0][k][t] = anew(word[0][k][t]);
                    }
                    top = anew(top);
#pragma unroll
                    for (int t = 0; t < kSteps; ++t) {
                        const int of = (int)((scale[t / 4] + 0x01010101u * (uint32_t)top) >> 8 * (t & 3) & 255) - top + (kRange + 1) * p;
                        const uint32_t mine = of <= kQuantZero && of >= kQuantZero - kRange ? ~0u : 0u;
#pragma unroll
                        for (int k = 0; k < kCols; ++k) acc[k] = mfma<0>(code[t] & mine, signs_of(word[0][k][t]), acc[k], (uint32_t)of & mine);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    put(turn, acc);
                    __syncthreads();
#pragma unroll
                    for (int q = 0; q < kAtOnce; ++q)
#pragma unroll
                        for (int j = 0; j < kOwn; ++j) total[q][j] = fma((double)sum_of(turn, q, j), unit[j] * down, total[q][j]);
                    turn ^= 1;
                    down *= 1.0 / (2 << kRange);
                }
                const bool last = z + 1 == parts;
                ask(last ? (i + 1 < count ? i + 1 : 0) : i, last ? 0 : z + 1, word[0]);
            }
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) finish(g, i * kAtOnce + q, total[q]);
        }
    }
}

__global__ __launch_bounds__(256) void nearest_kernel(const double *__restrict__ best_cos, const int *__restrict__ best_c, int64_t N, int splits,
                                                      int32_t *__restrict__ pred) {
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    Best best = {best_cos[n], best_c[n]};
    for (int k = 1; k < splits; ++k) best = better(best, Best{best_cos[k * N + n], best_c[k * N + n]});
    pred[n] = best.c == kNoClass ? 0 : best.c;
}

// Classes of a block and the waves that share a row: for no more than 16 classes (v_mfma_scale_f32_16x16x128_f8f6f4) half of the loads and
// registers (2947 samples of 10000 with 6 classes 6.9 us a call, in a block for 32 7.7; a batch of 64 in training 8.5 us, 8.9).
// Rows that eight waves of either kind hold in four steps go in a block for 32 (batches of 32 samples of 1024, 5 classes: 10.4 us a batch, in a
// block for 16 10.8).
struct Form {
    int classes, share;
};
Form whole_block(const hdc_ctx_impl *c) { return {c->p.C > 16 || c->W <= 4 * kWaves * (kWave / 32) ? 32 : 16, kWaves}; }

template <int kMode>
void launch(hdc_ctx_impl *c, Form form, dim3 grid, hipStream_t s, const uint32_t *hv, int64_t N, const uint32_t *codes, const uint8_t *scales, const double *norm,
            int tiles, int groups, double *part, float *cos_out, int32_t *pred, double *best_cos, int *best_c, const QuantWeights &weigh = {}, const int *wide = nullptr) {
#define HDC_SEARCH(CLASSES, STEPS, SHARE, PARTS)                                                                                                             \
    hipLaunchKernelGGL((search_quantized_kernel<CLASSES, STEPS, SHARE, PARTS, kMode>), grid, dim3(kThreads), 0, s, hv, N, c->W, c->p.C, codes, scales, norm, \
                       sqrt((double)c->p.D), tiles, groups, part, cos_out, pred, best_cos, best_c, weigh, wide)
    // Steps of a wave: as many as a row needs, up to 20 or 28 (the registers); rows of more than that go in parts of 16.
    const int blocks = form.share * (kWave / form.classes), steps = ((c->W + blocks - 1) / blocks + 3) / 4 * 4;
    if constexpr (kMode == kNearest) {
#define HDC_SEARCH_SHORT(CLASSES)                                                                              \
    switch (form.share * 100 + std::max(steps, form.share == 1 ? 8 : 12)) {                                    \
        case 108: HDC_SEARCH(CLASSES, 8, 1, false); break;                                                     \
        case 112: HDC_SEARCH(CLASSES, 12, 1, false); break;                                                    \
        case 116: HDC_SEARCH(CLASSES, 16, 1, false); break;                                                    \
        case 212: HDC_SEARCH(CLASSES, 12, 2, false); break;                                                    \
        case 216: HDC_SEARCH(CLASSES, 16, 2, false); break;                                                    \
        case 412: HDC_SEARCH(CLASSES, 12, 4, false); break;                                                    \
        default: HDC_SEARCH(CLASSES, 16, 4, false); break;                                                     \
    }
        if (form.share < kWaves) {
            if (form.classes == 16) {
                HDC_SEARCH_SHORT(16)
            } else {
                HDC_SEARCH_SHORT(32)
            }
            return;
        }
#undef HDC_SEARCH_SHORT
    }
    if constexpr (kMode != kDots) {   // (dot products of up to 32 classes become weights where they are formed)
        if (form.classes == 16) {
            switch (steps) {
                case 4: HDC_SEARCH(16, 4, 8, false); break;
                case 8: HDC_SEARCH(16, 8, 8, false); break;
                case 12: HDC_SEARCH(16, 12, 8, false); break;
                case 16: HDC_SEARCH(16, 16, 8, false); break;
                case 20: HDC_SEARCH(16, 20, 8, false); break;
                default: HDC_SEARCH(16, 16, 8, true); break;
            }
            return;
        }
    }
    switch (steps) {
        case 4: HDC_SEARCH(32, 4, 8, false); break;
        case 8: HDC_SEARCH(32, 8, 8, false); break;
        case 12: HDC_SEARCH(32, 12, 8, false); break;
        case 16: HDC_SEARCH(32, 16, 8, false); break;
        case 20: HDC_SEARCH(32, 20, 8, false); break;
        case 24: HDC_SEARCH(32, 24, 8, false); break;
        case 28: HDC_SEARCH(32, 28, 8, false); break;
        default: HDC_SEARCH(32, 16, 8, true); break;
    }
#undef HDC_SEARCH
}

// Many samples of short rows: a row to as few waves as hold it in 16 steps, so that a block has up to eight tiles of samples at once.  us,
// eight waves a row and so, nearest classes only; classes by samples of 1000 dimensions: 26 by 40000 (five tiles a compute unit) 11.4 10.5,
// by 65000 14.6 10.7, by 1000000 142 49 (with cosines 152 83), 6 by 1000000 128 39; of 4096: 26 by 50000 15.5 16.0, 10 by 300000 54 37;
// of 500: 26 by 1000000 137 38.  Longer rows of up to 16 classes in blocks of 32 while these hold them in 20 steps, with words ahead: a wave's
// share is not rounded up as far.  In blocks of 16 and of 32, 6 classes: 200000 of 8500 56 54, of 10000 62 58, of 10240 63 55; of 10400 57 80,
// 60000 of 12288 26 33, of 14336 31 33; in parts then, 60000 of 14400 30 82, of 20480 37 128.
Form form_of(const hdc_ctx_impl *c, int64_t tiles) {
    const int classes = c->p.C > 16 ? 32 : 16;
    if (tiles <= 6 * (int64_t)c->num_cus) return whole_block(c);
    for (int share = 1; share < kWaves; share *= 2)
        if (c->W <= share * (kWave / classes) * 16) return {classes, share};
    return c->W <= kWaves * (kWave / 32) * 20 ? Form{32, kWaves} : whole_block(c);
}

}  // namespace

// Entries of the scratch where the nearest classes of splits meet: kTile samples a compute unit here, where a launch has splits only while
// its tiles leave compute units idle; the other kernel takes as many samples at a time as there is room for.
int64_t search_quantized_entries(const hdc_ctx_impl *c) { return std::max<int64_t>((int64_t)kTile * c->num_cus, 1 << 18); }

static int launch_nearest(hdc_ctx_impl *c, int64_t N, int splits, int32_t *pred, hipStream_t s) {
    hipLaunchKernelGGL(nearest_kernel, dim3((unsigned)((N + 255) / 256)), dim3(256), 0, s, c->qs_cos_d, c->qs_class_d, N, splits, pred);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

// wide: null, or by class whether its scales lie far apart: if none's do, the call has been answered.
static int launch_search_few(hdc_ctx_impl *c, const uint32_t *hv, int64_t N, const uint32_t *codes, const uint8_t *scales, const double *norm,
                             float *cos_out, int32_t *pred, const int *wide, hipStream_t s) {
    const int groups = (c->p.C + kTile - 1) / kTile;   // (of 16 classes there is one)
    const int64_t tiles = (N + kTile - 1) / kTile, cus = c->num_cus;
    // One block a compute unit.  One group of classes: as many tiles as that gives a block; more groups: the block walks over its tiles
    // for each, and where there are fewer tiles than compute units, the groups are split among blocks.
    const Form form = form_of(c, tiles);
    const int at_once = kWaves / form.share;
    int64_t per = std::max<int64_t>(1, (tiles + cus - 1) / cus + at_once - 1) / at_once * at_once;
    if (groups > 1) per = std::min<int64_t>(per, kMaxTiles);
    const int splits_most = wide ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(groups, cus / tiles));
    const int of_split = (groups + splits_most - 1) / splits_most, splits = (groups + of_split - 1) / of_split;
    const int64_t blocks = (tiles + per - 1) / per, most = 1 << 22;   // blocks a launch
    for (int64_t b = 0; b < blocks; b += most) {
        const int64_t n0 = b * per * kTile, n = std::min(N - n0, most * per * kTile);
        launch<kNearest>(c, form, dim3((unsigned)std::min(most, blocks - b), (unsigned)splits), s, hv + n0 * c->W, n, codes, scales, norm, (int)per, of_split, nullptr,
                         cos_out ? cos_out + n0 * c->p.C : nullptr, splits > 1 ? nullptr : pred + n0, c->qs_cos_d, c->qs_class_d, {}, wide);
    }
    HDC_HIP(hipGetLastError());
    return splits > 1 ? launch_nearest(c, N, splits, pred, s) : HDC_OK;
}

int launch_search_quantized(hdc_ctx_impl *c, const uint32_t *hv, int64_t N, const uint32_t *codes, const uint8_t *scales, const double *norm,
                            float *cos_out, int32_t *pred, hipStream_t s) {
    ProfScope prof(c, HDC_K_SEARCH_QUANTIZED, s);
    if (search_many_takes(c, N)) {
        const int64_t most = search_quantized_entries(c) / ((c->p.C + 127) / 128) / 256 * 256;   // samples at a time
        for (int64_t n0 = 0; n0 < N; n0 += most) {
            const int64_t n = std::min(most, N - n0);
            float *const cos_of = cos_out ? cos_out + n0 * c->p.C : nullptr;
            int splits = 1;
            int rc = launch_search_many(c, hv + n0 * c->W, n, codes, scales, norm, cos_of, pred + n0, n0 == 0, &splits, s);
            if (rc == HDC_OK && splits > 1) rc = launch_nearest(c, n, splits, pred + n0, s);
            if (rc != HDC_OK) return rc;
        }
        return launch_search_few(c, hv, N, codes, scales, norm, cos_out, pred, c->qs_limits_d + search_many_limits() / 2, s);
    }
    return launch_search_few(c, hv, N, codes, scales, norm, cos_out, pred, nullptr, s);
}

int launch_quantized_dots(hdc_ctx_impl *c, const uint32_t *hv, int64_t nb, const uint32_t *codes, const uint8_t *scales, double *part, int *slices,
                          hipStream_t s) {
    ProfScope prof(c, HDC_K_ONLINE_FWD, s);
    *slices = 1;
    const int64_t tiles = (nb + kTile - 1) / kTile, groups = (c->p.C + kTile - 1) / kTile;
    const int64_t per = std::max<int64_t>(1, (tiles * groups + c->num_cus - 1) / c->num_cus);
    launch<kDots>(c, Form{32, kWaves}, dim3((unsigned)((tiles + per - 1) / per), (unsigned)groups), s, hv, nb, codes, scales, nullptr, (int)per, 1, part, nullptr, nullptr, nullptr,
                 nullptr);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

// Where a block has all classes of a sample.  us a batch of rows of 10000, so and by launch_quantized_dots with online_weights_kernel after it: 6
// classes, 64 samples 15.7 18.9, 1024 24.4 27.9, 4096 43 45, 32768 260 249; 26 classes 20.8 29.5, 29.7 37.6, 42.5 50.7, 269 275.
bool quantized_weights_takes(int C) { return C <= kTile; }

int launch_quantized_weights(hdc_ctx_impl *c, const uint32_t *hv, int64_t nb, const uint32_t *codes, const uint8_t *scales, const QuantWeights &out,
                             hipStream_t s) {
    ProfScope prof(c, HDC_K_ONLINE_FWD, s);
    const int64_t tiles = out.ld / kTile, per = std::max<int64_t>(1, (tiles + c->num_cus - 1) / c->num_cus);
    launch<kWeights>(c, whole_block(c), dim3((unsigned)((tiles + per - 1) / per + out.tblocks)), s, hv, nb, codes, scales, nullptr, (int)per, 1, nullptr, nullptr, nullptr,
                     nullptr, nullptr, out);
    HDC_HIP(hipGetLastError());
    return HDC_OK;
}

}  // namespace hdc
