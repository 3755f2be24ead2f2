// hb_linear and hb_linear_i8: which kernel a call takes and into how many parts the sum over k is split; host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace hb {

// How the rows of x and w stand in memory: at 16-byte addresses with K a multiple of 8, so that they can be copied to LDS directly; at
// 4-byte addresses; or at odd elements, too.
enum LinRows { kLinCopied, kLinEven, kLinOdd };

enum LinKernel { kLinRows16, kLinRows32, kLinRows64, kLinTile64, kLinTile128x64, kLinTile128, kLinTile256, kLinKernels };

// Most rows of x: the kernels number rows in 32 bits, up to the end of the last tile.
constexpr int kLinMostRows = 0x7fffff00;

struct LinPlan {
    LinKernel kernel;
    int parts, steps;             // of the sum, and steps of 64 k of one part
};

// The time of a call in us, as a model with a few constants per kernel: a workgroup alone on a compute unit takes `alone` a step and
// `begin` beside it, one of several `shared` and `end`; a kernel for few rows of x has its waves take turns at the steps.  `odd`:
// what rows at odd addresses add.  The constants were fitted to 1200 calls of random sizes (1 .. 2^20 x 16 .. 8192, K 16 ..
// 8192; fp16 output, no residual), each timed with every kernel and with 1 to 32 parts; `odd` of 64 x 64 was set anew when that kernel came to
// move its odd rows behind the products.  On 1200 other calls, of the kernels as they are now, the choice is on average 1.1 % behind the fastest.
// fp32 output and residuals are not in the model: with both of them it is 2.5 % behind, and up to 38 % where N is below 50.
struct LinCost {
    int m, n;                     // outputs of a workgroup
    int waves;                    // that share the steps; 0: tiles
    double alone, shared, begin, end, odd;
};
constexpr LinCost kLinCost[kLinKernels] = {
    {16, 16, 16, 0.749, 0.068, 0.00, 0.00, 0.91}, {32, 16, 8, 0.953, 0.135, 0.00, 0.00, 0.70}, {64, 16, 8, 1.447, 0.264, 0.00, 0.00, 0.32},
    {64, 64, 0, 0.353, 0.219, 1.29, 0.77, 0.40},  {128, 64, 0, 0.452, 0.358, 2.69, 1.55, 1.11}, {128, 128, 0, 0.528, 0.410, 1.63, 1.35, 0.00},
    {256, 256, 0, 0.744, 1.149, 9.12, 9.24, 0.00},
};
constexpr int kLinThreads[kLinKernels] = {1024, 512, 512, 512, 256, 512, 256};                // of a workgroup
// 64 x 64 copied to LDS directly, 128 x 128 through registers.  A call of one step has one stage of LDS, and more workgroups on a compute unit; only
// 128 x 64 gains by it, by kLinOneStep.  261 calls of K up to 64 took, in the median and in terms of the model without it, 0.81 (rows at even
// addresses) and 0.87 (odd) with 128 x 64, 1.00 and 1.05 with 64 x 64, 0.97 and 0.99 with 128 x 128, 0.95 with 256 x 256; the choice among them
// is 1.3 % behind the fastest with it, 2.9 % without (K from 65 to 128: 0.7 %).
constexpr LinCost kLinCostTile64Copied = {64, 64, 0, 0.240, 0.184, 0.27, 0.60, 0.00}, kLinCostTile128Held = {128, 128, 0, 0.802, 0.296, 2.45, 2.90, 0.34};
constexpr double kLinOneStep = 0.72;
constexpr double kLinLaunch = 2.5, kLinJoin = 2.58, kLinJoinPart = 0.28, kLinJoinRate = 6.9e6;      // us, us, us, bytes per us

// The same for one kind of operands; linear_cost() and linear_plan() take one of these.
struct LinCosts {
    LinCost of[kLinKernels], tile64_copied, tile128_held;
    double one_step, join, join_part, join_rate;
};
constexpr LinCosts kLinCostsF16 = {{kLinCost[0], kLinCost[1], kLinCost[2], kLinCost[3], kLinCost[4], kLinCost[5], kLinCost[6]}, kLinCostTile64Copied, kLinCostTile128Held,
                                   kLinOneStep, kLinJoin, kLinJoinPart, kLinJoinRate};
// 8-bit integers, a step being 128 k.  Fitted to 5000 calls of the same sizes with every kernel and number of parts, of a half with a residual and a third with fp32 output, as they were launched
// through ctypes (which no call is faster than; those under 6.3 us were left out).  On 4000 other calls the choice is 3.2 % behind the fastest in the mean, 2.8 % on those of 30 us and more, and 2.2 % with fp16
// output and no residual; with fp32 output and a residual, which the model leaves out, 6 %.  With the constants above it was 3.6, 5.4, 3.1 and 6 %.
constexpr LinCosts kLinCostsI8 = {{{16, 16, 16, 0.343, 0.062, 3.03, 0.00, 0.96}, {32, 16, 8, 0.459, 0.148, 2.83, 0.00, 0.81}, {64, 16, 8, 1.076, 0.276, 2.20, 0.00, 0.67},
                                   {64, 64, 0, 0.346, 0.292, 2.06, 1.21, 0.25}, {128, 64, 0, 0.699, 0.423, 2.29, 1.98, 0.52}, {128, 128, 0, 0.801, 0.538, 1.36, 2.42, 0.00},
                                   {256, 256, 0, 1.697, 1.664, 9.56, 13.95, 0.00}},
                                  {64, 64, 0, 0.257, 0.274, 2.16, 0.77, 0.00}, {128, 128, 0, 1.488, 0.998, 2.78, 2.61, 0.00}, 0.95, 1.39, 0.20, 5.6e6};

inline double linear_cost(LinKernel kernel, int64_t M, int64_t N, int parts, int steps, LinRows rows, const LinCosts& costs = kLinCostsF16) {
    const LinCost& c = kernel == kLinTile128 && rows != kLinCopied  ? costs.tile128_held
                       : kernel == kLinTile64 && rows == kLinCopied ? costs.tile64_copied
                                                                    : costs.of[kernel];
    const int64_t wgs = ((M + c.m - 1) / c.m) * ((N + c.n - 1) / c.n) * parts;
    const double slow = rows == kLinOdd ? 1.0 + c.odd : 1.0;
    double t;
    if (c.waves) {
        const double waves = (steps + c.waves - 1) / c.waves * c.alone, all = wgs / 256.0 * steps * c.shared;
        t = c.begin + (waves > all ? waves : all) * slow;
    } else {
        const double one = steps * c.alone * slow + c.begin, all = (double)((wgs + 255) / 256) * (steps * c.shared * slow + c.end);
        t = (one > all ? one : all) * (steps == 1 && kernel == kLinTile128x64 ? costs.one_step : 1.0);
    }
    if (parts > 1) t += costs.join + parts * costs.join_part + 8.0 * parts * M * N / costs.join_rate;
    return t + kLinLaunch;
}

inline LinPlan linear_plan(int M, int N, int K, LinRows rows, const LinCosts& costs = kLinCostsF16) {
    const int steps = (K - 1) / 64 + 1;
    LinPlan best = {kLinTile64, 1, steps};
    double least = 0.0;
    bool any = false;
    for (int i = 0; i < kLinKernels; ++i) {
        const LinKernel kernel = (LinKernel)i;
        const LinCost& c = kLinCost[i];
        if (c.waves ? M > c.m || (i > 0 && M <= kLinCost[i - 1].m) : M <= 32) continue;         // few rows have their kernel
        if (kernel == kLinTile256 && (rows != kLinCopied || M <= 128 || N <= 128)) continue;
        const int64_t wgs = (((int64_t)M + c.m - 1) / c.m) * (((int64_t)N + c.n - 1) / c.n);
        if (kernel != kLinTile256 && wgs >= ((int64_t)1 << 32) / kLinThreads[i]) continue;      // more than a launch holds; the large tile's workgroups stay
        constexpr int kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
        for (int parts : kParts) {
            if (parts > 1 && (kernel == kLinTile256 || wgs * parts > 1024 || steps < (c.waves ? 8 : 2) * parts)) break;
            const int per = (steps - 1) / parts + 1, count = (steps - 1) / per + 1;             // no part is empty
            const double t = linear_cost(kernel, M, N, count, per, rows, costs);
            if (!any || t < least) {
                any = true;
                least = t;
                best = {kernel, count, per};
            }
        }
    }
    return best;
}

// Bytes for the parts' sums, whatever the rows' addresses.
inline size_t linear_workspace(int M, int N, int K, const LinCosts& costs = kLinCostsF16) {
    int most = 1;
    for (LinRows rows : {kLinCopied, kLinEven, kLinOdd}) {
        const int parts = linear_plan(M, N, K, rows, costs).parts;
        most = parts > most ? parts : most;
    }
    return most > 1 ? ((size_t)most * M * N * 4 + 255) / 256 * 256 : 0;
}

}  // namespace hb
