// hb_linear: which kernel a call takes and into how many parts the sum over k is split; host arithmetic.
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

inline double linear_cost(LinKernel kernel, int64_t M, int64_t N, int parts, int steps, LinRows rows) {
    const LinCost& c = kernel == kLinTile128 && rows != kLinCopied  ? kLinCostTile128Held
                       : kernel == kLinTile64 && rows == kLinCopied ? kLinCostTile64Copied
                                                                    : kLinCost[kernel];
    const int64_t wgs = ((M + c.m - 1) / c.m) * ((N + c.n - 1) / c.n) * parts;
    const double slow = rows == kLinOdd ? 1.0 + c.odd : 1.0;
    double t;
    if (c.waves) {
        const double waves = (steps + c.waves - 1) / c.waves * c.alone, all = wgs / 256.0 * steps * c.shared;
        t = c.begin + (waves > all ? waves : all) * slow;
    } else {
        const double one = steps * c.alone * slow + c.begin, all = (double)((wgs + 255) / 256) * (steps * c.shared * slow + c.end);
        t = (one > all ? one : all) * (steps == 1 && kernel == kLinTile128x64 ? kLinOneStep : 1.0);
    }
    if (parts > 1) t += kLinJoin + parts * kLinJoinPart + 8.0 * parts * M * N / kLinJoinRate;
    return t + kLinLaunch;
}

inline LinPlan linear_plan(int M, int N, int K, LinRows rows) {
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
            const double t = linear_cost(kernel, M, N, count, per, rows);
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
inline size_t linear_workspace(int M, int N, int K) {
    int most = 1;
    for (LinRows rows : {kLinCopied, kLinEven, kLinOdd}) {
        const int parts = linear_plan(M, N, K, rows).parts;
        most = parts > most ? parts : most;
    }
    return most > 1 ? ((size_t)most * M * N * 4 + 255) / 256 * 256 : 0;
}

}  // namespace hb
