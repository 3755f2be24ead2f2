// hb_linear: which kernel a call takes and into how many parts the sum over k is split; host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace hb {

// How the rows of x and w stand in memory: at 16-byte addresses with K a multiple of 8, so that they can be copied to LDS directly; at
// 4-byte addresses; or at odd elements, too.
enum LinRows { kLinCopied, kLinEven, kLinOdd };

enum LinKernel { kLinRows16, kLinRows32, kLinRows64, kLinTile64, kLinTile128x64, kLinTile128, kLinTile256, kLinKernels };

struct LinPlan {
    LinKernel kernel;
    int parts, steps;             // of the sum, and steps of 64 k of one part
};

// The time of a call in us, as a model with a few constants per kernel: a workgroup alone on a compute unit takes `alone` a step and
// `begin` beside it, one of several `shared` and `end`; a kernel for few rows of x has its waves take turns at the steps.  `odd`:
// what rows at odd addresses add.  The constants were fitted to 1200 calls of random sizes (1 .. 2^20 x 16 .. 8192, K 16 ..
// 8192), each timed with every kernel and with 1 to 32 parts: the choice is on average 1.5 % behind the fastest.
struct LinCost {
    int m, n;                     // outputs of a workgroup
    int waves;                    // that share the steps; 0: tiles
    double alone, shared, begin, end, odd;
};
constexpr LinCost kLinCost[kLinKernels] = {
    {16, 16, 16, 0.350, 0.043, 0.21, 0.00, 0.12}, {32, 16, 8, 0.419, 0.070, 0.35, 0.00, 0.10}, {64, 16, 8, 0.582, 0.169, 0.27, 0.00, 0.11},
    {64, 64, 0, 0.290, 0.192, 1.26, 0.90, 0.25},  {128, 64, 0, 1.328, 0.227, 1.00, 1.50, 0.27}, {128, 128, 0, 0.528, 0.393, 2.46, 1.34, 0.00},
    {256, 256, 0, 0.497, 1.064, 3.00, 6.60, 0.00},
};
constexpr double kLinLaunch = 3.3, kLinJoin = 1.2, kLinJoinPart = 0.05, kLinJoinRate = 12.5e6;      // us, us, us, bytes per us

inline double linear_cost(LinKernel kernel, int64_t M, int64_t N, int parts, int steps, LinRows rows) {
    const LinCost& c = kLinCost[kernel];
    const int64_t wgs = ((M + c.m - 1) / c.m) * ((N + c.n - 1) / c.n) * parts;
    double slow = rows == kLinOdd ? 1.0 + c.odd : 1.0, t;
    if (kernel == kLinTile128 && rows != kLinCopied) slow = 0.85;     // through registers: faster alone, and it waits for nobody
    if (c.waves) {
        const double waves = (steps + c.waves - 1) / c.waves * c.alone, all = wgs / 256.0 * steps * c.shared;
        t = c.begin + (waves > all ? waves : all) * slow;
    } else {
        const double one = steps * c.alone * slow + c.begin, all = (double)((wgs + 255) / 256) * (steps * c.shared * slow + c.end);
        t = one > all ? one : all;
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
