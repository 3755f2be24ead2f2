// hb_attention: into how many parts the keys are split, and how many groups of waves share a part; host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace hb {

constexpr int kAttMostParts = 64;
// Most keys, and most rows of a key head: the kernels count both in 32 bits, and look up to three tiles of 64 keys past the last one.
constexpr int kAttMost = 0x7fffff00;

// Workgroups (128 rows each) per key head.
inline int64_t attention_tiles(int Lq, int group) { return ((int64_t)Lq * group + 127) / 128; }
// Workgroups of one part of the keys; in double, where no sizes overflow.
inline double attention_workgroups(int B, int Lq, int Hq, int Hkv) { return (double)B * Hkv * (double)attention_tiles(Lq, Hq / Hkv); }

struct AttentionPlan {
    int parts;                    // of the keys, in workgroups of their own; a second launch joins them
    int groups;                   // of four waves in a workgroup, which take turns at its tiles of 64 keys and join their sums in LDS
};

// Few rows leave compute units idle, and a workgroup alone on one computes its tiles of 64 keys one after the other: their keys are split.
// Into how many parts and groups is the least of a model of the call's time in us: a tile takes `alone` for a workgroup alone and
// `shared` where several are on a compute unit, and `wave` more for each wave with rows; two groups take about two thirds of the time of
// one.  The constants, by the channels rounded up to 32, were fitted to 516 calls of random sizes (1 to 4096 queries, 65 to 16384
// keys), each timed with one and two groups and 1 to 64 parts.  On 338 other calls, of the kernels as they are now, the choice is on average
// 1.4 % behind the fastest (one part and one group always: 96 %).
inline AttentionPlan attention_plan(int B, int Lq, int Lk, int Hq, int Hkv, int D) {
    struct Cost {
        double alone, alone_wave, shared, shared_wave;
    };
    constexpr Cost kCost[] = {{0.616, 0.021, 0.139, 0.075}, {0.773, 0.032, 0.186, 0.101}, {0.903, 0.069, 0.371, 0.093}, {1.062, 0.085, 0.541, 0.140}};
    constexpr double kBegin[] = {0.9, 1.5}, kEnd[] = {0.7, 2.4}, kGroup[] = {1.0, 0.689}, kGroupWave[] = {1.0, 0.955};
    constexpr double kJoin = 3.0, kJoinPart = 0.04, kJoinRate = 4.5e6;                          // us, us, bytes per us
    const Cost& c = kCost[(D - 1) / 32 < 3 ? (D - 1) / 32 : 3];
    const int64_t rows = (int64_t)Lq * (Hq / Hkv), wgs = (int64_t)B * Hkv * attention_tiles(Lq, Hq / Hkv), tiles = ((int64_t)Lk + 63) / 64;
    const double waves = rows >= 128 ? 4 : (double)((rows + 31) / 32), shared = c.shared + waves * c.shared_wave;
    AttentionPlan best = {1, 1};
    double least = 0.0;
    for (int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, kAttMostParts}) {
        if (parts > 1 && (parts > tiles || wgs * parts > 4096)) break;
        const double per = (double)((tiles + parts - 1) / parts), join = parts > 1 ? kJoin + parts * kJoinPart + 8.0 * parts * B * Hq * Lq * D / kJoinRate : 0.0;
        for (int g = 0; g < (per > 1 ? 2 : 1); ++g) {
            const double alone = per * (kGroup[g] * c.alone + kGroupWave[g] * waves * c.alone_wave) + kBegin[g];
            double t = (double)((wgs * parts + 255) / 256) * (per * shared + kEnd[g]);
            if (t < alone) t = alone;
            t += join;
            if ((parts == 1 && g == 0) || t < least) {
                least = t;
                best = {parts, g + 1};
            }
        }
    }
    return best;
}

// Bytes for the parts' sums, references and sums of weights; 0 where there is one part.
inline size_t attention_workspace(int B, int Lq, int Lk, int Hq, int Hkv, int D) {
    const int parts = attention_plan(B, Lq, Lk, Hq, Hkv, D).parts;
    return parts > 1 ? ((size_t)parts * B * Hq * Lq * (D + 2) * 4 + 255) / 256 * 256 : 0;
}

}  // namespace hb
