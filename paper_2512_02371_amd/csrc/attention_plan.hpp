// hb_attention: into how many parts the keys are split; host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace hb {

constexpr int kAttMostParts = 64;

// Workgroups (128 rows each) per key head.
inline int64_t attention_tiles(int Lq, int group) { return ((int64_t)Lq * group + 127) / 128; }

// Few rows leave compute units idle, and a workgroup alone on one waits for its tiles of 64 keys one after the other: their keys are
// split into parts, which a second launch joins.  How many is the least of a model of the call's time in us: a tile takes `alone` for a
// workgroup alone, `shared` and `wave` for each wave with rows where several are on a compute unit.  The constants, by the channels
// rounded up to 32, were fitted to 469 calls of random sizes (1 to 4096 queries, 65 to 16384 keys), each timed with 1 to 64 parts:
// the choice is on average 1.3 % behind the fastest (one part always: 66 %).
inline int attention_parts(int B, int Lq, int Lk, int Hq, int Hkv, int D) {
    constexpr double kAlone[] = {0.673, 0.813, 1.034, 1.250}, kShared[] = {0.071, 0.186, 0.305, 0.391}, kWave[] = {0.094, 0.101, 0.107, 0.159};
    constexpr double kBegin = 0.5, kEnd = 1.3, kJoin = 3.7, kJoinRate = 5.0e6;                  // us, us, us, bytes per us
    const int c = (D - 1) / 32 < 3 ? (D - 1) / 32 : 3;
    const int64_t rows = (int64_t)Lq * (Hq / Hkv), wgs = (int64_t)B * Hkv * attention_tiles(Lq, Hq / Hkv), tiles = ((int64_t)Lk + 63) / 64;
    const double one = kShared[c] + kWave[c] * (rows >= 128 ? 4 : (double)((rows + 31) / 32));
    int best = 1;
    double least = 0.0;
    for (int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, kAttMostParts}) {
        if (parts > 1 && (parts > tiles || wgs * parts > 4096)) break;
        const double per = (double)((tiles + parts - 1) / parts), alone = per * kAlone[c] + kBegin;
        double t = (double)((wgs * parts + 255) / 256) * (per * one + kEnd);
        if (t < alone) t = alone;
        if (parts > 1) t += kJoin + 8.0 * parts * B * Hq * Lq * D / kJoinRate;
        if (parts == 1 || t < least) {
            least = t;
            best = parts;
        }
    }
    return best;
}

// Bytes for the parts' sums, references and sums of weights; 0 where there is one part.
inline size_t attention_workspace(int B, int Lq, int Lk, int Hq, int Hkv, int D) {
    const int parts = attention_parts(B, Lq, Lk, Hq, Hkv, D);
    return parts > 1 ? ((size_t)parts * B * Hq * Lq * (D + 2) * 4 + 255) / 256 * 256 : 0;
}

}  // namespace hb
