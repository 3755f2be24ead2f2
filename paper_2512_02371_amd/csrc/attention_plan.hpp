// hb_attention: into how many parts the keys are split; host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace hb {

// Workgroups (128 rows each) per key head.
inline int64_t attention_tiles(int Lq, int group) { return ((int64_t)Lq * group + 127) / 128; }

// Few rows leave compute units idle: their keys are split until there are about two workgroups a unit, in parts of four tiles of 64
// keys at least.
inline int attention_parts(int B, int Lq, int Lk, int Hq, int Hkv) {
    const int64_t wgs = (int64_t)B * Hkv * attention_tiles(Lq, Hq / Hkv), tiles = ((int64_t)Lk + 63) / 64;
    int64_t parts = (512 + wgs - 1) / wgs;
    if (wgs >= 256) parts = 1;
    if (parts > tiles / 4) parts = tiles / 4;
    return parts < 1 ? 1 : (int)parts;
}

// Bytes for the parts' sums, maxima and sums of weights; 0 where there is one part.
inline size_t attention_workspace(int B, int Lq, int Lk, int Hq, int Hkv, int D) {
    const int parts = attention_parts(B, Lq, Lk, Hq, Hkv);
    return parts > 1 ? ((size_t)parts * B * Hq * Lq * (D + 2) * 4 + 255) / 256 * 256 : 0;
}

}  // namespace hb
