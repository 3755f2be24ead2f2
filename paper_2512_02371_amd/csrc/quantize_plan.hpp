// hb_quantize_rows: how many lanes take a row together; host arithmetic.
#pragma once
#include <stdint.h>

namespace hb {

constexpr int kQuantizeHeld = 8;          // vectors of a lane that stay in registers

// Workgroups of max(lanes, 256) lanes take 256 / lanes rows, or one.
inline int64_t quantize_workgroups(int M, int lanes) { return lanes > 256 ? M : ((int64_t)M - 1) / (256 / lanes) + 1; }
inline int quantize_threads(int lanes) { return lanes > 256 ? lanes : 256; }

// So many lanes that each has two vectors of a row, up to a wave; more waves where a wave does not hold the row, and where rows are so few that one is read sooner by several
// (91824 x 35 with a wave each 33 us).  1024 lanes for each of 2^22 rows are the 2^32 that no launch holds: with so many rows, 256 take also those that they do not hold.
inline int quantize_lanes(int M, int K) {
    if ((K > 8 * 256 * kQuantizeHeld && M < 1 << 22) || (M < 64 && K > 4096)) return 1024;
    if (K > 8 * 64 * kQuantizeHeld || (M < 1024 && K > 512)) return 256;
    return K <= 128 ? 8 : K <= 256 ? 16 : K <= 512 ? 32 : 64;
}

}  // namespace hb
