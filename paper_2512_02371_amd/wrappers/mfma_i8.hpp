// The product of 8-bit integers on the matrix units: the one place that issues it.  hb_device.hpp holds the wrappers of the floating-point products, and a test
// holds that header to exactly those; this one stands beside the sources with a test of its own.
#pragma once

namespace hb {

typedef int intx4 __attribute__((ext_vector_type(4)));

// v_mfma_i32_16x16x64_i8    D[16x16] += A[16x64] * B[64x16]      (lane = 16*g + c)
//   A: lane (c, g) holds 16 bytes of A[c][.];  B: lane (c, g) holds 16 bytes of B[.][c], the same k as A's lane: any order of k serves
//   D: lane (c, g) holds D[4g .. 4g+3][c]        (4 integers)
// As with the fp16 products there is one shape: an accumulator never sees another.
__device__ __forceinline__ intx4 mfma16x16x64i8(intx4 a, intx4 b, intx4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

}  // namespace hb
