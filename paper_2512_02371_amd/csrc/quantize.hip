// hb_quantize_rows: rows of fp16 values as 8-bit integers with a scale.
#include "hb_device.hpp"
#include "hb_host.hpp"

namespace hb {

struct QuantizeArgs {
    const half_t* x;
    int8_t* q;
    float* scale;
    int M, K;
    int64_t x_pitch, q_pitch;
};

// The integer nearest to 127 x / top, ties to even.  127 x is exact; the quotient, between 2^e and 2^(e + 1), is a half or at least 2^(e - 20) away from one
// (x and top are 11-bit numbers, x at most 2^(8 - e) times smaller), and one step of Newton's from the reciprocal is within 2^(e - 22) of it, and exact
// where it is a half: rounding it gives the integer of the exact quotient.
__device__ __forceinline__ float quantized(float x, float top, float inverse) {
    const float t = 127.f * x, q = t * inverse;
    return rintf(fmaf(fmaf(-q, top, t), inverse, q));
}

constexpr int kQuantizeHeld = 8;          // vectors of a lane that stay in registers

// Eight adjacent values, zeros from `valid` on, and their integers.  WHOLE: all eight are there; others stand at any address.
template <bool WHOLE>
__device__ __forceinline__ half8 quantize_load(const half_t* from, int valid) {
    if (WHOLE || valid >= 8) return *reinterpret_cast<const half8_u*>(from);
    half8 r = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < valid) r[i] = from[i];
    return r;
}
template <bool WHOLE>
__device__ __forceinline__ void quantize_store(int8_t* to, half8 x, float top, float inverse, int valid) {
    typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(1)));
    int q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = (int)quantized((float)x[i], top, inverse);
    if (WHOLE || valid >= 8) {
        u32x2_u r;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t low = __builtin_amdgcn_perm((uint32_t)q[4 * i + 1], (uint32_t)q[4 * i], 0x0c0c0400u), high = __builtin_amdgcn_perm((uint32_t)q[4 * i + 3], (uint32_t)q[4 * i + 2], 0x04000c0cu);
            r[i] = low | high;
        }
        *reinterpret_cast<u32x2_u*>(to) = r;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) to[i] = (int8_t)q[i];
    }
}

// WAVES waves take a row together; a workgroup has 4 / WAVES rows (or one).  Rows of up to 512 WAVES kQuantizeHeld values stay in registers, of longer ones what is beyond is
// read twice, the second time from the caches.
template <int WAVES, bool WHOLE>
__global__ void __launch_bounds__(WAVES > 4 ? 64 * WAVES : 256) quantize_rows_kernel(QuantizeArgs p) {
    constexpr int kRows = WAVES > 4 ? 1 : 4 / WAVES, kLanes = 64 * WAVES;
    __shared__ uint32_t s_top[WAVES > 4 ? WAVES : 4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x % kLanes;
    const int64_t m = (int64_t)blockIdx.x * kRows + wave / WAVES;
    const bool there = m < p.M;
    const half_t* const x = p.x + (there ? m : 0) * p.x_pitch;
    int8_t* const out = p.q + (there ? m : 0) * p.q_pitch;
    half8 held[kQuantizeHeld];
    const int steps = (p.K + 8 * kLanes - 1) / (8 * kLanes);                 // uniform
#pragma unroll
    for (int i = 0; i < kQuantizeHeld; ++i)
        if (i < steps) {
            const int k = 8 * (lane + i * kLanes);
            held[i] = quantize_load<WHOLE>(x + (WHOLE ? min(k, p.K - 8) : k), p.K - k);
        }
    // magnitudes compare as their bits do, infinities above all numbers and NaN above them
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};
    auto take = [&](half8 v) __attribute__((always_inline)) {
        const u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    };
#pragma unroll
    for (int i = 0; i < kQuantizeHeld; ++i)
        if (i < steps) take(held[i]);
    for (int k = 8 * (lane + kQuantizeHeld * kLanes); k < p.K; k += 8 * kLanes) take(quantize_load<WHOLE>(x + k, p.K - k));
    uint32_t bits = most[0] > most[1] ? most[0] : most[1];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) bits = max(bits, (uint32_t)__shfl_xor(bits, d));
    if (WAVES > 1) {
        s_top[wave] = bits;
        __syncthreads();
        const int first = wave / WAVES * WAVES;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) bits = max(bits, s_top[first + i]);
    }
    if (!there) return;
    float top = bits < 0x7c00u ? (float)__builtin_bit_cast(half_t, (uint16_t)bits) : __builtin_nanf("");
    const bool some = top > 0.f;                          // neither zeros nor a NaN
    const float inverse = some ? 1.f / top : 0.f, scale = top / 127.f;
    if (!some) top = 0.f;                                 // 0 * 127 x + 0: a NaN or an infinity in x is made a zero below
    auto put = [&](half8 v, int k) __attribute__((always_inline)) {
        if (!some) v = half8{0, 0, 0, 0, 0, 0, 0, 0};
        if (k < p.K) quantize_store<WHOLE>(out + k, v, top, inverse, p.K - k);
    };
#pragma unroll
    for (int i = 0; i < kQuantizeHeld; ++i)
        if (i < steps) put(held[i], 8 * (lane + i * kLanes));
    for (int k = 8 * (lane + kQuantizeHeld * kLanes); k < p.K; k += 8 * kLanes) put(quantize_load<WHOLE>(x + k, p.K - k), k);
    if (lane == 0) p.scale[m] = scale;
}

constexpr int kQuantizeMostK = 0x7fffffff - (1 << 17) + 1;                     // places count in 32 bits, up to a step beyond the row

// A wave takes a row alone while there are rows for all of the chip and it holds the row; more of them where rows are few or long.
static int quantize_waves(int M, int K) {
    if (K > 512 * 4 * kQuantizeHeld || (M < 64 && K > 4096)) return 16;
    return K > 512 * kQuantizeHeld || (M < 1024 && K > 512) ? 4 : 1;
}

template <int WAVES>
static hb_status quantize_launch(const QuantizeArgs& a, hipStream_t st) {
    constexpr int kRows = WAVES > 4 ? 1 : 4 / WAVES;
    const dim3 grid((unsigned)((a.M - 1) / kRows + 1)), block(WAVES > 4 ? 64 * WAVES : 256);
    if (a.K % 8 == 0) hipLaunchKernelGGL((quantize_rows_kernel<WAVES, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((quantize_rows_kernel<WAVES, false>), grid, block, 0, st, a);
    return launch_status();
}

}  // namespace hb

extern "C" hb_status hb_quantize_rows(const hb_half* x, int8_t* q, float* scale, int M, int K, int64_t x_pitch, int64_t q_pitch, hb_stream stream) {
    using namespace hb;
    if (!x || !q || !scale || M < 1 || K < 1) return HB_ERR_INVALID_ARG;
    if (M == 1) x_pitch = q_pitch = K;
    if (x_pitch < K || q_pitch < K || !aligned_to(x, 2) || !aligned_to(scale, 4)) return HB_ERR_INVALID_ARG;
    if (M >= 1 << 24 || K > kQuantizeMostK) return HB_ERR_UNSUPPORTED;
    const QuantizeArgs a = {reinterpret_cast<const half_t*>(x), q, scale, M, K, x_pitch, q_pitch};
    const auto st = reinterpret_cast<hipStream_t>(stream);
    return quantize_waves(M, K) == 1 ? quantize_launch<1>(a, st) : quantize_waves(M, K) == 4 ? quantize_launch<4>(a, st) : quantize_launch<16>(a, st);
}
