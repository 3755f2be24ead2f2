// hb_quantize_rows: rows of fp16 values as 8-bit integers with a scale.
#include "hb_device.hpp"
#include "hb_host.hpp"
#include "quantize_plan.hpp"

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

// Eight adjacent values at any address, zeros from `valid` on (in pieces of four, two and one), and their integers.  WHOLE: all eight are there.
template <bool WHOLE>
__device__ __forceinline__ half8 quantize_load(const half_t* from, int valid) {
    if (WHOLE || valid >= 8) return *reinterpret_cast<const half8_u*>(from);
    half8 r = {0, 0, 0, 0, 0, 0, 0, 0};
    if (valid <= 0) return r;
    typedef half_t half2_u __attribute__((ext_vector_type(2), aligned(2)));
    const int four = valid & 4, two = valid & 2;
    half4_u a = {0, 0, 0, 0};
    half2_u b = {0, 0};
    half_t c = 0;
    if (four) a = *reinterpret_cast<const half4_u*>(from);
    if (two) b = *reinterpret_cast<const half2_u*>(from + four);
    if (valid & 1) c = from[four + two];
    const half4 rest = two ? half4{b[0], b[1], c, 0} : half4{c, 0, 0, 0};
    return four ? join(a, rest) : join(rest, half4{0, 0, 0, 0});
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

// LANES lanes take a row together, of 256 or of LANES; 8 to 64 of them are of one wave.  Rows of up to 8 LANES kQuantizeHeld values stay in registers, of longer ones what is beyond is
// read twice, the second time from the caches.  Memory: 32768 x 1024 20.4 us, 4.9 TB/s;
// 1917 x 1079 in wider rows, of odd addresses, 4.4 us and 1 x 4096 3.3 to 3.8, the launch.
template <int LANES, bool WHOLE>
__global__ void __launch_bounds__(LANES > 256 ? LANES : 256) quantize_rows_kernel(QuantizeArgs p) {
    constexpr int kRows = LANES > 256 ? 1 : 256 / LANES, kWaves = LANES / 64;
    __shared__ uint32_t s_top[kWaves > 1 ? kRows * kWaves : 1];
    const int lane = threadIdx.x % LANES, in = threadIdx.x / LANES;
    const int64_t m = (int64_t)blockIdx.x * kRows + in;
    const bool there = m < p.M;
    const half_t* const x = p.x + (there ? m : 0) * p.x_pitch;
    int8_t* const out = p.q + (there ? m : 0) * p.q_pitch;
    half8 held[kQuantizeHeld];
    const int steps = (p.K - 1) / (8 * LANES) + 1;                           // uniform
#pragma unroll
    for (int i = 0; i < kQuantizeHeld; ++i)
        if (i < steps) {
            const int k = 8 * (lane + i * LANES);
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
    for (int k = 8 * (lane + kQuantizeHeld * LANES); k < p.K; k += 8 * LANES) take(quantize_load<WHOLE>(x + k, p.K - k));
    uint32_t bits = most[0] > most[1] ? most[0] : most[1];
#pragma unroll
    for (int d = (LANES < 64 ? LANES : 64) / 2; d > 0; d >>= 1) bits = max(bits, (uint32_t)__shfl_xor(bits, d));
    if (kWaves > 1) {
        s_top[threadIdx.x >> 6] = bits;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) bits = max(bits, s_top[in * kWaves + i]);
    }
    if (!there) return;
    float top = bits < 0x7c00u ? (float)__builtin_bit_cast(half_t, (uint16_t)bits) : __builtin_nanf("");
    const bool some = top > 0.f;                          // neither zeros nor a NaN
    const float inverse = some ? 1.f / top : 0.f, scale = top / 127.f;
    if (!some) top = 0.f;                                 // zeros divided by it are zeros
    auto put = [&](half8 v, int k) __attribute__((always_inline)) {
        if (!some) v = half8{0, 0, 0, 0, 0, 0, 0, 0};
        if (k < p.K) quantize_store<WHOLE>(out + k, v, top, inverse, p.K - k);
    };
#pragma unroll
    for (int i = 0; i < kQuantizeHeld; ++i)
        if (i < steps) put(held[i], 8 * (lane + i * LANES));
    for (int k = 8 * (lane + kQuantizeHeld * LANES); k < p.K; k += 8 * LANES) put(quantize_load<WHOLE>(x + k, p.K - k), k);
    if (lane == 0) p.scale[m] = scale;
}

constexpr int kQuantizeMostK = 0x7fffffff - (1 << 17) + 1;                     // places count in 32 bits, up to a step beyond the row

template <int LANES>
static hb_status quantize_launch(const QuantizeArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)quantize_workgroups(a.M, LANES)), block(quantize_threads(LANES));
    if (a.K % 8 == 0) hipLaunchKernelGGL((quantize_rows_kernel<LANES, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((quantize_rows_kernel<LANES, false>), grid, block, 0, st, a);
    return launch_status();
}
static hb_status quantize_call(const QuantizeArgs& a, hipStream_t st) {
    switch (quantize_lanes(a.M, a.K)) {
        case 8: return quantize_launch<8>(a, st);
        case 16: return quantize_launch<16>(a, st);
        case 32: return quantize_launch<32>(a, st);
        case 64: return quantize_launch<64>(a, st);
        case 256: return quantize_launch<256>(a, st);
        default: return quantize_launch<1024>(a, st);
    }
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
    return quantize_call(a, st);
}
