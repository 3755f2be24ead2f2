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

// A row per workgroup, read twice.
__global__ void __launch_bounds__(256) quantize_plain_kernel(QuantizeArgs p) {
    __shared__ float s[256];
    const half_t* x = p.x + (int64_t)blockIdx.x * p.x_pitch;
    int8_t* q = p.q + (int64_t)blockIdx.x * p.q_pitch;
    float top = 0.f;
    for (int k = threadIdx.x; k < p.K; k += 256) {
        const float v = fabsf((float)x[k]);
        top = v <= top ? top : v;                         // a NaN is kept, and nothing is larger
        if (v < __builtin_inff()) continue;
        top = __builtin_nanf("");
        break;
    }
    s[threadIdx.x] = top;
    __syncthreads();
    for (int half = 128; half > 0; half >>= 1) {
        if ((int)threadIdx.x < half) {
            const float a = s[threadIdx.x], b = s[threadIdx.x + half];
            s[threadIdx.x] = a != a || a >= b ? a : b;
        }
        __syncthreads();
    }
    top = s[0];
    const float inverse = 1.f / top;
    for (int k = threadIdx.x; k < p.K; k += 256) q[k] = top > 0.f ? (int8_t)quantized((float)x[k], top, inverse) : (int8_t)0;
    if (threadIdx.x == 0) p.scale[blockIdx.x] = top / 127.f;
}

}  // namespace hb

extern "C" hb_status hb_quantize_rows(const hb_half* x, int8_t* q, float* scale, int M, int K, int64_t x_pitch, int64_t q_pitch, hb_stream stream) {
    using namespace hb;
    if (!x || !q || !scale || M < 1 || K < 1) return HB_ERR_INVALID_ARG;
    if (M == 1) x_pitch = q_pitch = K;
    if (x_pitch < K || q_pitch < K || !aligned_to(x, 2) || !aligned_to(scale, 4)) return HB_ERR_INVALID_ARG;
    if (!launch_holds((double)M, 256)) return HB_ERR_UNSUPPORTED;
    const QuantizeArgs a = {reinterpret_cast<const half_t*>(x), q, scale, M, K, x_pitch, q_pitch};
    hipLaunchKernelGGL(quantize_plain_kernel, dim3((unsigned)M), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
    return launch_status();
}
