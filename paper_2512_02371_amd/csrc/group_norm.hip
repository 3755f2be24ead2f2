// hb_group_norm: group norm with an activation, channels last.
#include <math.h>

#include "hb_device.hpp"
#include "hb_host.hpp"
#include "token_epilogue.hpp"

namespace hb {

struct NormArgs {
    const void* x;
    void* out;
    const half_t* weight;      // null: ones
    const half_t* bias;        // null: zeros
    float eps;
    int act;
    int N, P, C, G;
    int64_t x_image, x_pixel, out_image, out_pixel;
};

// The sum over a workgroup of 256, in a fixed order.
__device__ __forceinline__ float norm_sum(float v, float* s) {
    s[threadIdx.x] = v;
    __syncthreads();
    for (int half = 128; half > 0; half >>= 1) {
        if ((int)threadIdx.x < half) s[threadIdx.x] += s[threadIdx.x + half];
        __syncthreads();
    }
    const float r = s[0];
    __syncthreads();
    return r;
}

// One group of one image per workgroup, read three times: the mean, the squares of what is left, the results.
template <class X, class O>
__global__ void __launch_bounds__(256) group_norm_plain_kernel(NormArgs p) {
    __shared__ float s[256];
    const int n = blockIdx.x / p.G, g = blockIdx.x % p.G, D = p.C / p.G;
    const X* x = static_cast<const X*>(p.x) + n * p.x_image + g * D;
    O* out = static_cast<O*>(p.out) + n * p.out_image + g * D;
    const int64_t count = (int64_t)p.P * D;
    float sum = 0.f;
    for (int64_t i = threadIdx.x; i < count; i += 256) sum += (float)x[i / D * p.x_pixel + i % D];
    float mean = norm_sum(sum, s) / (float)count, left = 0.f;
    sum = 0.f;
    for (int64_t i = threadIdx.x; i < count; i += 256) {
        const float d = (float)x[i / D * p.x_pixel + i % D] - mean;
        left += d;
        sum = fmaf(d, d, sum);
    }
    // what the rounded sum left of the mean
    left = norm_sum(left, s) / (float)count;
    mean += left;
    const float rstd = 1.f / sqrtf(fmaxf(norm_sum(sum, s) / (float)count - left * left, 0.f) + p.eps);
    for (int64_t i = threadIdx.x; i < count; i += 256) {
        const int c = (int)(i % D);
        float v = ((float)x[i / D * p.x_pixel + c] - mean) * rstd;
        if (p.weight) v *= (float)p.weight[g * D + c];
        if (p.bias) v += (float)p.bias[g * D + c];
        out[i / D * p.out_pixel + c] = (O)linear_act(v, p.act);
    }
}

template <class X, class O>
static hb_status norm_call(const NormArgs& a, hipStream_t st) {
    if (!launch_holds((double)a.N * a.G, 256)) return HB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((group_norm_plain_kernel<X, O>), dim3((unsigned)(a.N * a.G)), dim3(256), 0, st, a);
    return launch_status();
}

}  // namespace hb

extern "C" size_t hb_group_norm_workspace_size(int, int, int, int) { return 0; }

extern "C" hb_status hb_group_norm(const void* x, hb_type x_type, const hb_half* weight, const hb_half* bias, void* out, hb_type out_type,
                                   hb_act act, float eps, int N, int P, int C, int groups, int64_t x_image, int64_t x_pixel,
                                   int64_t out_image, int64_t out_pixel, void* workspace, size_t workspace_bytes, hb_stream stream) {
    using namespace hb;
    (void)workspace;
    (void)workspace_bytes;
    if (!x || !out || N < 1 || P < 1 || C < 1 || groups < 1 || C % groups) return HB_ERR_INVALID_ARG;
    if ((x_type != HB_F16 && x_type != HB_F32) || (out_type != HB_F16 && out_type != HB_F32) || act < HB_ACT_NONE || act > HB_ACT_SILU) return HB_ERR_INVALID_ARG;
    if (!(eps > 0.f) || isinf(eps)) return HB_ERR_INVALID_ARG;
    if (!aligned_to(x, x_type == HB_F32 ? 4 : 2) || !aligned_to(out, out_type == HB_F32 ? 4 : 2) || !aligned_to(weight, 2) || !aligned_to(bias, 2)) return HB_ERR_INVALID_ARG;
    if (C / groups > HB_GROUP_NORM_MAX_CHANNELS || P >= 1 << 30 || (int64_t)N * groups >= 1 << 30) return HB_ERR_UNSUPPORTED;
    // the stride of a single image or pixel has no meaning
    if (P == 1) x_pixel = out_pixel = C;
    if (N == 1) x_image = out_image = C;
    if (x_pixel < C || out_pixel < C || x_image < C || out_image < C) return HB_ERR_INVALID_ARG;
    const NormArgs a = {x, out, reinterpret_cast<const half_t*>(weight), reinterpret_cast<const half_t*>(bias), eps, act, N, P, C, groups, x_image, x_pixel, out_image, out_pixel};
    const auto st = reinterpret_cast<hipStream_t>(stream);
    if (x_type == HB_F32) return out_type == HB_F32 ? norm_call<float, float>(a, st) : norm_call<float, half_t>(a, st);
    return out_type == HB_F32 ? norm_call<half_t, float>(a, st) : norm_call<half_t, half_t>(a, st);
}
