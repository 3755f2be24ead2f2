// hb_linear: matrix product with bias, activation and residual in its epilogue, and its vector-ALU twin.
#include "hb_device.hpp"
#include "hb_host.hpp"

namespace hb {

struct LinearArgs {
    const half_t* x;
    const half_t* w;
    const half_t* bias;        // null: none
    const void* residual;      // null: none
    void* out;
    int M, N, K, act;
    int64_t x_pitch, w_pitch, res_pitch, out_pitch;
};

__device__ __forceinline__ float linear_act(float v, int act) {
    switch (act) {
        case HB_ACT_RELU: return v < 0.f ? 0.f : v;                       // a NaN stays one
        case HB_ACT_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678f));
        // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
        case HB_ACT_GELU_TANH: return v / (1.f + __expf(-1.5957691f * (v + 0.044715f * v * v * v)));
        case HB_ACT_SILU: return v / (1.f + __expf(-v));
        default: return v;
    }
}

// ---------------------------------------------------------------------------
// Vector-ALU twin: 64 x 64 outputs per workgroup, 4 x 4 per thread, 16 k at a time through LDS.
constexpr int kLvT = 64, kLvK = 16;

template <class O>
__global__ void __launch_bounds__(256) linear_valu_kernel(LinearArgs p) {
    __shared__ float s_x[kLvK][kLvT + 4], s_w[kLvK][kLvT + 4];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int tiles_n = (p.N + kLvT - 1) / kLvT;
    const int m0 = (int)(blockIdx.x / (unsigned)tiles_n) * kLvT, n0 = (int)(blockIdx.x % (unsigned)tiles_n) * kLvT;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < p.K; k0 += kLvK) {
        for (int i = tid; i < kLvT * kLvK; i += 256) {
            const int r = i / kLvK, k = i % kLvK;
            s_x[k][r] = m0 + r < p.M && k0 + k < p.K ? (float)p.x[(m0 + r) * p.x_pitch + k0 + k] : 0.f;
            s_w[k][r] = n0 + r < p.N && k0 + k < p.K ? (float)p.w[(n0 + r) * p.w_pitch + k0 + k] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kLvK; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(s_x[k][4 * ty + i], s_w[k][4 * tx + j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + 4 * ty + i, n = n0 + 4 * tx + j;
            if (m >= p.M || n >= p.N) continue;
            float v = linear_act(acc[i][j] + (p.bias ? (float)p.bias[n] : 0.f), p.act);
            if (p.residual) v += (float)static_cast<const O*>(p.residual)[m * p.res_pitch + n];
            static_cast<O*>(p.out)[m * p.out_pitch + n] = (O)v;
        }
}

static hb_status linear_prepare(LinearArgs& a, const hb_half* x, const hb_half* w, const hb_half* bias, const void* residual, void* out,
                                int out_type, int act, int M, int N, int K, int64_t x_pitch, int64_t w_pitch, int64_t res_pitch,
                                int64_t out_pitch) {
    if (!x || !w || !out || M < 1 || N < 1 || K < 1) return HB_ERR_INVALID_ARG;
    if ((out_type != HB_F16 && out_type != HB_F32) || act < HB_ACT_NONE || act > HB_ACT_SILU) return HB_ERR_INVALID_ARG;
    if (!residual) res_pitch = N;
    if (x_pitch < K || w_pitch < K || res_pitch < N || out_pitch < N) return HB_ERR_INVALID_ARG;
    const size_t size = out_type == HB_F32 ? 4 : 2;
    if (!aligned_to(x, 2) || !aligned_to(w, 2) || !aligned_to(bias, 2) || !aligned_to(residual, size) || !aligned_to(out, size)) return HB_ERR_INVALID_ARG;
    for (int64_t p : {x_pitch, w_pitch, res_pitch, out_pitch})
        if (p > HB_LINEAR_MAX_PITCH) return HB_ERR_UNSUPPORTED;
    a = {reinterpret_cast<const half_t*>(x), reinterpret_cast<const half_t*>(w), reinterpret_cast<const half_t*>(bias), residual, out, M, N, K, act,
         x_pitch, w_pitch, res_pitch, out_pitch};
    return HB_OK;
}

}  // namespace hb

extern "C" size_t hb_linear_workspace_size(int M, int N, int K) { return 0; }

extern "C" hb_status hb_linear_valu(const hb_half* x, const hb_half* w, const hb_half* bias, const void* residual, void* out, hb_type out_type,
                                    hb_act act, int M, int N, int K, int64_t x_pitch, int64_t w_pitch, int64_t residual_pitch,
                                    int64_t out_pitch, void* workspace, size_t workspace_bytes, hb_stream stream) {
    using namespace hb;
    LinearArgs a;
    if (hb_status s = linear_prepare(a, x, w, bias, residual, out, out_type, act, M, N, K, x_pitch, w_pitch, residual_pitch, out_pitch)) return s;
    const int64_t tiles = (int64_t)ceil_div(M, kLvT) * ceil_div(N, kLvT);
    if (tiles > 0x7fffffff) return HB_ERR_UNSUPPORTED;
    const auto st = reinterpret_cast<hipStream_t>(stream);
    if (out_type == HB_F32) hipLaunchKernelGGL(linear_valu_kernel<float>, dim3((unsigned)tiles), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(linear_valu_kernel<half_t>, dim3((unsigned)tiles), dim3(256), 0, st, a);
    return launch_status();
}

extern "C" hb_status hb_linear(const hb_half* x, const hb_half* w, const hb_half* bias, const void* residual, void* out, hb_type out_type,
                               hb_act act, int M, int N, int K, int64_t x_pitch, int64_t w_pitch, int64_t residual_pitch,
                               int64_t out_pitch, void* workspace, size_t workspace_bytes, hb_stream stream) {
    return hb_linear_valu(x, w, bias, residual, out, out_type, act, M, N, K, x_pitch, w_pitch, residual_pitch, out_pitch, workspace,
                          workspace_bytes, stream);
}
