// hb_linear_i8: matrix product in 8-bit integers with a scale for each row of both operands and hb_linear's epilogue, and its vector-ALU twin.
#include "linear_tiles.hpp"

namespace hb {

// ---------------------------------------------------------------------------
// Vector-ALU twin: 64 x 64 outputs per workgroup, 4 x 4 per thread, 16 k at a time through LDS.
constexpr int kI8vT = 64, kI8vK = 16;

template <class O>
__global__ void __launch_bounds__(256) linear_i8_valu_kernel(LinearArgs<LinI8> p) {
    __shared__ int s_x[kI8vK][kI8vT + 4], s_w[kI8vK][kI8vT + 4];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int tiles_n = (p.N + kI8vT - 1) / kI8vT;
    const int m0 = (int)(blockIdx.x / (unsigned)tiles_n) * kI8vT, n0 = (int)(blockIdx.x % (unsigned)tiles_n) * kI8vT;
    int acc[4][4] = {};
    for (int k0 = 0; k0 < p.K; k0 += kI8vK) {
        for (int i = tid; i < kI8vT * kI8vK; i += 256) {
            const int r = i / kI8vK, k = i % kI8vK;
            s_x[k][r] = m0 + r < p.M && k0 + k < p.K ? p.x[(m0 + r) * p.x_pitch + k0 + k] : 0;
            s_w[k][r] = n0 + r < p.N && k0 + k < p.K ? p.w[(n0 + r) * p.w_pitch + k0 + k] : 0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kI8vK; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += s_x[k][4 * ty + i] * s_w[k][4 * tx + j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + 4 * ty + i, n = n0 + 4 * tx + j;
            if (m >= p.M || n >= p.N) continue;
            float v = linear_act(lin_scaled(acc[i][j], p.x_scale[m], p.w_scale[n], p.bias ? (float)p.bias[n] : 0.f), p.act);
            if (p.residual) v += (float)static_cast<const O*>(p.residual)[m * p.res_pitch + n];
            static_cast<O*>(p.out)[m * p.out_pitch + n] = (O)v;
        }
}

static hb_status linear_i8_prepare(LinearArgs<LinI8>& a, const int8_t* x, const int8_t* w, const float* x_scale, const float* w_scale, const hb_half* bias,
                                   const void* residual, void* out, int out_type, int act, int M, int N, int K, int64_t x_pitch, int64_t w_pitch,
                                   int64_t res_pitch, int64_t out_pitch) {
    if (!x || !w || !x_scale || !w_scale || !out || M < 1 || N < 1 || K < 1) return HB_ERR_INVALID_ARG;
    if ((out_type != HB_F16 && out_type != HB_F32) || act < HB_ACT_NONE || act > HB_ACT_SILU) return HB_ERR_INVALID_ARG;
    if (!residual) res_pitch = N;
    if (x_pitch < K || w_pitch < K || res_pitch < N || out_pitch < N) return HB_ERR_INVALID_ARG;
    const size_t size = out_type == HB_F32 ? 4 : 2;
    if (!aligned_to(x_scale, 4) || !aligned_to(w_scale, 4) || !aligned_to(bias, 2) || !aligned_to(residual, size) || !aligned_to(out, size)) return HB_ERR_INVALID_ARG;
    for (int64_t p : {x_pitch, w_pitch, res_pitch, out_pitch})
        if (p > HB_LINEAR_MAX_PITCH) return HB_ERR_UNSUPPORTED;
    if (M > kLinMostRows || K > HB_LINEAR_I8_MAX_K) return HB_ERR_UNSUPPORTED;
    a = {x, w, reinterpret_cast<const half_t*>(bias), residual, out, M, N, K, act, x_pitch, w_pitch, res_pitch, out_pitch, (K - 1) / LinI8::kK + 1, x_scale, w_scale};
    return HB_OK;
}

}  // namespace hb

extern "C" size_t hb_linear_i8_workspace_size(int M, int N, int K) {
    return M < 1 || N < 1 || K < 1 ? 0 : hb::linear_workspace(M, N, hb::LinI8::halves(K), hb::LinI8::costs());
}

extern "C" hb_status hb_linear_i8_valu(const int8_t* x, const int8_t* w, const float* x_scale, const float* w_scale, const hb_half* bias, const void* residual,
                                       void* out, hb_type out_type, hb_act act, int M, int N, int K, int64_t x_pitch, int64_t w_pitch,
                                       int64_t residual_pitch, int64_t out_pitch, void* workspace, size_t workspace_bytes, hb_stream stream) {
    using namespace hb;
    LinearArgs<LinI8> a;
    if (hb_status s = linear_i8_prepare(a, x, w, x_scale, w_scale, bias, residual, out, out_type, act, M, N, K, x_pitch, w_pitch, residual_pitch, out_pitch)) return s;
    const int64_t tiles = (int64_t)ceil_div(M, kI8vT) * ((N - 1) / kI8vT + 1);
    if (!launch_holds((double)tiles, 256)) return HB_ERR_UNSUPPORTED;
    const auto st = reinterpret_cast<hipStream_t>(stream);
    if (out_type == HB_F32) hipLaunchKernelGGL(linear_i8_valu_kernel<float>, dim3((unsigned)tiles), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(linear_i8_valu_kernel<half_t>, dim3((unsigned)tiles), dim3(256), 0, st, a);
    return launch_status();
}

extern "C" hb_status hb_linear_i8(const int8_t* x, const int8_t* w, const float* x_scale, const float* w_scale, const hb_half* bias, const void* residual,
                                  void* out, hb_type out_type, hb_act act, int M, int N, int K, int64_t x_pitch, int64_t w_pitch,
                                  int64_t residual_pitch, int64_t out_pitch, void* workspace, size_t workspace_bytes, hb_stream stream) {
    using namespace hb;
    LinearArgs<LinI8> a;
    if (hb_status s = linear_i8_prepare(a, x, w, x_scale, w_scale, bias, residual, out, out_type, act, M, N, K, x_pitch, w_pitch, residual_pitch, out_pitch)) return s;
    const auto st = reinterpret_cast<hipStream_t>(stream);
    return out_type == HB_F32 ? linear_call<LinI8, float>(a, workspace, workspace_bytes, st) : linear_call<LinI8, half_t>(a, workspace, workspace_bytes, st);
}
