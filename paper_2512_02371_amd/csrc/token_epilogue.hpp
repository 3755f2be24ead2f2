// Pieces of the token operators' epilogues: activations, and the loads and stores of a lane's adjacent elements.
#pragma once
#include "hb_device.hpp"
#include "token_tiles.hpp"

namespace hb {

// 1 / (1 + exp(-v)); the hardware's reciprocal is within 1 ulp, a division would take ten instructions.
__device__ __forceinline__ float lin_sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * v)); }
__device__ __forceinline__ float linear_act(float v, int act) {
    switch (act) {
        case HB_ACT_RELU: return v < 0.f ? 0.f : v;                       // a NaN stays one
        case HB_ACT_GELU: {
            // v times the normal distribution at v.  Its tail is exp(-a^2 / 2) times a function of a = |v| that falls from 1/2 as 1 / a: here t times a
            // polynomial in t = 1 / (1 + 0.303 a), of least relative error (Remez exchange, a up to 14): 1e-7, 4e-7 as computed.  Small results
            // keep their digits: the exponent's roundings add v^2 2^-23 at most, 4e-6 at -8.
            const float t = __builtin_amdgcn_rcpf(fmaf(0.303f, fabsf(v), 1.f));
            float q = fmaf(t, 0.0363918774f, -0.155077848f);
            q = fmaf(t, fmaf(t, fmaf(t, q, 0.194474897f), -0.0445769286f), 0.124181752f);
            q = fmaf(t, fmaf(t, fmaf(t, q, 0.101983908f), 0.121787084f), 0.120835214f) * t;
            const float tail = q * __builtin_amdgcn_exp2f(-0.72134752f * v * v);
            return v * (v < 0.f ? tail : 1.f - tail);
        }
        case HB_ACT_GELU_TANH: {                                              // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
            const float e = __builtin_amdgcn_exp2f(v * fmaf(v * v, -2.3022082f * 0.044715f, -2.3022082f));
            return v * __builtin_amdgcn_rcpf(1.f + e);
        }
        case HB_ACT_SILU: return v * lin_sigmoid(v);
        default: return v;
    }
}

// `count` of V adjacent elements, at any address that their type allows.  Stores are streaming, whole lines of a row at a time, which is for what
// they would push out of the caches: 100000 x 200 fp32, K 96, with a residual 48 -> 38 us, but 23 -> 33 without one; 2^20 x 64, K 64 with a residual
// 83.8 -> 82.5; 8192 x 8192, K 2048 with gelu_tanh 245 -> 243, without 234 -> 238; smaller outputs within 5 %.
template <int V, class S, class T>
__device__ __forceinline__ void lin_load(S (&v)[V], const T* from, int count) {
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (count >= V) {
        const vec q = *reinterpret_cast<const vec*>(from);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (S)q[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < count ? (S)from[i] : (S)0;
    }
}
template <int V, class T>
__device__ __forceinline__ void lin_store(T* to, const float (&v)[V], int count) {
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (count >= V) {
        vec q;
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = (T)v[i];
        __builtin_nontemporal_store(q, reinterpret_cast<vec*>(to));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < count) to[i] = (T)v[i];
    }
}
// One branch for all of them: a branch for each would leave its exponential's latency bare.
template <int V>
__device__ __forceinline__ void lin_act(float (&v)[V], int act) {
    auto all = [&](auto f) HB_INLINE {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = f(v[i]);
    };
    switch (act) {
        case HB_ACT_RELU: return all([](float x) HB_INLINE { return linear_act(x, HB_ACT_RELU); });
        case HB_ACT_GELU: return all([](float x) HB_INLINE { return linear_act(x, HB_ACT_GELU); });
        case HB_ACT_GELU_TANH: return all([](float x) HB_INLINE { return linear_act(x, HB_ACT_GELU_TANH); });
        case HB_ACT_SILU: return all([](float x) HB_INLINE { return linear_act(x, HB_ACT_SILU); });
        default: return;
    }
}

}  // namespace hb
