// hb_rope_axes: rotary positions with several axes.
#include "hb_device.hpp"
#include "hb_host.hpp"

namespace hb {

struct RopeArgs {
    const half_t* x;
    half_t* out;
    const int32_t* pos;
    const float* freq;
    int B, L, H, D, P;
    int64_t x_batch, x_token, x_head, out_batch, out_token, out_head, pos_batch, pos_token;
    int end[HB_ROPE_MAX_AXES];     // the first pair beyond each axis' section
    int interleaved;
};

// cos and sin of pos * freq radians.  The product is taken in turns, as a sum of two floats (Dekker: the fused multiply-add
// gives the rounding error of a product exactly), and loses its whole turns before anything is rounded away: an angle of
// thousands of turns keeps an error of 2^-24 of a turn, where the rounded product of radians would be off by thousands of that.
__device__ __forceinline__ void rope_turn(int pos, float freq, float& co, float& si) {
#pragma clang fp contract(off)                                            // a product merged into a sum would count its rounding error twice
    constexpr float kHi = 0.15915494f, kLo = 6.4206383e-09f;           // 1 / (2 pi)
    const float f = freq * kHi, fe = fmaf(freq, kHi, -f) + freq * kLo;    // freq in turns
    const int low = (uint32_t)pos + (1u << 24) > (2u << 24) ? pos & 255 : 0;   // positions that a float does not hold: in two parts
    const float ph = (float)(pos - low), pe = (float)low;
    const float t = ph * f, u = pe * f;
    float r = (t - rintf(t)) + ((u - rintf(u)) + (fmaf(ph, f, -t) + (fmaf(pe, f, -u) + fmaf(ph, fe, pe * fe))));
    // the nearest quarter turn, and Taylor's series for the rest: the next terms are 3e-8 at an eighth of a turn
    const float quarter = rintf(4.f * r), a = 6.2831853f * fmaf(-0.25f, quarter, r), b = a * a;
    const float s = a * fmaf(b, fmaf(b, fmaf(b, fmaf(b, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float c = fmaf(b, fmaf(b, fmaf(b, fmaf(b, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const int n = (int)quarter;
    co = n & 1 ? s : c;
    si = n & 1 ? c : s;
    co = (n + 1) & 2 ? -co : co;
    si = n & 2 ? -si : si;
}

__device__ __forceinline__ int rope_axis(const RopeArgs& p, int pair) {
    int a = 0;
#pragma unroll
    for (int i = 0; i < HB_ROPE_MAX_AXES - 1; ++i) a += pair >= p.end[i] ? 1 : 0;
    return a;
}

// A thread per pair (or channel beyond the pairs) of one token, all heads.
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs p) {
    const int per = p.P + (p.D - 2 * p.P);
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= (int64_t)p.B * p.L * per) return;
    const int e = (int)(t % per);
    const int64_t tok = t / per;
    const int l = (int)(tok % p.L), b = (int)(tok / p.L);
    const half_t* x = p.x + b * p.x_batch + l * p.x_token;
    half_t* o = p.out + b * p.out_batch + l * p.out_token;
    if (e >= p.P) {
        const int d = e + p.P;
        for (int h = 0; h < p.H; ++h) o[h * p.out_head + d] = x[h * p.x_head + d];
        return;
    }
    float co, si;
    rope_turn(p.pos[b * p.pos_batch + l * p.pos_token + rope_axis(p, e)], p.freq[e], co, si);
    const int du = p.interleaved ? 2 * e : e, dv = p.interleaved ? 2 * e + 1 : e + p.P;
    for (int h = 0; h < p.H; ++h) {
        const float u = x[h * p.x_head + du], v = x[h * p.x_head + dv];
        o[h * p.out_head + du] = (half_t)(u * co - v * si);
        o[h * p.out_head + dv] = (half_t)(v * co + u * si);
    }
}

}  // namespace hb

extern "C" hb_status hb_rope_axes(const hb_half* x, hb_half* out, const int32_t* positions, const float* freq, int B, int L, int H, int D,
                                  int64_t x_batch, int64_t x_token, int64_t x_head, int64_t out_batch, int64_t out_token, int64_t out_head,
                                  int64_t pos_batch, int64_t pos_token, const int32_t* sections, int axes, int interleaved, hb_stream stream) {
    using namespace hb;
    if (!x || !out || !positions || !freq || !sections || B < 1 || L < 1 || H < 1 || D < 2 || axes < 1) return HB_ERR_INVALID_ARG;
    if (!aligned_to(x, 2) || !aligned_to(out, 2) || !aligned_to(positions, 4) || !aligned_to(freq, 4)) return HB_ERR_INVALID_ARG;
    for (int64_t s : {x_batch, x_token, x_head, out_batch, out_token, out_head, pos_batch, pos_token})
        if (s < 0) return HB_ERR_INVALID_ARG;
    if (axes > HB_ROPE_MAX_AXES || D > 65536) return HB_ERR_UNSUPPORTED;
    RopeArgs a = {reinterpret_cast<const half_t*>(x), reinterpret_cast<half_t*>(out), positions, freq, B, L, H, D, 0,
                  x_batch, x_token, x_head, out_batch, out_token, out_head, pos_batch, pos_token, {}, interleaved != 0};
    int64_t pairs = 0;
    for (int i = 0; i < HB_ROPE_MAX_AXES; ++i) {
        if (i < axes && sections[i] < 0) return HB_ERR_INVALID_ARG;
        pairs += i < axes ? sections[i] : 0;
        if (2 * pairs > D) return HB_ERR_INVALID_ARG;
        a.end[i] = (int)pairs;
    }
    if (pairs < 1) return HB_ERR_INVALID_ARG;
    a.P = (int)pairs;
    const int64_t blocks = ((int64_t)B * L * (D - a.P) + 255) / 256;
    if (blocks > 0x7fffffff) return HB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(rope_kernel, dim3((unsigned)blocks), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
    return launch_status();
}
