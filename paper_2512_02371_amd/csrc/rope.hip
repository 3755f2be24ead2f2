// hb_rope_axes: rotary positions with several axes.
#include <algorithm>

#include "hb_device.hpp"
#include "hb_host.hpp"

namespace hb {

// Threads that share a token's heads, at most, and the heads that a loop over them can count in 32 bits.
constexpr int kRopeMostGroups = 1 << 20, kRopeMostHeads = 0x7fffffff - kRopeMostGroups + 1;

struct RopeArgs {
    const half_t* x;
    half_t* out;
    const int32_t* pos;
    const float* freq;
    int B, L, H, D, P;
    int64_t x_batch, x_token, x_head, out_batch, out_token, out_head, pos_batch, pos_token;
    int end[HB_ROPE_MAX_AXES];     // the first pair beyond each axis' section
    int interleaved;
    int groups;                    // threads that share the heads of a token and its pairs
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

// Bound by reading x and writing out once.  A thread turns V pairs of one token (8 that lie P channels apart, 16 bytes each, or 4 that lie
// together, 16 bytes) in every kHeads-th head from its own on: the angles' cost is shared by the heads, and the loads of several heads are on
// their way at the same time.  Threads beyond the pairs copy V pairs' worth of channels.  V = 1: any address.
// 8 x 4096 tokens, 16 heads of 64: 24 us, 5.5 TB/s; 24960 tokens, 24 heads of 128, interleaved: 56 us, 5.5 TB/s.
template <int V, bool INTERLEAVED>
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs p) {
    constexpr int W = INTERLEAVED ? 2 * V : V;            // channels in one access
    typedef half_t vec __attribute__((ext_vector_type(W), aligned(V == 1 ? 2 : 2 * W)));
    const int turning = p.P / V, rest = p.D - 2 * p.P, copied = (rest + W - 1) / W, per = turning + copied;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, total = (int64_t)p.B * p.L * p.groups * per;
    if (t >= total) return;
    int e, group, l, b;
    auto place = [&](auto at) {                           // of t, in 32 bits where these hold it: a division in 64 takes 100 instructions
        using T = decltype(at);
        const T u = at / (T)per, tok = u / (T)p.groups;
        e = (int)(at - u * (T)per);
        group = (int)(u - tok * (T)p.groups);
        b = (int)(tok / (T)p.L);
        l = (int)(tok - (T)b * (T)p.L);
    };
    if (total <= 0x7fffffff) place((uint32_t)t);
    else place((uint64_t)t);
    const half_t* x = p.x + b * p.x_batch + l * p.x_token;
    half_t* o = p.out + b * p.out_batch + l * p.out_token;
    constexpr int U = 4;                                  // heads at a time
    if (e >= turning) {
        const int d = 2 * p.P + (e - turning) * W;
        for (int h = group; h < p.H; h += p.groups) {
            const half_t* from = x + (int64_t)h * p.x_head + d;
            half_t* to = o + (int64_t)h * p.out_head + d;
            if (d + W <= p.D) *reinterpret_cast<vec*>(to) = *reinterpret_cast<const vec*>(from);
            else *to = *from;                             // one channel behind the last pair
        }
        return;
    }
    float co[V], si[V];
    const int32_t* pos = p.pos + b * p.pos_batch + l * p.pos_token;
#pragma unroll
    for (int i = 0; i < V; ++i) rope_turn(pos[rope_axis(p, e * V + i)], p.freq[e * V + i], co[i], si[i]);
    const int d0 = e * W, d1 = INTERLEAVED ? d0 : d0 + p.P;
    auto turn = [&](vec& a, vec& c) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float f = INTERLEAVED ? a[2 * i % W] : a[i % W], g = INTERLEAVED ? a[(2 * i + 1) % W] : c[i % W];
            const half_t r = (half_t)(f * co[i] - g * si[i]), s = (half_t)(g * co[i] + f * si[i]);
            if (INTERLEAVED) {
                a[2 * i % W] = r;
                a[(2 * i + 1) % W] = s;
            } else {
                a[i % W] = r;
                c[i % W] = s;
            }
        }
    };
    int h = group;
    for (const int last = p.H - (U - 1) * p.groups; h < last; h += U * p.groups) {
        vec a[U], c[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const half_t* q = x + (int64_t)(h + i * p.groups) * p.x_head;
            a[i] = *reinterpret_cast<const vec*>(q + d0);
            if (!INTERLEAVED) c[i] = *reinterpret_cast<const vec*>(q + d1);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            turn(a[i], c[i]);
            half_t* q = o + (int64_t)(h + i * p.groups) * p.out_head;
            __builtin_nontemporal_store(a[i], reinterpret_cast<vec*>(q + d0));
            if (!INTERLEAVED) __builtin_nontemporal_store(c[i], reinterpret_cast<vec*>(q + d1));
        }
    }
    for (; h < p.H; h += p.groups) {
        vec a = *reinterpret_cast<const vec*>(x + (int64_t)h * p.x_head + d0), c = a;
        if (!INTERLEAVED) c = *reinterpret_cast<const vec*>(x + (int64_t)h * p.x_head + d1);
        turn(a, c);
        *reinterpret_cast<vec*>(o + (int64_t)h * p.out_head + d0) = a;
        if (!INTERLEAVED) *reinterpret_cast<vec*>(o + (int64_t)h * p.out_head + d1) = c;
    }
}

template <int V, bool INTERLEAVED>
static hb_status rope_launch(RopeArgs a, hipStream_t st) {
    constexpr int W = INTERLEAVED ? 2 * V : V;
    const int64_t per_token = a.P / V + (a.D - 2 * a.P + W - 1) / W;
    // heads are shared out until there are 16 waves a SIMD to come and go (4: 64 us for 24960 tokens, 24 heads of 128, 57 with 16)
    if (!launch_holds((double)a.B * a.L * per_token, 1)) return HB_ERR_UNSUPPORTED;
    const int64_t threads = a.B * (int64_t)a.L * per_token, wanted = (int64_t)num_cu() * 4096;
    a.groups = (int)std::min<int64_t>(std::min(a.H, kRopeMostGroups), std::max<int64_t>(1, wanted / threads));
    const int64_t blocks = (threads * a.groups + 255) / 256;
    if (!launch_holds((double)blocks, 256)) return HB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((rope_kernel<V, INTERLEAVED>), dim3((unsigned)blocks), dim3(256), 0, st, a);
    return launch_status();
}

}  // namespace hb

extern "C" hb_status hb_rope_axes(const hb_half* x, hb_half* out, const int32_t* positions, const float* freq, int B, int L, int H, int D,
                                  int64_t x_batch, int64_t x_token, int64_t x_head, int64_t out_batch, int64_t out_token, int64_t out_head,
                                  int64_t pos_batch, int64_t pos_token, const int32_t* sections, int axes, int interleaved, hb_stream stream) {
    using namespace hb;
    if (!x || !out || !positions || !freq || !sections || B < 1 || L < 1 || H < 1 || D < 2 || axes < 1) return HB_ERR_INVALID_ARG;
    if (!aligned_to(x, 2) || !aligned_to(out, 2) || !aligned_to(positions, 4) || !aligned_to(freq, 4)) return HB_ERR_INVALID_ARG;
    // the stride of a single batch, token or head has no meaning, and must not decide how wide the accesses are
    if (B == 1) x_batch = out_batch = pos_batch = 0;
    if (L == 1) x_token = out_token = pos_token = 0;
    if (H == 1) x_head = out_head = 0;
    for (int64_t s : {x_batch, x_token, x_head, out_batch, out_token, out_head, pos_batch, pos_token})
        if (s < 0) return HB_ERR_INVALID_ARG;
    if (axes > HB_ROPE_MAX_AXES || D > 65536 || H > kRopeMostHeads) return HB_ERR_UNSUPPORTED;
    RopeArgs a = {reinterpret_cast<const half_t*>(x), reinterpret_cast<half_t*>(out), positions, freq, B, L, H, D, 0,
                  x_batch, x_token, x_head, out_batch, out_token, out_head, pos_batch, pos_token, {}, interleaved != 0, 1};
    int64_t pairs = 0;
    for (int i = 0; i < HB_ROPE_MAX_AXES; ++i) {
        if (i < axes && sections[i] < 0) return HB_ERR_INVALID_ARG;
        pairs += i < axes ? sections[i] : 0;
        if (2 * pairs > D) return HB_ERR_INVALID_ARG;
        a.end[i] = (int)pairs;
    }
    if (pairs < 1) return HB_ERR_INVALID_ARG;
    a.P = (int)pairs;
    const auto st = reinterpret_cast<hipStream_t>(stream);
    const int64_t strides = x_batch | x_token | x_head | out_batch | out_token | out_head;
    const bool aligned = aligned_to(x, 16) && aligned_to(out, 16) && strides % 8 == 0;
    if (interleaved) return aligned && a.P % 4 == 0 && D % 8 == 0 ? rope_launch<4, true>(a, st) : rope_launch<1, true>(a, st);
    return aligned && a.P % 8 == 0 && D % 8 == 0 ? rope_launch<8, false>(a, st) : rope_launch<1, false>(a, st);
}
