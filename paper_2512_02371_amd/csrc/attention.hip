// hb_attention: attention of queries to an encoder's states of another length, and its vector-ALU twin.
#include <float.h>
#include <math.h>

#include "hb_device.hpp"
#include "hb_host.hpp"

namespace hb {

struct AttentionArgs {
    const half_t* q;
    const half_t* k;
    const half_t* v;
    half_t* out;
    int B, Lq, Lk, Hq, Hkv, D;
    int group;                 // query heads per key head
    int64_t q_batch, q_token, q_head, k_batch, k_token, k_head, v_batch, v_token, v_head, out_batch, out_token, out_head;
    float scale2;              // scale * log2(e): the weights are powers of two
    const int32_t* key_len;    // null: all
    const uint8_t* key_mask;   // null: all
    int64_t mask_pitch;
};

__device__ __forceinline__ int attention_keys(const AttentionArgs& p, int b) { return p.key_len ? clampi(p.key_len[b], 0, p.Lk) : p.Lk; }

// ---------------------------------------------------------------------------
// Vector-ALU twin: a wave per query row.  64 keys at a time, first a lane per key (scores), then a lane per two channels (sums of
// the values), with the running maximum and sum of the softmax in between.
__global__ void __launch_bounds__(256) attention_valu_kernel(AttentionArgs p) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)p.B * p.Hq * p.Lq) return;
    const int i = (int)(row % p.Lq), h = (int)(row / p.Lq % p.Hq), b = (int)(row / p.Lq / p.Hq), hk = h / p.group;
    const half_t* q = p.q + b * p.q_batch + i * p.q_token + h * p.q_head;
    const half_t* k = p.k + b * p.k_batch + hk * p.k_head;
    const half_t* v = p.v + b * p.v_batch + hk * p.v_head;
    const uint8_t* mask = p.key_mask ? p.key_mask + b * p.mask_pitch : nullptr;
    const int len = attention_keys(p, b);
    float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j0 = 0; j0 < len; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < len && (!mask || mask[j]);
        float s = -INFINITY;
        if (seen) {
            const half_t* kj = k + j * p.k_token;
            float dot = 0.f;
            for (int d = 0; d < p.D; ++d) dot = fmaf((float)q[d], (float)kj[d], dot);
            s = dot * p.scale2;
        }
        const uint64_t any = __ballot(seen);
        if (!any) continue;
        float most = s;
        for (int m = 32; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
        const float now = fmaxf(top, most), base = now == -INFINITY ? 0.f : now;
        const float keep = exp2f(top - base), e = seen ? exp2f(s - base) : 0.f;
        float part = e;
        for (int m = 32; m; m >>= 1) part += __shfl_xor(part, m);
        sum = sum * keep + part;
        o0 *= keep;
        o1 *= keep;
        top = now;
        for (int n = 0; n < 64; ++n) {
            if (!((any >> n) & 1)) continue;
            const float w = __shfl(e, n);
            const half_t* vj = v + (j0 + n) * p.v_token;
            if (lane < p.D) o0 = fmaf(w, (float)vj[lane], o0);
            if (lane + 64 < p.D) o1 = fmaf(w, (float)vj[lane + 64], o1);
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    half_t* o = p.out + b * p.out_batch + i * p.out_token + h * p.out_head;
    if (lane < p.D) o[lane] = (half_t)(o0 * inv);
    if (lane + 64 < p.D) o[lane + 64] = (half_t)(o1 * inv);
}

static hb_status attention_prepare(AttentionArgs& a, const hb_half* q, const hb_half* k, const hb_half* v, hb_half* out, int B, int Lq, int Lk,
                                   int Hq, int Hkv, int D, const int64_t (&st)[12], float scale, const int32_t* key_len,
                                   const uint8_t* key_mask, int64_t mask_pitch) {
    if (!q || !out || (Lk > 0 && (!k || !v))) return HB_ERR_INVALID_ARG;
    if (B < 1 || Lq < 1 || Lk < 0 || Hq < 1 || Hkv < 1 || D < 1 || Hq % Hkv != 0) return HB_ERR_INVALID_ARG;
    if (!isfinite(scale) || !aligned_to(key_len, 4)) return HB_ERR_INVALID_ARG;
    for (const void* x : {(const void*)q, (const void*)k, (const void*)v, (const void*)out})
        if (!aligned_to(x, 16)) return HB_ERR_INVALID_ARG;
    for (int64_t s : st)
        if (s < 0 || s % 8 != 0) return HB_ERR_INVALID_ARG;
    if (key_mask && mask_pitch < 0) return HB_ERR_INVALID_ARG;
    if (D % 8 != 0 || D > HB_ATTENTION_MAX_D) return HB_ERR_UNSUPPORTED;
    if (st[4] > (1 << 20) || st[7] > (1 << 20)) return HB_ERR_UNSUPPORTED;
    a = {reinterpret_cast<const half_t*>(q), reinterpret_cast<const half_t*>(k), reinterpret_cast<const half_t*>(v), reinterpret_cast<half_t*>(out),
         B, Lq, Lk, Hq, Hkv, D, Hq / Hkv, st[0], st[1], st[2], st[3], st[4], st[5], st[6], st[7], st[8], st[9], st[10], st[11],
         scale * 1.44269504f, key_len, key_mask, mask_pitch};
    return HB_OK;
}

}  // namespace hb

#define HB_ATTENTION_PARAMS                                                                                                                 \
    const hb_half *q, const hb_half *k, const hb_half *v, hb_half *out, int B, int Lq, int Lk, int Hq, int Hkv, int D, int64_t q_batch,     \
        int64_t q_token, int64_t q_head, int64_t k_batch, int64_t k_token, int64_t k_head, int64_t v_batch, int64_t v_token, int64_t v_head, \
        int64_t out_batch, int64_t out_token, int64_t out_head, float scale, const int32_t *key_len, const uint8_t *key_mask,               \
        int64_t mask_pitch, void *workspace, size_t workspace_bytes, hb_stream stream
#define HB_ATTENTION_PREPARE(a)                                                                                                             \
    attention_prepare(a, q, k, v, out, B, Lq, Lk, Hq, Hkv, D, {q_batch, q_token, q_head, k_batch, k_token, k_head, v_batch, v_token, v_head, \
                      out_batch, out_token, out_head}, scale, key_len, key_mask, mask_pitch)

extern "C" size_t hb_attention_workspace_size(int B, int Lq, int Lk, int Hq, int Hkv, int D) { return 0; }

extern "C" hb_status hb_attention_valu(HB_ATTENTION_PARAMS) {
    using namespace hb;
    AttentionArgs a;
    if (hb_status s = HB_ATTENTION_PREPARE(a)) return s;
    const int64_t blocks = ((int64_t)B * Hq * Lq + 3) / 4;
    if (blocks > 0x7fffffff) return HB_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(attention_valu_kernel, dim3((unsigned)blocks), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
    return launch_status();
}

extern "C" hb_status hb_attention(HB_ATTENTION_PARAMS) {
    return hb_attention_valu(q, k, v, out, B, Lq, Lk, Hq, Hkv, D, q_batch, q_token, q_head, k_batch, k_token, k_head, v_batch, v_token, v_head,
                             out_batch, out_token, out_head, scale, key_len, key_mask, mask_pitch, workspace, workspace_bytes, stream);
}
