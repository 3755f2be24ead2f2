// hb_attention: attention of queries to an encoder's states of another length, and its vector-ALU twin.
#include <float.h>
#include <math.h>

#include "attention_plan.hpp"
#include "hb_device.hpp"
#include "hb_host.hpp"
#include "token_tiles.hpp"

namespace hb {

struct AttentionArgs {
    const half_t* q;
    const half_t* k;
    const half_t* v;
    half_t* out;
    int B, Lq, Lk, Hq, Hkv, D;
    int group;                 // query heads per key head
    int64_t q_batch, q_token, q_head, k_batch, k_token, k_head, v_batch, v_token, v_head, out_batch, out_token, out_head;
    float scale2;              // |scale| * log2(e): the weights are powers of two
    bool negate;               // scale < 0: the queries' sign
    const int32_t* key_len;    // null: all
    const uint8_t* key_mask;   // null: all
    int64_t mask_pitch;
    float* parts;              // keys split: sums of the parts, [part][row][D], then their maximum and sum of weights, [part][row][2]
    int nparts;
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
    const float scale2 = p.negate ? -p.scale2 : p.scale2;
    float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j0 = 0; j0 < len; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < len && (!mask || mask[j]);
        float s = -INFINITY;
        if (seen) {
            const half_t* kj = k + j * p.k_token;
            float dot = 0.f;
            for (int d = 0; d < p.D; ++d) dot = fmaf((float)q[d], (float)kj[d], dot);
            s = dot * scale2;
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

// ---------------------------------------------------------------------------
// On the matrix units.  The query heads that share a key head are rows of one product: row r is query r / group of head r % group.
//
// A wave holds 32 rows, a workgroup of four waves shares the keys, 64 at a time.  With v_mfma_f32_32x32x16_f16 the scores are formed as
// S^T = K Q^T, so that a lane (c, h) has 32 of the 64 scores of ONE row c (keys 8 q + 4 h + r of each 32): maximum and sum need one
// exchange with lane c + 32, and the weights, rounded to fp16, are in place as the operand of O^T = V^T P^T, whose contraction runs
// over the keys in the order that the lanes hold them.  V^T is read from LDS by transposing reads.
constexpr int kAttRows = 32, kAttWaves = 4, kAttTile = kAttRows * kAttWaves;
constexpr int kAttThreads = 64 * kAttWaves;               // of a workgroup, at least

// A tile of keys in LDS: rows of PC 16-byte pieces (8 up to 64 channels, else 16), a piece at place piece ^ flip: what the fragments' reads
// take at one time (16 rows of one piece of k; 4 rows of 64 bytes of v) lies in different banks.
template <int DP, int GROUPS>
constexpr int kAttLds = GROUPS * (DP <= 64 ? 32768 : 65536);                           // two stages of a tile of k and v, for each group
template <int PC>
__device__ __forceinline__ int att_flip_k(int row) { return PC == 8 ? (row >> 1) & 7 : row & 15; }
template <int PC>
__device__ __forceinline__ int att_flip_v(int row) { return PC == 8 ? (row << 1) & 4 : (row << 2) & 12; }

// A workgroup's place in the order of batch, key head, part and rows.  Without lengths every XCD takes a contiguous eighth.  With lengths
// (`same` workgroups, a key head's, have one) that could give one XCD all the short batches: key heads go round the XCDs then, and those
// that are left over when their number is no multiple of 8 are cut into eighths.  4 x 4096 queries, 16 heads of 64, 2048 to 4096 keys: 308
// -> 247 us; all of 4096 keys: 322, and contiguous eighths 321; one query, 16384 keys, 4 x 8 heads over 32 of 128: 56 and 54.
__device__ __forceinline__ int attention_place(int wg, int nwg, int same) {
    const int first = same ? nwg / (8 * same) * (8 * same) : 0;
    return wg < first ? xcd_blocked(wg, first, same) : first + xcd_contiguous(wg - first, nwg - first);
}

// What bounds it, by size (queries x keys, heads of 64 unless said): many keys, the power of matrix and vector units together (4 x 4096 x 4096, 16 heads
// 312 us, 880 TFLOP/s at 2.0 GHz, 0.42 and 0.59 busy); few keys, a workgroup's chain from its queries to its rows, with two on a compute unit
// (8 x 4096 x 77, 16 heads 37.5 us of 22 for the bytes); one query, memory (4 x 16384 keys, 8 heads of 128: 39 us, 4.9 TB/s, and the join).
// LDS conflicts are those of the rows on their way out, 192 cycles a workgroup whatever the keys: 0.22 of all cycles of LDS with 77 keys,
// where these are few, and 2 % of a workgroup's time.
// Products of the next tile ahead of the weights gain 1 to 6 % with many keys and lose with few; a third stage of LDS gains nothing.
//
// The weights are rounded to fp16 for their product with v, which makes a result's error 1.4 times that of its own rounding (2.9e-4 of its
// root mean square in place of 2.1e-4).  TERMS 2: a second product with what the rounding left over takes that away.  Where keys are many it
// costs 30 to 35 % (4 x 4096 x 4096, 16 heads of 64: 307 -> 415 us; 3 x 1079 x 1917, 12 heads over 4 of 80: 47 -> 62), with up to 128 keys 5 to
// 11 % (8 x 4096 x 77: 41.4 -> 44.6), and is left out.  With split keys and rows of one wave, the form of single tokens, the units wait for
// memory for most of the time, and it is there: 1 to 8 %, 5 % in the mean of 144 calls (4 x 1 x 16384, 32 heads over 8 of 128: 53.6 -> 54.5;
// 8 x 1 x 8192, 8 heads of 64: 33.4 -> 33.6; 4 x 2 x 5000, 8 heads of 80: 15.4 -> 16.5).
//
// D rounded up to DP; PARTS: the sums go to the workspace.  GROUPS 2: eight waves, four for the even tiles of the keys and four for the odd
// ones, each with tiles of its own in LDS; they join their sums there.  A workgroup that has a compute unit to itself takes about two thirds of the time.
template <int DP, int GROUPS, bool PARTS, int TERMS>
__global__ void __launch_bounds__(64 * kAttWaves * GROUPS, 2) attention_mfma_kernel(AttentionArgs p) {
    constexpr int PC = DP <= 64 ? 8 : 16, kSteps = DP / 16, kBlocks = DP / 32;
    constexpr int kPitch = 16 * PC, kMatrix = 64 * kPitch, kStage = 2 * kMatrix;      // bytes: a row, a tile of k or v, both
    constexpr int kOwn = PC / 4, kRowsOf = 64 / PC;                                    // copies of 1 KB per matrix and wave, rows in one
    constexpr int kOutPitch = 2 * DP + 16;                                             // bytes of a row on its way out
    static_assert(TERMS == 1 || TERMS == 2);
    static_assert(kAttLds<DP, GROUPS> >= GROUPS * 2 * kStage && kAttLds<DP, GROUPS> >= kAttTile * kOutPitch);
    extern __shared__ __attribute__((aligned(1024))) char s_all[];
    __shared__ __attribute__((aligned(16))) float s_hide[GROUPS][2][64];               // of the tiles with hidden keys: 0, or -inf for these
    __shared__ float s_sums[GROUPS > 1 ? kAttWaves : 1][64][2];                        // references and sums of the second group's rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wv = wave % kAttWaves, team = wave / kAttWaves;
    char* const s_tiles = s_all + team * 2 * kStage;
    float(&s_hidden)[2][64] = s_hide[team];
    const int c = lane & 31, h = lane >> 5;

    // neighbouring workgroups read the same keys
    const int rows = p.Lq * p.group, tiles = (rows + kAttTile - 1) / kAttTile;
    const int id = attention_place(blockIdx.x, gridDim.x, p.key_len ? tiles * p.nparts : 0);
    const int tile = id % tiles, part = id / tiles % p.nparts, bh = id / tiles / p.nparts;
    const int hk = bh % p.Hkv, b = bh / p.Hkv;
    const int row0 = tile * kAttTile + wv * kAttRows;
    const bool active = row0 < rows;

    // this part's keys
    const int len = attention_keys(p, b), all = (len + 63) >> 6;
    const int first = (int)((int64_t)all * part / p.nparts), last = (int)((int64_t)all * (part + 1) / p.nparts);
    const uint8_t* const mask = p.key_mask ? p.key_mask + b * p.mask_pitch : nullptr;

    // copies of a tile: slot `lane` of copy i is row kRowsOf * i + lane / PC, place lane % PC
    const char* const k0 = reinterpret_cast<const char*>(p.k + b * p.k_batch + hk * p.k_head);
    const char* const v0 = reinterpret_cast<const char*>(p.v + b * p.v_batch + hk * p.v_head);
    const uint32_t lds0 = tk_lds_addr(s_tiles);
    auto seen_of = [&](int t, uint32_t byte) HB_INLINE {      // the visible keys of tile t; `byte` is a lane's key's mask
        const int j = 64 * t + lane;
        return __ballot(j < len && byte != 0);
    };
    auto mask_of = [&](int t) HB_INLINE { return (uint32_t)mask[min(64 * t + lane, len - 1)]; };
    uint32_t off_k[kOwn], off_v[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int row = kRowsOf * (kOwn * wv + i) + lane / PC, place = lane % PC;
        const int ck = place ^ att_flip_k<PC>(row), cv = place ^ att_flip_v<PC>(row);
        off_k[i] = 8 * ck < p.D ? (uint32_t)row * (uint32_t)(2 * p.k_token) + 16 * ck : kTkOutside;
        off_v[i] = 8 * cv < p.D ? (uint32_t)row * (uint32_t)(2 * p.v_token) + 16 * cv : kTkOutside;
    }
    auto request = [&](int t, uint64_t seen, int buf) HB_INLINE {
        const u32x4 rk = tk_rsrc(k0 + (int64_t)t * 128 * p.k_token), rv = tk_rsrc(v0 + (int64_t)t * 128 * p.v_token);
        const uint32_t to = lds0 + buf * kStage + 1024 * kOwn * wv;
        if (~seen == 0) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                tk_dma16(rk, off_k[i], 0, to + 1024 * i);
                tk_dma16(rv, off_v[i], 0, to + 1024 * i + kMatrix);
            }
        } else {                                              // what is hidden arrives as zeros
            if (wv == 0) s_hidden[buf][lane] = (seen >> lane) & 1 ? 0.f : -INFINITY;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const bool there = (seen >> (kRowsOf * (kOwn * wv + i) + lane / PC)) & 1;
                tk_dma16(rk, there ? off_k[i] : kTkOutside, 0, to + 1024 * i);
                tk_dma16(rv, there ? off_v[i] : kTkOutside, 0, to + 1024 * i + kMatrix);
            }
        }
    };

    typedef short short4v __attribute__((ext_vector_type(4)));
    uint32_t at_k[kSteps], at_v[kBlocks];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) at_k[i] = lds0 + c * kPitch + ((16 * (h ^ att_flip_k<PC>(c))) ^ (32 * i));
    const int vrow = 4 * h + ((lane & 15) >> 2);
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
        at_v[i] = lds0 + kMatrix + vrow * kPitch + ((16 * (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1))) ^ (16 * att_flip_v<PC>(vrow)) ^ (64 * i)) + 8 * (lane & 1);
    auto read_k = [&](int step, int at) HB_INLINE { return *reinterpret_cast<const __attribute__((address_space(3))) half8*>(at_k[step] + at); };
    auto read_v = [&](int block, int at) HB_INLINE {          // 4 keys from the one at `at` (+ 4 h) on of channel 32 block + c
        return __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) short4v*>(at_v[block] + at)));
    };

    floatx16 o[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float top = -INFINITY, base = 0.f;                        // the score that this row's weights refer to
    float sums[4] = {0.f, 0.f, 0.f, 0.f};                     // of this lane's weights
    bool careful = true;                                      // a row has no such score yet, or scores are beyond 2^13

    half8 qf[kSteps];                                         // queries: lane (c, h) has channels 16 s + 8 h .. + 7 of row c
    auto attend = [&](uint64_t seen, auto index) HB_INLINE {
        constexpr int kAt = decltype(index)::value * kStage;
        floatx16 s[2];
        auto score = [&]() HB_INLINE {
            half8 kf[2][kSteps];
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) kf[k][i] = read_k(i, kAt + 32 * kPitch * k);
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) s[k] = mfma32x32x16(kf[k][i], qf[i], s[k]);
        };
        if (~seen) {                                          // the scores of hidden keys (whose k arrived as zeros) start from -inf
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const floatx4 e = *reinterpret_cast<const floatx4*>(&s_hidden[decltype(index)::value][2 * j + 4 * h]);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[j / 16][j % 16 + i] = e[i];
            }
            score();
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[k][j] = 0.f;
            score();
        }
        half8 w[TERMS][4];
        half4 vf[2][kBlocks];                                 // of the first 16 keys: on their way while the weights are computed
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            vf[0][i] = read_v(i, kAt);
            vf[1][i] = read_v(i, kAt + 8 * kPitch);
        }
        // Weights are 2^7 at the score that they refer to, the largest of a first tile: fp16 then holds those down to 2^-21 of it in full, and
        // up to 2^8 more is as good.  So they are computed first; only where one is larger the maximum is sought and the sums are moved.
        float part[4];
        auto weigh = [&](auto power) HB_INLINE {
            floatx16 e[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < 16; ++j) e[k][j] = power(s[k][j]);
#pragma unroll
            for (int j = 0; j < 4; ++j) part[j] = e[0][j];
#pragma unroll
            for (int j = 4; j < 32; ++j) part[j % 4] += e[j / 16][j % 16];
            if constexpr (TERMS == 1) {
#pragma unroll
                for (int j = 0; j < 32; ++j) w[0][j / 8][j % 8] = (half_t)e[j / 16][j % 16];
            } else {                                          // truncated, so that the rest is exact in fp32
                typedef half_t half2v __attribute__((ext_vector_type(2)));
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    const float a = e[j / 16][j % 16], b = e[j / 16][j % 16 + 1];
                    const half2v most = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(a, b));
                    const half2v rest = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(a - (float)most[0], b - (float)most[1]));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        w[0][j / 8][j % 8 + i] = most[i];
                        w[TERMS - 1][j / 8][j % 8 + i] = rest[i];
                    }
                }
            }
        };
        bool redo = careful;
        if (!careful) {
            weigh([&](float x) HB_INLINE { return __builtin_amdgcn_exp2f(fmaf(x, p.scale2, -base)); });
            redo = __any((part[0] + part[1]) + (part[2] + part[3]) > 32768.f);
        }
        if (redo) {
            // a NaN makes the maximum one, and then moves nothing; its weight makes the row one
            float most = __builtin_elementwise_maximum(s[0][0], s[1][0]);
#pragma unroll
            for (int j = 1; j < 16; ++j) most = __builtin_elementwise_maximum(most, __builtin_elementwise_maximum(s[0][j], s[1][j]));
            const uint32_t bits = __builtin_bit_cast(uint32_t, most);
            const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);         // of lanes c, and of lanes c + 32
            const uint32_t low = both[0], high = both[1];
            most = __builtin_elementwise_maximum(__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)) * p.scale2;
            const float before = top;
            top = fmaxf(top, most);
            base = top == -INFINITY ? 0.f : top - 7.f;
            const float keep = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(before - top);
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[j] *= keep;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] *= keep;
            careful = __any(top == -INFINITY || fabsf(base) > 8192.f);
            // the rounding of a large product would show: the same product for the maximum and for the scores
            weigh([&](float x) HB_INLINE {
                x *= p.scale2;
                asm volatile("" : "+v"(x));
                return __builtin_amdgcn_exp2f(x - base);
            });
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[j] += part[j];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            half8 v[kBlocks];
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) v[i] = join(vf[0][i], vf[1][i]);
            if (k < 3) {
#pragma unroll
                for (int i = 0; i < kBlocks; ++i) {
                    vf[0][i] = read_v(i, kAt + (16 * k + 16) * kPitch);
                    vf[1][i] = read_v(i, kAt + (16 * k + 24) * kPitch);
                }
            }
#pragma unroll
            for (int term = 0; term < TERMS; ++term)
#pragma unroll
                for (int i = 0; i < kBlocks; ++i) o[i] = mfma32x32x16(v[i], w[term][k], o[i]);
        }
    };

    uint64_t seen = 0;
    uint32_t byte = 1;
    int t = first + team;
    if (t < last) {
        if (mask) byte = mask_of(t);
        seen = seen_of(t, byte);
        request(t, seen, 0);
        if (mask) byte = mask_of(t + GROUPS);
    }
    // behind the first tile's request: the queries are on their way with it
    {
        const int row = min(row0 + c, rows - 1), i = row / p.group, g = row - i * p.group;
        const half_t* q = p.q + b * p.q_batch + i * p.q_token + (hk * p.group + g) * p.q_head + 8 * h;
        const uint32_t turn = p.negate ? 0x80008000u : 0u;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            u32x4 v = {0, 0, 0, 0};
            if (16 * s + 8 * h < p.D) v = *reinterpret_cast<const u32x4*>(q + 16 * s);
            qf[s] = __builtin_bit_cast(half8, v ^ turn);
        }
    }
    auto turn = [&](auto index) HB_INLINE {
        const int then = t + GROUPS;
        const uint64_t next = then < last ? seen_of(then, byte) : 0;
        tk_wait_loads<0>();
        lds_barrier();
        if (then < last) {
            request(then, next, decltype(index)::value ^ 1);
            if (mask) byte = mask_of(then + GROUPS);
        }
        if (active && seen) attend(seen, index);
        seen = next;
        t = then;
    };
    for (int left = (last - first + GROUPS - 1) / GROUPS; left > 0; left -= 2) {          // as many turns for either group
        turn(TkInt<0>{});
        if (left > 1) turn(TkInt<1>{});
    }
    float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    sum += __shfl_xor(sum, 32);
    if (GROUPS > 1) {
        // the second group's sums, in the lanes' own order, through its tiles
        lds_barrier();
        float* const across = reinterpret_cast<float*>(s_all + 2 * kStage) + wv * (16 * kBlocks * 64) + lane;
        if (team) {
#pragma unroll
            for (int i = 0; i < kBlocks; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) across[(16 * i + j) * 64] = o[i][j];
            s_sums[wv][lane][0] = top;
            s_sums[wv][lane][1] = sum;
        }
        lds_barrier();
        if (team) return;
        const float other = s_sums[wv][lane][0], both = fmaxf(top, other);
        // a group that saw nothing has sums of 0, or NaN
        const float mine = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - both), theirs = other == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(other - both);
        sum = sum * mine + s_sums[wv][lane][1] * theirs;
        top = both;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = o[i][j] * mine + across[(16 * i + j) * 64] * theirs;
    }
    if (PARTS) {
        if (active && row0 + c < rows) {
            const int64_t total = (int64_t)p.B * p.Hkv * rows, at = part * total + (int64_t)bh * rows + row0 + c;
            float* to = p.parts + at * p.D + 4 * h;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (32 * i + 8 * q < p.D) *reinterpret_cast<floatx4*>(to + 32 * i + 8 * q) = floatx4{o[i][4 * q], o[i][4 * q + 1], o[i][4 * q + 2], o[i][4 * q + 3]};
            if (h == 0) {
                float* ml = p.parts + p.nparts * total * p.D + 2 * at;
                ml[0] = top;
                ml[1] = sum;
            }
        }
        return;
    }
    // out: through LDS, in the tiles of the first group, which nobody reads any more.  Whole rows past the caches: pieces of 32 bytes from
    // registers took 46 us where this takes 42 (8 x 4096 queries, 77 keys, 16 heads of 64), and rows that the caches keep 46 too.
    if (GROUPS == 1) lds_barrier();
    if (!active) return;
    char* const patch = s_all + wv * kAttRows * kOutPitch;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<half4*>(patch + c * kOutPitch + 2 * (32 * i + 8 * q + 4 * h)) =
                to_half4(floatx4{o[i][4 * q], o[i][4 * q + 1], o[i][4 * q + 2], o[i][4 * q + 3]} * inv);
    wave_lds_fence();
    constexpr int kLanes = DP / 8 <= 8 ? 8 : 16;
    const int piece = lane % kLanes;
#pragma unroll
    for (int r = lane / kLanes; r < kAttRows; r += 64 / kLanes) {
        const int row = row0 + r, i = row / p.group, g = row - i * p.group;
        if (row < rows && 8 * piece < p.D)
            __builtin_nontemporal_store(*reinterpret_cast<const half8*>(patch + r * kOutPitch + 16 * piece),
                                        reinterpret_cast<half8*>(p.out + b * p.out_batch + i * p.out_token + (hk * p.group + g) * p.out_head + 8 * piece));
    }
}

// The parts' sums of a row brought to their common reference, in their order: a wave per row, first a lane per part (their weights), then a
// lane per two channels.  Bound by its launch and two trips to memory (128 rows of 16 parts 4.2 us).
__global__ void __launch_bounds__(256) attention_join_kernel(AttentionArgs p) {
    const int lane = threadIdx.x & 63, rows = p.Lq * p.group;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), total = (int64_t)p.B * p.Hkv * rows;
    if (at >= total) return;
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    static_assert(kAttMostParts <= 64 && HB_ATTENTION_MAX_D <= 128);
    const int d = min(2 * lane, p.D - 2);
    const float* o = p.parts + at * p.D + d;
    floatx2 ml = {-INFINITY, 0.f};
    if (lane < p.nparts) ml = *reinterpret_cast<const floatx2*>(p.parts + p.nparts * total * p.D + 2 * (lane * total + at));
    float top = ml[0];
    for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    const float w = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - top);      // a part that saw nothing has sums of 0, or NaN
    float sum = w * ml[1];
    for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
    floatx2 v = {0.f, 0.f};
    auto add = [&](const floatx2& q, int s) HB_INLINE {
        const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), s));
        v[0] = fmaf(f, q[0], v[0]);
        v[1] = fmaf(f, q[1], v[1]);
    };
    int s = 0;
    for (; s + 8 <= p.nparts; s += 8) {
        floatx2 q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = *reinterpret_cast<const floatx2*>(o + (s + i) * total * p.D);
#pragma unroll
        for (int i = 0; i < 8; ++i) add(q[i], s + i);
    }
    for (; s < p.nparts; ++s) add(*reinterpret_cast<const floatx2*>(o + s * total * p.D), s);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int bh = (int)(at / rows), row = (int)(at - (int64_t)bh * rows), i = row / p.group, g = row - i * p.group, b = bh / p.Hkv, hk = bh - b * p.Hkv;
    if (2 * lane < p.D) {
        typedef half_t half2v __attribute__((ext_vector_type(2)));
        *reinterpret_cast<half2v*>(p.out + b * p.out_batch + i * p.out_token + (hk * p.group + g) * p.out_head + d) = half2v{(half_t)(v[0] * inv), (half_t)(v[1] * inv)};
    }
}

static hb_status attention_prepare(AttentionArgs& a, const hb_half* q, const hb_half* k, const hb_half* v, hb_half* out, int B, int Lq, int Lk,
                                   int Hq, int Hkv, int D, const int64_t (&strides)[12], float scale, const int32_t* key_len,
                                   const uint8_t* key_mask, int64_t mask_pitch) {
    if (!q || !out || (Lk > 0 && (!k || !v))) return HB_ERR_INVALID_ARG;
    if (B < 1 || Lq < 1 || Lk < 0 || Hq < 1 || Hkv < 1 || D < 1 || Hq % Hkv != 0) return HB_ERR_INVALID_ARG;
    if (!isfinite(scale) || !aligned_to(key_len, 4)) return HB_ERR_INVALID_ARG;
    for (const void* x : {(const void*)q, (const void*)k, (const void*)v, (const void*)out})
        if (!aligned_to(x, 16)) return HB_ERR_INVALID_ARG;
    // batch, token and head strides of q, k, v, out; that of a single batch, token or head has no meaning
    const int sizes[12] = {B, Lq, Hq, B, Lk, Hkv, B, Lk, Hkv, B, Lq, Hq};
    int64_t st[12];
    for (int i = 0; i < 12; ++i) {
        st[i] = sizes[i] > 1 ? strides[i] : 0;
        if (st[i] < 0 || st[i] % 8 != 0) return HB_ERR_INVALID_ARG;
    }
    if (key_mask && mask_pitch < 0) return HB_ERR_INVALID_ARG;
    if (D % 8 != 0 || D > HB_ATTENTION_MAX_D) return HB_ERR_UNSUPPORTED;
    if (st[4] > (1 << 20) || st[7] > (1 << 20) || (int64_t)Lq * (Hq / Hkv) > kAttMost || Lk > kAttMost) return HB_ERR_UNSUPPORTED;
    a = {reinterpret_cast<const half_t*>(q), reinterpret_cast<const half_t*>(k), reinterpret_cast<const half_t*>(v), reinterpret_cast<half_t*>(out),
         B, Lq, Lk, Hq, Hkv, D, Hq / Hkv, st[0], st[1], st[2], st[3], st[4], st[5], st[6], st[7], st[8], st[9], st[10], st[11],
         // a scale of 0 as one that is too small to tell: hidden scores are -inf, and that times 0 is no number; nor are scores of 0 times
         // infinity, which the largest scales would become
         fminf(fmaxf(fabsf(scale) * 1.44269504f, 1e-30f), FLT_MAX), scale < 0.f, key_len, key_mask, mask_pitch, nullptr, 1};
    return HB_OK;
}

template <int DP, int GROUPS, bool PARTS, int TERMS>
static hb_status attention_launch(const AttentionArgs& a, hipStream_t st) {
    if (!launch_holds(attention_workgroups(a.B, a.Lq, a.Hq, a.Hkv) * a.nparts, 64 * kAttWaves * GROUPS)) return HB_ERR_UNSUPPORTED;
    const int64_t wgs = (int64_t)a.B * a.Hkv * attention_tiles(a.Lq, a.group) * a.nparts;
    const auto kernel = attention_mfma_kernel<DP, GROUPS, PARTS, TERMS>;
    constexpr int kLds = kAttLds<DP, GROUPS>;
    if (kLds > 32768)
        if (hb_status s = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), kLds)) return s;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(64 * kAttWaves * GROUPS), kLds, st, a);
    return launch_status();
}
template <int GROUPS, bool PARTS, int TERMS>
static hb_status attention_run(const AttentionArgs& a, hipStream_t st) {
    if (a.D <= 32) return attention_launch<32, GROUPS, PARTS, TERMS>(a, st);
    if (a.D <= 64) return attention_launch<64, GROUPS, PARTS, TERMS>(a, st);
    if (a.D <= 96) return attention_launch<96, GROUPS, PARTS, TERMS>(a, st);
    return attention_launch<128, GROUPS, PARTS, TERMS>(a, st);
}
template <bool PARTS, int TERMS>
static hb_status attention_run(int groups, const AttentionArgs& a, hipStream_t st) {
    return groups > 1 ? attention_run<2, PARTS, TERMS>(a, st) : attention_run<1, PARTS, TERMS>(a, st);
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

extern "C" size_t hb_attention_workspace_size(int B, int Lq, int Lk, int Hq, int Hkv, int D) {
    if (B < 1 || Lq < 1 || Lk < 1 || Hq < 1 || Hkv < 1 || D < 1 || Hq % Hkv != 0 || (int64_t)Lq * (Hq / Hkv) > hb::kAttMost || Lk > hb::kAttMost) return 0;
    if (!hb::launch_holds(hb::attention_workgroups(B, Lq, Hq, Hkv), hb::kAttThreads)) return 0;
    return hb::attention_workspace(B, Lq, Lk, Hq, Hkv, D);
}

extern "C" hb_status hb_attention_valu(HB_ATTENTION_PARAMS) {
    using namespace hb;
    AttentionArgs a;
    if (hb_status s = HB_ATTENTION_PREPARE(a)) return s;
    if (!launch_holds(((double)B * Hq * Lq + 3.0) / 4.0, 256)) return HB_ERR_UNSUPPORTED;
    const int64_t blocks = ((int64_t)B * Hq * Lq + 3) / 4;
    hipLaunchKernelGGL(attention_valu_kernel, dim3((unsigned)blocks), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
    return launch_status();
}

extern "C" hb_status hb_attention(HB_ATTENTION_PARAMS) {
    using namespace hb;
    AttentionArgs a;
    if (hb_status s = HB_ATTENTION_PREPARE(a)) return s;
    if (!launch_holds(attention_workgroups(B, Lq, Hq, Hkv), kAttThreads)) return HB_ERR_UNSUPPORTED;
    const auto st = reinterpret_cast<hipStream_t>(stream);
    const AttentionPlan plan = attention_plan(B, Lq, Lk, Hq, Hkv, D);
    if (plan.parts == 1) return attention_run<false, 1>(plan.groups, a, st);
    if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < attention_workspace(B, Lq, Lk, Hq, Hkv, D)) return HB_ERR_WORKSPACE;
    a.nparts = plan.parts;
    a.parts = static_cast<float*>(workspace);
    const bool one_wave = (int64_t)Lq * a.group <= kAttRows;
    if (hb_status s = one_wave ? attention_run<true, 2>(plan.groups, a, st) : attention_run<true, 1>(plan.groups, a, st)) return s;
    const int64_t blocks = ((int64_t)B * Hq * Lq + 3) / 4;
    hipLaunchKernelGGL(attention_join_kernel, dim3((unsigned)blocks), dim3(256), 0, st, a);
    return launch_status();
}
