// The matrix products of hb_linear and hb_linear_i8: tiles on the matrix units, few rows, sums in parts, and the choice among them.  Both move the same bytes the
// same way, rows in steps of 128 bytes; what the elements are (Op) decides how many k that is, the product and what becomes of a sum.
#pragma once
#include <algorithm>
#include <type_traits>

#include "hb_device.hpp"
#include "hb_host.hpp"
#include "linear_plan.hpp"
#include "token_epilogue.hpp"
#include "token_tiles.hpp"
#include "../wrappers/mfma_i8.hpp"

namespace hb {

// fp16 operands, fp32 sums
struct LinF16 {
    using T = half_t;
    using Elems = half8;                                  // 16 bytes
    using Frag = half8;
    using Acc = floatx4;
    using Sum = float;
    static constexpr int kPer = 8, kK = 64;               // elements in 16 bytes, and in the 128 bytes of a step
    static constexpr uint32_t kOdd = 2;                   // what an address can have over a multiple of four
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ Acc mul(Frag a, Frag b, Acc c) { return mfma16x16x32(a, b, c); }
    static __device__ __forceinline__ uint32_t next(uint32_t odd) { return 8 * odd; }        // to the fifth dword where it is wanted
    static __device__ __forceinline__ u32x4 shift(u32x4 v, int d) { return __builtin_bit_cast(u32x4, shift_in_from_right<true>(__builtin_bit_cast(half8, v), d)); }
    static int halves(int K) { return K; }                // the K of hb_linear whose rows have as many bytes
    static const LinCosts& costs() { return kLinCostsF16; }
};

// 8-bit integers, sums in 32 bits, a scale for each row of both operands.  A fragment is 16 bytes of a lane as above, twice as many k in the time of one product.
struct LinI8 {
    using T = int8_t;
    typedef int8_t Elems __attribute__((ext_vector_type(16)));
    using Frag = intx4;
    using Acc = intx4;
    using Sum = int;
    static constexpr int kPer = 16, kK = 128;
    static constexpr uint32_t kOdd = 3;
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ Acc mul(Frag a, Frag b, Acc c) { return mfma16x16x64i8(a, b, c); }
    static __device__ __forceinline__ uint32_t next(uint32_t odd) { return odd ? 16 : 0; }
    static __device__ __forceinline__ u32x4 shift(u32x4 v, int d) { return shift_in_bytes(v, d); }
    static int halves(int K) { return (K - 1) / 2 + 1; }
    static const LinCosts& costs() { return kLinCostsI8; }
};

template <class Op>
struct LinearArgs {
    const typename Op::T* x;
    const typename Op::T* w;
    const half_t* bias;        // null: none
    const void* residual;      // null: none
    void* out;
    int M, N, K, act;
    int64_t x_pitch, w_pitch, res_pitch, out_pitch;
    int steps;                 // tiles: steps of kK k of one part of the sum (blockIdx.y); the parts' results are out_pitch * M apart
    const float* x_scale;      // LinI8
    const float* w_scale;
};

// A sum of products, rounded to 24 bits, times its scales, and the bias.
template <class S>
__device__ __forceinline__ float lin_scaled(S sum, float xs, float ws, float bias) { return fmaf((float)sum * xs, ws, bias); }

// Four sums of a part.
__device__ __forceinline__ void lin_store_sums(int* to, intx4 v, int count) {
    typedef intx4 intx4_u __attribute__((aligned(4)));
    if (count >= 4) *reinterpret_cast<intx4_u*>(to) = v;
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) to[i] = v[i];
}

// The 16-byte pieces of a row stand in LDS at piece ^ this, so that 16 lanes that read one piece of 16 rows meet no bank twice.
__device__ __forceinline__ int lin_flip(int row) { return (row >> 1) & 7; }

// 16 bytes of adjacent elements.  At addresses that are no multiple of four 16-byte loads take several times as long: the dwords around the elements are
// loaded and moved by what is over (the fifth only where it holds one of them; a dword that holds one is in the same allocation).
template <class Op, LinRows ROWS>
__device__ __forceinline__ u32x4 lin_get(const typename Op::T* q) {
    typedef u32x4 u32x4_u __attribute__((aligned(4)));
    if (ROWS != kLinOdd) return *reinterpret_cast<const u32x4_u*>(q);
    const uint32_t odd = (uint32_t)(uintptr_t)q & Op::kOdd;
    const char* at = reinterpret_cast<const char*>(q) - odd;
    const u32x4 d = *reinterpret_cast<const u32x4_u*>(at);
    const uint32_t e = *reinterpret_cast<const uint32_t*>(at + Op::next(odd)), shift = 8 * odd;
    return u32x4{__builtin_amdgcn_alignbit(d[1], d[0], shift), __builtin_amdgcn_alignbit(d[2], d[1], shift), __builtin_amdgcn_alignbit(d[3], d[2], shift),
                 __builtin_amdgcn_alignbit(e, d[3], shift)};
}
// 16 bytes of a row from k on, zeros from K on: the last ones are loaded from where 16 bytes fit and moved.
template <class Op>
__device__ __forceinline__ u32x4 lin_last(const typename Op::T* row, int k, int K) {
    if (K >= Op::kPer) {                                  // uniform
        const int at = min(k, K - Op::kPer);
        return Op::shift(lin_get<Op, kLinOdd>(row + at), k - at);
    }
    typename Op::Elems r = {};
#pragma unroll
    for (int i = 0; i < Op::kPer; ++i)
        if (k + i < K) r[i] = row[k + i];
    return __builtin_bit_cast(u32x4, r);
}

// The epilogue of a wave: its WM x WN sums leave through a patch of LDS that is its own (TILES x 16 rows of WN floats at a time), because a
// lane holds four columns of one row of a fragment and 16 lanes 16 different rows: from the patch, whole runs of a row are
// finished and stored, 16 bytes a lane.  The 16-byte pieces of a row stand at piece ^ row % 16 (writes meet no bank twice).  Sums of integers meet the scales of
// their rows of x on the way into the patch, where a lane has one row of a fragment: eight values for 128 rows, requested at once.  What begin() requests, finish() waits for.
template <class Op, class O, int WM, int WN, int TILES, int BATCH>
struct LinEnd {
    using Acc = typename Op::Acc;
    static constexpr bool kSums = std::is_same<O, int>::value, kScaled = Op::kScaled && !kSums;      // parts of a sum of integers are stored as they are
    using Patch = typename std::conditional<kSums, Acc, floatx4>::type;
    static_assert(WN >= 32 && (WM / 16) % TILES == 0);
    static constexpr int kFlip = WN / 4 < 16 ? WN / 4 - 1 : 15;
    static constexpr int V = 16 / sizeof(O), kLanes = WN / V, kStep = 64 / kLanes;                   // elements and lanes per row, rows per pass
    static constexpr int kPasses = 16 * TILES / kStep, kBatch = kPasses < BATCH ? kPasses : BATCH;
    typedef O vec __attribute__((ext_vector_type(V), aligned(sizeof(O))));
    int m0, n0, lane, x, count, r0;
    float x_scale[kScaled ? WM / 16 : 1], w_scale[V], bias[kScaled ? 1 : V];
    typedef half_t halves __attribute__((ext_vector_type(V), aligned(2)));
    halves half_bias;          // beside scales, two to a register
    vec ahead[kBatch];         // the residual of a batch of rows is requested while the batch before is finished

    __device__ __forceinline__ void request(const LinearArgs<Op>& p, int first) {
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int64_t m = m0 + first + b * kStep + r0;
            const O* from = static_cast<const O*>(p.residual) + m * p.res_pitch + n0 + x;
            if (m < p.M && first < WM) {
                if (count >= V) ahead[b] = *reinterpret_cast<const vec*>(from);
                else
#pragma unroll
                    for (int i = 0; i < V; ++i) ahead[b][i] = i < count ? from[i] : (O)0.f;
            }
        }
    }
    __device__ __forceinline__ void begin(const LinearArgs<Op>& p, int m0_, int n0_) {
        m0 = m0_;
        n0 = n0_;
        lane = threadIdx.x & 63;
        x = lane % kLanes * V;
        count = p.N - (n0 + x);
        r0 = lane / kLanes;
        if (kScaled) {
#pragma unroll
            for (int j = 0; j < WM / 16; ++j) {
                const int64_t m = (int64_t)m0 + 16 * j + (lane & 15);
                x_scale[j] = p.x_scale[m < p.M ? m : p.M - 1];
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w_scale[i] = 0.f;
            if (!kScaled) bias[i] = 0.f;
        }
        half_bias = halves{};
        if constexpr (kScaled) {
            lin_load<V>(w_scale, p.w_scale + n0 + x, count);
            if (p.bias) {
                if (count >= V) half_bias = *reinterpret_cast<const halves*>(p.bias + n0 + x);
                else
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (i < count) half_bias[i] = p.bias[n0 + x + i];
            }
        } else if (p.bias) {
            lin_load<V>(bias, p.bias + n0 + x, count);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) ahead[b] = vec{};
        if (p.residual) request(p, 0);
    }
    __device__ __forceinline__ void finish(const LinearArgs<Op>& p, O* out, const Acc (&acc)[WN / 16][WM / 16], typename Op::Sum* patch) {
        const int c = lane & 15, g = lane >> 4;
        vec res[kBatch] = {};
#pragma unroll 1
        for (int h = 0; h < WM / 16; h += TILES) {
            tk_for<WM / 16>([&](auto tile) HB_INLINE {
                constexpr int j = decltype(tile)::value;
                if (TILES == WM / 16 || (j / TILES) * TILES == h) {
                    tk_for<WN / 16>([&](auto index) HB_INLINE {
                        constexpr int i = decltype(index)::value;
                        Patch v;
                        if constexpr (kScaled) {
                            Acc t = acc[i][j];
                            asm volatile("" : "+v"(t));       // or all of them would be made floats ahead of the loop
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = (float)t[e] * x_scale[j];
                        } else {
                            v = acc[i][j];
                        }
                        *reinterpret_cast<Patch*>(patch + (16 * (j % TILES) + c) * WN + 4 * ((4 * i + g) ^ (c & kFlip))) = v;
                    });
                    asm volatile("; fragments %0" ::"n"(j));  // keeps the branches apart: merged, they would index registers
                }
            });
            wave_lds_fence();
#pragma unroll 1
            for (int q = 0; q < kPasses; q += kBatch) {
                const int first = 16 * h + q * kStep;     // row of the wave
                if constexpr (kSums) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) {
                        const int r = (q + b) * kStep + r0;
                        const Acc t = *reinterpret_cast<const Acc*>(patch + r * WN + 4 * ((x / 4) ^ (r & kFlip)));
                        const int64_t m = m0 + first + b * kStep + r0;
                        if (m < p.M && count > 0) lin_store_sums(out + m * p.out_pitch + n0 + x, t, count);
                    }
                    continue;
                }
                float v[kBatch][V];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int r = (q + b) * kStep + r0;
#pragma unroll
                    for (int e = 0; e < V; e += 4) {
                        const Patch t = *reinterpret_cast<const Patch*>(patch + r * WN + 4 * (((x + e) / 4) ^ (r & kFlip)));
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[b][e + i] = kScaled ? fmaf(t[i], w_scale[e + i], (float)half_bias[e + i]) : t[i] + bias[kScaled ? 0 : e + i];     // as lin_scaled
                    }
                }
                if (!kScaled && p.residual) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) res[b] = ahead[b];
                    request(p, first + kBatch * kStep);
                }
                lin_act<kBatch * V>(reinterpret_cast<float(&)[kBatch * V]>(v), p.act);
                if (p.residual) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
#pragma unroll
                        for (int i = 0; i < V; ++i) v[b][i] += (float)(kScaled ? ahead : res)[b][i];
                    if (kScaled) request(p, first + kBatch * kStep);         // after it: the scales leave no registers for a copy
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int64_t m = m0 + first + b * kStep + r0;
                    if (m < p.M && count > 0) lin_store<V>(out + m * p.out_pitch + n0 + x, v[b], count);
                }
            }
            wave_lds_fence();
        }
    }
};
constexpr int kLinPatch = 1;                              // fragments of 16 rows in a patch

// Which tile a workgroup takes: groups of 8 tile rows, column after column, in the order in which the workgroups of one XCD follow
// each other, so that what runs there at one time shares rows and columns in its L2.
__device__ __forceinline__ void lin_tile(int wg, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int id = xcd_contiguous(wg, tiles_m * tiles_n);
    const int group = id / (8 * tiles_n), first = 8 * group, rows = min(8, tiles_m - first), in = id - group * 8 * tiles_n;
    tm = first + in % rows;
    tn = in / rows;
}

// A workgroup of (BM / WM) x (BN / WN) waves computes BM x BN outputs, a wave WM x WN of them in products of 16 x 16; the rows
// of w are the product's rows, so that a lane ends with four adjacent n of one m.  Two stages of G steps of 128 bytes of each row take
// turns in LDS.
//
// A lone workgroup of 64 x 64 is bound by the chain of a step (barrier, reads from LDS, products): two steps behind one barrier (1024 x 1024,
// K 1024 8.3 -> 7.2 us; 1920 x 1088, K 1024 11.8 -> 9.9), and more stages without that gain nothing.  Of 128 x 128 two workgroups share a compute
// unit instead.  Rows that are not copied pass through registers (1917 x 1079, K 1023 15.3 us, 16.8 with silu and an fp32 residual; K 1024,
// copied, 11.8), where a second step gains nothing.
// Few k are bound by memory (1M x 64, K 64 with residual: 80 us, 5.0 TB/s); odd rows by their loads, two or three for 16 bytes.
template <class Op, class O, int BM, int BN, int WM, int WN, LinRows ROWS, int G>
__global__ void __launch_bounds__(64 * (BM / WM) * (BN / WN), 1) linear_mfma_kernel(LinearArgs<Op> p) {
    using T = typename Op::T;
    constexpr int kLinK = Op::kK, kPer = Op::kPer;
    constexpr int kWaves = (BM / WM) * (BN / WN), kMT = WM / 16, kNT = WN / 16;
    constexpr int kPieces = (BM + BN) / 8, kOwn = kPieces / kWaves;          // copies of 1 KB (8 rows) per stage, and of a wave
    static_assert(kPieces % kWaves == 0 && BM % 8 == 0);
    constexpr int kStage = (BM + BN) * 128;
    extern __shared__ __attribute__((aligned(128))) char s_tiles[];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    int tm, tn;
    lin_tile(blockIdx.x, (p.M + BM - 1) / BM, (p.N + BN - 1) / BN, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    const int kb = (int)blockIdx.y * p.steps * kLinK, K = p.K - kb, steps = min(p.steps, (K + kLinK - 1) / kLinK);
    const T* const x0 = p.x + m0 * p.x_pitch + kb;
    const T* const w0 = p.w + n0 * p.w_pitch + kb;

    typename Op::Acc acc[kNT][kMT];
#pragma unroll
    for (int i = 0; i < kNT; ++i)
#pragma unroll
        for (int j = 0; j < kMT; ++j) acc[i][j] = typename Op::Acc{0, 0, 0, 0};

    // copies: piece j = rows 8j .. 8j + 7 of the stage (x rows, then w rows); slot `lane` of it is row lane / 8, place lane % 8
    auto row_of = [&](int i) HB_INLINE { return 8 * (wv * kOwn + i) + (lane >> 3); };  // in the stage
    auto chunk_of = [&](int row) HB_INLINE { return (lane & 7) ^ lin_flip(row); };
    static_assert(BM % 16 == 0);                                             // the flip of a w row is that of its place in the stage
    const u32x4 rx = tk_rsrc(x0), rw = tk_rsrc(w0);
    uint32_t off[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int row = row_of(i);
        const bool is_x = row < BM;
        const int at = is_x ? row : row - BM;
        const bool there = is_x ? m0 + at < p.M : n0 + at < p.N;
        off[i] = there ? (uint32_t)(at * (is_x ? p.x_pitch : p.w_pitch) * sizeof(T)) + 16 * chunk_of(row) : kTkOutside;
    }
    const uint32_t lds0 = tk_lds_addr(s_tiles);
    auto request = [&](int step, int buf) HB_INLINE {
        const int k0 = step * kLinK;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            uint32_t o = off[i];
            if (k0 + kLinK > K && k0 + kPer * chunk_of(row_of(i)) >= K) o = kTkOutside;
            const bool is_x = 8 * (wv * kOwn + i) < BM;                      // uniform
            tk_dma16(is_x ? rx : rw, o, (uint32_t)k0 * sizeof(T), lds0 + buf * kStage + 1024 * (wv * kOwn + i));
        }
    };
    // or they pass through registers; rows beyond the matrix repeat its last one (their sums are dropped)
    constexpr int kHeld = ROWS == kLinCopied ? 1 : kOwn;
    u32x4 held[kHeld];                                                       // as lin_get loads them, moved on their way to LDS
    uint32_t next[kHeld];
    const T* from[kHeld];
    uint32_t odd[kHeld];
    if (ROWS != kLinCopied) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int row = row_of(i);
            from[i] = row < BM ? x0 + min(row, p.M - 1 - m0) * p.x_pitch : w0 + min(row - BM, p.N - 1 - n0) * p.w_pitch;
            from[i] += kPer * chunk_of(row);
            odd[i] = ROWS == kLinOdd ? (uint32_t)(uintptr_t)from[i] & Op::kOdd : 0u;
        }
    }
    auto fetch = [&](int step) HB_INLINE {                                   // a step that is all there
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const char* at = reinterpret_cast<const char*>(from[i] + step * kLinK) - odd[i];
            typedef u32x4 u32x4_u __attribute__((aligned(4)));
            held[i] = *reinterpret_cast<const u32x4_u*>(at);
            if (ROWS == kLinOdd) next[i] = *reinterpret_cast<const uint32_t*>(at + Op::next(odd[i]));
        }
    };
    auto fetch_last = [&](int step) HB_INLINE {                              // the rest of K, in place
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int k = step * kLinK + kPer * chunk_of(row_of(i));
            held[i] = lin_last<Op>(from[i] + step * kLinK - k, k, K);
        }
    };
    auto put = [&](int buf, auto moved) HB_INLINE {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            u32x4 v = held[i];
            if (ROWS == kLinOdd && decltype(moved)::value) {
                const uint32_t shift = 8 * odd[i];
                v = u32x4{__builtin_amdgcn_alignbit(v[1], v[0], shift), __builtin_amdgcn_alignbit(v[2], v[1], shift), __builtin_amdgcn_alignbit(v[3], v[2], shift),
                          __builtin_amdgcn_alignbit(next[i], v[3], shift)};
            }
            *reinterpret_cast<u32x4*>(s_tiles + buf * kStage + 1024 * (wv * kOwn + i) + 16 * lane) = v;
        }
    };

    const int wm = wv / (BN / WN) * WM, wn = wv % (BN / WN) * WN;
    const uint32_t at_x = (uint32_t)(wm + c) * 128 + 16 * (g ^ lin_flip(c)), at_w = (uint32_t)(BM + wn + c) * 128 + 16 * (g ^ lin_flip(c));
    // scales and the first of the residual are requested ahead of the rows (32768 x 1024, K 1024 with a residual 66 -> 62 us), where there are registers for them
    LinEnd<Op, O, WM, WN, kLinPatch, 4> end;
    constexpr bool kEarly = Op::kScaled && sizeof(O) == 2;
    if (kEarly) end.begin(p, m0 + wm, n0 + wn);
    auto compute = [&](int buf) HB_INLINE {
        const char* base = s_tiles + buf * kStage;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            typename Op::Frag a[kNT], b[kMT];
#pragma unroll
            for (int j = 0; j < kMT; ++j) b[j] = *reinterpret_cast<const typename Op::Frag*>(base + (at_x ^ (64 * ks)) + 2048 * j);
#pragma unroll
            for (int i = 0; i < kNT; ++i) a[i] = *reinterpret_cast<const typename Op::Frag*>(base + (at_w ^ (64 * ks)) + 2048 * i);
#pragma unroll
            for (int i = 0; i < kNT; ++i)
#pragma unroll
                for (int j = 0; j < kMT; ++j) acc[i][j] = Op::mul(a[i], b[j], acc[i][j]);
        }
    };
    if (ROWS == kLinCopied) {
        int buf = 0;
#pragma unroll
        for (int i = 0; i < G; ++i)
            if (i == 0 || i < steps) request(i, i);
        for (int s = 0; s < steps; s += G) {
            tk_wait_loads<0>();
            lds_barrier();
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (s + G + i < steps) request(s + G + i, G - buf + i);
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (i == 0 || s + i < steps) compute(buf + i);
            buf = G - buf;
        }
    } else if (kOwn > 2) {
        auto take = [&](int step) HB_INLINE {
            if (step * kLinK + kLinK <= K) {
#pragma unroll
                for (int i = 0; i < kOwn; ++i) held[i] = lin_get<Op, ROWS>(from[i] + step * kLinK);
            } else {
                fetch_last(step);
            }
        };
        take(0);
        put(0, TkInt<0>{});
        for (int s = 0; s < steps; ++s) {
            lds_barrier();
            if (s + 1 < steps) take(s + 1);
            compute(s & 1);
            if (s + 1 < steps) put((s + 1) & 1, TkInt<0>{});
        }
    } else {
        // odd rows are moved behind the products, so that these need not wait for them (1917 x 1079, K 1023, no activation 19.2 -> 16.4 us; with more rows a wave, in
        // the larger tiles, that is slower: 4000 x 4001, K 2001 119 -> 124)
        const int whole = min(steps, K / kLinK);
        if (whole > 0) {
            fetch(0);
            put(0, TkInt<1>{});
        } else {
            fetch_last(0);
            put(0, TkInt<0>{});
        }
        int s = 0;
        for (; s + 1 < whole; ++s) {
            lds_barrier();
            fetch(s + 1);
            compute(s & 1);
            put((s + 1) & 1, TkInt<1>{});
        }
        if (s + 1 < steps) {
            lds_barrier();
            fetch_last(s + 1);
            compute(s & 1);
            put((s + 1) & 1, TkInt<0>{});
            ++s;
        }
        lds_barrier();
        compute(s & 1);
    }
    lds_barrier();
    if (!kEarly) end.begin(p, m0 + wm, n0 + wn);
    end.finish(p, static_cast<O*>(p.out) + (int64_t)blockIdx.y * p.M * p.out_pitch, acc, reinterpret_cast<typename Op::Sum*>(s_tiles) + 16 * kLinPatch * WN * wv);
}

// The large tile: 256 x 256 outputs, four waves of 128 x 128, one to a SIMD.  A wave reads 16 fragments from LDS for 64 products (half of
// what eight waves of 128 x 64 would read), and nothing but its own products hides these reads: while the 64 products of one half of a
// stage run, the fragments of the next half are on their way, one read or copy between two products.  A workgroup stays and takes tile
// after tile, and the first two stages of the next tile are copied while the last one's results leave.
// 8192 x 8192, K 2048 with gelu_tanh: 243 us, 1.13 PFLOP/s at the 2.2 GHz that its power leaves, the matrix units busy for 0.48 of the time (tiles
// of 128 x 128 280 us); 4096 x 4096, K 4096 111 us (131), K 2048 61 (69), K 1024 35 (40).  Each round of tiles costs some 9 us beside its products.
// Of integers 8192 x 8192, K 2048 with gelu_tanh: 138 to 148 us on one card and another, 1.86 to 1.99 POPS (163 us with fp32 output), some 95 of them products and the rest four epilogues, 22 of that the results at the memory's rate; K 8192 without
// an activation 434 to 450 us, 2.4 to 2.5 POPS; 32768 x 1024, K 1024 with a residual 60.6 to 62.8 us, products 27 and memory 34, one after the other.
constexpr int kLinLargeLds = 160 * 1024;                                    // two stages of 64 KB and 8 KB of patch a wave
template <class Op, class O>
__global__ void __launch_bounds__(256, 1) linear_large_kernel(LinearArgs<Op> p) {
    using T = typename Op::T;
    using Frag = typename Op::Frag;
    constexpr int kLinK = Op::kK, kPer = Op::kPer;
    constexpr int BM = 256, BN = 256, kOwn = 16, kStage = 65536;
    extern __shared__ __attribute__((aligned(128))) char s_tiles[];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN, tiles = tiles_m * tiles_n;
    const int steps = p.steps;

    // waves 0 and 1 copy x, 2 and 3 w: 16 pieces of 8 rows each, two steps ahead of the products
    const bool is_x = wv < 2;
    const int r0 = 128 * (wv & 1) + (lane >> 3);
    const uint32_t pitch = (uint32_t)(is_x ? p.x_pitch : p.w_pitch);
    auto chunk_of = [&](int i) HB_INLINE { return (lane & 7) ^ lin_flip(r0 + 8 * i); };
    const uint32_t lds0 = tk_lds_addr(s_tiles) + 16384 * wv;
    int ahead_tile = blockIdx.x, ahead_step = 0;          // what is requested next
    uint32_t ahead_at = lds0;
    u32x4 rsrc;
    uint32_t off[kOwn];
    // before the requests of a step: where a tile begins, and of the last step only the pieces below K
    auto aim = [&]() HB_INLINE {
        if (ahead_step == 0) {
            if (ahead_tile >= tiles) {
                rsrc = u32x4{0, 0, 0, 0x00020000u};       // zeros
            } else {
                int tm, tn;
                lin_tile(ahead_tile, tiles_m, tiles_n, tm, tn);
                const int limit = is_x ? p.M - tm * BM : p.N - tn * BN;
                rsrc = tk_rsrc(is_x ? p.x + (int64_t)tm * BM * p.x_pitch : p.w + (int64_t)tn * BN * p.w_pitch);
#pragma unroll
                for (int i = 0; i < kOwn; ++i) off[i] = r0 + 8 * i < limit ? ((r0 + 8 * i) * pitch) * (uint32_t)sizeof(T) + 16 * chunk_of(i) : kTkOutside;
            }
        }
        if (ahead_step == steps - 1 && steps * kLinK > p.K) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
                if (ahead_step * kLinK + kPer * chunk_of(i) >= p.K) off[i] = kTkOutside;
        }
    };
    auto request = [&](int i) HB_INLINE { tk_dma16(rsrc, off[i], (uint32_t)ahead_step * 128, ahead_at + 1024 * i); };
    auto advance = [&]() HB_INLINE {
        ahead_at ^= kStage;                               // the stages are 64 KB each, from a multiple of 128 KB on
        if (++ahead_step == steps) {
            ahead_step = 0;
            ahead_tile += gridDim.x;
        }
    };

    const int wm = (wv >> 1) * 128, wn = (wv & 1) * 128;
    uint32_t at_x = tk_lds_addr(s_tiles) + (uint32_t)(wm + c) * 128 + 16 * (g ^ lin_flip(c));
    uint32_t at_w = tk_lds_addr(s_tiles) + (uint32_t)(BM + wn + c) * 128 + 16 * (g ^ lin_flip(c));
    // fragments: 8 of w, each replaced by that of the next half once its 8 products are done, and 8 of x for this half and for the next
    Frag fw[8], fx[2][8];
    auto read = [&](uint32_t at) HB_INLINE { return *reinterpret_cast<const __attribute__((address_space(3))) Frag*>(at); };
    auto pin = []() HB_INLINE { __builtin_amdgcn_sched_barrier(0); };

    aim();
    tk_for<kOwn>([&](auto i) HB_INLINE { request(decltype(i)::value); });
    advance();
    aim();
    tk_for<kOwn>([&](auto i) HB_INLINE { request(decltype(i)::value); });
    advance();
    tk_wait_loads<kOwn>();
    lds_barrier();
    tk_for<8>([&](auto index) HB_INLINE {
        constexpr int i = decltype(index)::value;
        fx[0][i] = read(at_x + 2048 * i);
        fw[i] = read(at_w + 2048 * i);
    });
#pragma unroll 1
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        typename Op::Acc acc[8][8];
        tk_for<64>([&](auto index) HB_INLINE {
            constexpr int k = decltype(index)::value;
            acc[k / 8][k % 8] = typename Op::Acc{0, 0, 0, 0};
        });
        // products k of a half: FROM <= k < TO, fragment k / 8 of w with fragment k % 8 of x
        auto products = [&](auto half, auto from, auto to, auto between) HB_INLINE {
            constexpr int kFrom = decltype(from)::value;
            tk_for<decltype(to)::value - kFrom>([&](auto index) HB_INLINE {
                constexpr int k = kFrom + decltype(index)::value;
                acc[k / 8][k % 8] = Op::mul(fw[k / 8], fx[decltype(half)::value][k % 8], acc[k / 8][k % 8]);
                pin();
                between(TkInt<k>{});
                pin();
            });
        };
#pragma unroll 1
        for (int s = 0; s < steps; ++s) {
#pragma unroll
            for (int k = 0; k < 64; ++k) asm volatile("" : "+a"(acc[k / 8][k % 8]));        // the sums live in the accumulation registers
            const uint32_t x1 = at_x ^ 64, w1 = at_w ^ 64;
            products(TkInt<0>{}, TkInt<0>{}, TkInt<64>{}, [&](auto index) HB_INLINE {
                constexpr int k = decltype(index)::value;
                if constexpr (k % 8 == 2) fx[1][k / 8] = read(x1 + 2048 * (k / 8));
                if constexpr (k % 8 == 7) fw[k / 8] = read(w1 + 2048 * (k / 8));
            });
            products(TkInt<1>{}, TkInt<0>{}, TkInt<8>{}, [&](auto) HB_INLINE {});
            // the other half of this stage is in registers, and the next stage in LDS, for all waves
            tk_wait_loads<0>();
            lds_barrier();
            aim();
            at_x ^= kStage;
            at_w ^= kStage;
            fw[0] = read(at_w);
            pin();
            products(TkInt<1>{}, TkInt<8>{}, TkInt<64>{}, [&](auto index) HB_INLINE {
                constexpr int k = decltype(index)::value;
                if constexpr (k % 4 == 1 && k < 40) fx[0][(k - 8) / 4] = read(at_x + 2048 * ((k - 8) / 4));
                if constexpr (k % 8 == 7) fw[k / 8] = read(at_w + 2048 * (k / 8));
                if constexpr (k % 2 == 0 && k < 40) request((k - 8) / 2);
            });
            advance();
        }
        int tm, tn;
        lin_tile(tile, tiles_m, tiles_n, tm, tn);
        LinEnd<Op, O, 128, 128, kLinPatch, 4> end;
        end.begin(p, tm * BM + wm, tn * BN + wn);
        end.finish(p, static_cast<O*>(p.out), acc, reinterpret_cast<typename Op::Sum*>(s_tiles + 2 * kStage) + 2048 * wv);
    }
    tk_wait_loads<0>();                                   // nothing may arrive in LDS that is no longer this workgroup's
}

// The parts of a split sum, added in their order, and the epilogue: a thread per four outputs.  Bound by its launch (2.6 us) and by reading the
// parts, which the caches hold, at some 7 TB/s.
template <class Op, class O>
__global__ void __launch_bounds__(256) linear_join_kernel(LinearArgs<Op> p, const typename Op::Sum* parts, int count) {
    constexpr int V = 4;
    const int per_row = (p.N + V - 1) / V;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = t / per_row;
    const int n = (int)(t - m * per_row) * V, have = p.N - n;
    if (m >= p.M) return;
    typename Op::Sum sum[V] = {}, part[V];
    float v[V], q[V], res[V];
    if (p.residual) lin_load<V>(res, static_cast<const O*>(p.residual) + m * p.res_pitch + n, have);
    const typename Op::Sum* from = parts + m * p.N + n;
#pragma unroll 4
    for (int s = 0; s < count; ++s) {
        lin_load<V>(part, from + s * ((int64_t)p.M * p.N), have);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += part[i];
    }
    float bias[V] = {};
    if (p.bias) lin_load<V>(bias, p.bias + n, have);
    if (Op::kScaled) {
        const float scale = p.x_scale[m];
        lin_load<V>(q, p.w_scale + n, have);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = lin_scaled(sum[i], scale, q[i], bias[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = sum[i] + bias[i];
    }
    lin_act<V>(v, p.act);
    if (p.residual) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += res[i];
    }
    lin_store<V>(static_cast<O*>(p.out) + m * p.out_pitch + n, v, have);
}

// Few rows of x: bound by reading w once.  A workgroup takes 16 rows of w and all of x; its waves take blocks of 128 bytes of each row in turn, straight
// from memory into fragments (a row of w is 16 bytes of four lanes, twice: whole lines), and add their sums up in LDS.  One row: N 4096, K 1024
// 3.7 us (the launch), K 4096 7.2 (4.7 TB/s), K 11008 17.4 (5.2 TB/s).  Few w rows leave compute units idle: k is split then.
template <class Op, class O, int MT, int WAVES, LinRows ROWS>
__global__ void __launch_bounds__(64 * WAVES) linear_rows_kernel(LinearArgs<Op> p) {
    using T = typename Op::T;
    using Acc = typename Op::Acc;
    constexpr int kLinK = Op::kK, kPer = Op::kPer;
    __shared__ __attribute__((aligned(16))) typename Op::Sum s_sum[WAVES][16 * MT][20];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int n0 = (int)blockIdx.x * 16, kb = (int)blockIdx.y * p.steps * kLinK, K = min(p.K - kb, p.steps * kLinK);
    const T *const w = p.w + (int64_t)min(n0 + c, p.N - 1) * p.w_pitch + kb + kPer * g, *x[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) x[j] = p.x + (int64_t)min(16 * j + c, p.M - 1) * p.x_pitch + kb + kPer * g;
    Acc acc[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[j] = Acc{0, 0, 0, 0};
    // U blocks at a time: load(row, its u-th block + h) of all of them before the first product
    auto blocks = [&](auto count, auto load) HB_INLINE {
        constexpr int U = decltype(count)::value;
        u32x4 a[U][2], b[U][MT][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                a[u][h] = load(w, u, kLinK / 2 * h);
#pragma unroll
                for (int j = 0; j < MT; ++j) b[u][j][h] = load(x[j], u, kLinK / 2 * h);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < MT; ++j) acc[j] = Op::mul(__builtin_bit_cast(typename Op::Frag, a[u][h]), __builtin_bit_cast(typename Op::Frag, b[u][j][h]), acc[j]);
    };
    constexpr int kAtOnce = MT == 1 ? 4 : 2;
    const int whole = K / kLinK;
    int s = wv;
    auto inside = [&](const T* q, int u, int h) HB_INLINE { return lin_get<Op, ROWS>(q + (s + u * WAVES) * kLinK + h); };
    for (; s + (kAtOnce - 1) * WAVES < whole; s += kAtOnce * WAVES) blocks(TkInt<kAtOnce>{}, inside);
    for (; s < whole; s += WAVES) blocks(TkInt<1>{}, inside);
    if (s == whole && K % kLinK) blocks(TkInt<1>{}, [&](const T* q, int, int h) HB_INLINE { return lin_last<Op>(q - kPer * g, s * kLinK + h + kPer * g, K); });
#pragma unroll
    for (int j = 0; j < MT; ++j) *reinterpret_cast<Acc*>(&s_sum[wv][16 * j + c][4 * g]) = acc[j];
    __syncthreads();
    for (int t = threadIdx.x; t < 256 * MT; t += 64 * WAVES) {
        const int r = t / 16, n = n0 + t % 16;
        if (r >= p.M || n >= p.N) continue;
        typename Op::Sum sum = 0;
#pragma unroll
        for (int q = 0; q < WAVES; ++q) sum += s_sum[q][r][t % 16];
        if constexpr (std::is_same<O, int>::value) {      // a part of a sum of integers
            static_cast<int*>(p.out)[((int64_t)blockIdx.y * p.M + r) * p.out_pitch + n] = sum;
            continue;
        }
        const float bias = p.bias ? (float)p.bias[n] : 0.f;
        float v = Op::kScaled ? lin_scaled(sum, p.x_scale[r], p.w_scale[n], bias) : (float)sum + bias;
        v = linear_act(v, p.act);
        if (p.residual) v += (float)static_cast<const O*>(p.residual)[r * p.res_pitch + n];
        static_cast<O*>(p.out)[((int64_t)blockIdx.y * p.M + r) * p.out_pitch + n] = (O)v;
    }
}
template <class Op, class O, int MT, int WAVES, LinRows ROWS>
static hb_status linear_launch_rows(const LinearArgs<Op>& a, int parts, hipStream_t st) {
    hipLaunchKernelGGL((linear_rows_kernel<Op, O, MT, WAVES, ROWS>), dim3(ceil_div(a.N, 16), parts), dim3(64 * WAVES), 0, st, a);
    return launch_status();
}

template <class Op, class O>
static hb_status linear_launch_large(const LinearArgs<Op>& a, hipStream_t st) {
    auto kernel = linear_large_kernel<Op, O>;
    const int64_t tiles = (int64_t)ceil_div(a.M, 256) * ceil_div(a.N, 256);
    if (tiles > 0x3fffffff) return HB_ERR_UNSUPPORTED;
    if (hb_status s = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), kLinLargeLds)) return s;
    const int wgs = (int)std::min<int64_t>(tiles, num_cu());
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), kLinLargeLds, st, a);
    return launch_status();
}

template <class Op, class O, int BM, int BN, int WM, int WN, LinRows ROWS, int G>
static hb_status linear_launch(const LinearArgs<Op>& a, int parts, hipStream_t st) {
    const int64_t tiles = (int64_t)ceil_div(a.M, BM) * ceil_div(a.N, BN);
    constexpr int kThreads = 64 * (BM / WM) * (BN / WN);
    static_assert(kThreads == (BM == 128 && BN == 64 ? kLinThreads[kLinTile128x64] : BM == 64 ? kLinThreads[kLinTile64] : kLinThreads[kLinTile128]));
    if (!launch_holds((double)tiles, kThreads)) return HB_ERR_UNSUPPORTED;
    auto kernel = linear_mfma_kernel<Op, O, BM, BN, WM, WN, ROWS, G>;
    // one step needs one stage, and twice as many workgroups are on a compute unit (1M x 64, K 64, residual: 101 -> 93 us)
    const int kStages = (BM + BN) * 128 * std::min(a.steps > G ? 2 * G : G, a.steps);
    constexpr int kPatches = 64 * kLinPatch * WN * (BM / WM) * (BN / WN);
    const int kLds = kStages > kPatches ? kStages : kPatches;
    if (kLds > 65536)
        if (hb_status s = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), kLds)) return s;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles, parts), dim3(kThreads), kLds, st, a);
    return launch_status();
}

// A plan's kernel on all of the sum (parts 1, the call's own output) or on its parts (sums to the workspace).
template <class Op, class O>
static hb_status linear_run(const LinPlan& plan, LinRows rows, const LinearArgs<Op>& a, int parts, hipStream_t st) {
    const bool odd = rows == kLinOdd;
    switch (plan.kernel) {
        case kLinRows16: return odd ? linear_launch_rows<Op, O, 1, 16, kLinOdd>(a, parts, st) : linear_launch_rows<Op, O, 1, 16, kLinEven>(a, parts, st);
        case kLinRows32: return odd ? linear_launch_rows<Op, O, 2, 8, kLinOdd>(a, parts, st) : linear_launch_rows<Op, O, 2, 8, kLinEven>(a, parts, st);
        case kLinRows64: return odd ? linear_launch_rows<Op, O, 4, 8, kLinOdd>(a, parts, st) : linear_launch_rows<Op, O, 4, 8, kLinEven>(a, parts, st);
        case kLinTile64:
            return rows == kLinCopied ? linear_launch<Op, O, 64, 64, 16, 32, kLinCopied, 2>(a, parts, st)
                   : odd              ? linear_launch<Op, O, 64, 64, 16, 32, kLinOdd, 1>(a, parts, st)
                                      : linear_launch<Op, O, 64, 64, 16, 32, kLinEven, 1>(a, parts, st);
        case kLinTile128x64: return odd ? linear_launch<Op, O, 128, 64, 32, 64, kLinOdd, 1>(a, parts, st) : linear_launch<Op, O, 128, 64, 32, 64, kLinEven, 1>(a, parts, st);
        case kLinTile128: return rows == kLinCopied ? linear_launch<Op, O, 128, 128, sizeof(O) == 2 && Op::kScaled ? 32 : 64, sizeof(O) == 2 && Op::kScaled ? 64 : 32, kLinCopied, 1>(a, parts, st) : linear_launch<Op, O, 128, 128, 64, 32, kLinOdd, 1>(a, parts, st);
        default: return linear_launch_large<Op, O>(a, st);
    }
}
template <class Op, class O>
static hb_status linear_call(const LinearArgs<Op>& a, void* workspace, size_t workspace_bytes, hipStream_t st) {
    const int64_t pitches = a.x_pitch | a.w_pitch;
    const LinRows rows = aligned_to(a.x, 16) && aligned_to(a.w, 16) && (pitches | a.K) % Op::kPer == 0 ? kLinCopied
                         : aligned_to(a.x, 4) && aligned_to(a.w, 4) && pitches % (Op::kPer / 4) == 0        ? kLinEven
                                                                                                : kLinOdd;
    if (const size_t need = linear_workspace(a.M, a.N, Op::halves(a.K), Op::costs()))
        if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < need) return HB_ERR_WORKSPACE;
    const LinPlan plan = linear_plan(a.M, a.N, Op::halves(a.K), rows, Op::costs());
    LinearArgs<Op> b = a;
    b.steps = plan.steps;
    if (plan.parts == 1) return linear_run<Op, O>(plan, rows, b, 1, st);
    b.out = workspace;
    b.out_pitch = a.N;
    b.bias = nullptr;
    b.residual = nullptr;
    b.act = HB_ACT_NONE;
    if (hb_status s = linear_run<Op, typename Op::Sum>(plan, rows, b, plan.parts, st)) return s;
    const int64_t blocks = ((int64_t)a.M * ceil_div(a.N, 4) + 255) / 256;
    hipLaunchKernelGGL((linear_join_kernel<Op, O>), dim3((unsigned)blocks), dim3(256), 0, st, a, static_cast<const typename Op::Sum*>(workspace), plan.parts);
    return launch_status();
}

}  // namespace hb
