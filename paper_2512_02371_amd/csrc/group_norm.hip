// hb_group_norm: group norm with an activation, channels last.
#include <math.h>

#include "group_norm_plan.hpp"
#include "hb_device.hpp"
#include "hb_host.hpp"
#include "token_epilogue.hpp"

namespace hb {

// Division by a number that the host knows: the product with floor(2^32 / d) is the quotient or one less.
struct NormDiv {
    uint32_t d, m;
    __device__ __forceinline__ uint32_t by(uint32_t a, uint32_t& rest) const {
        uint32_t q = __umulhi(a, m);
        rest = a - q * d;
        if (rest >= d) rest -= d, ++q;
        return q;
    }
};
static NormDiv norm_div(int d) { return {(uint32_t)d, d == 1 ? 0xffffffffu : (uint32_t)(((uint64_t)1 << 32) / d)}; }

struct NormArgs {
    const void* x;
    void* out;
    const half_t* weight;      // null: ones
    const half_t* bias;        // null: zeros
    float2* parts;             // mean and sum of squares of each chunk: [image][group][chunk]
    float2* stats;             // mean and 1 / sqrt(var + eps): [image][group]
    float eps;
    int act;
    int N, P, C, G, D;
    int64_t x_image, x_row, out_image, out_row;
    int pixels, groups, images, width, rows, blocks, passes, chunk, chunks;    // as in NormPlan
    int apply_chunk, apply_chunks;
    int log_pixels;
    int lanes_row;             // rows side by side in a workgroup
    int log_lanes;             // lanes that add up a group: 2^this
    int size;                  // most entries of a group in a row
    int step_d, step_r;        // these lanes in entries and rows
    NormDiv by_all, by_width, by_size, by_D, by_blocks, by_chunks, by_apply_chunks;     // images * width, ...
    double inverse_P;
    int stream;                // results past the caches
};

template <class X>
struct NormVec {
    static constexpr int V = 16 / sizeof(X);
    typedef X type __attribute__((ext_vector_type(V), aligned(sizeof(X))));
};

// Where a lane stands.
struct NormLane {
    int row;                   // of the workgroup
    int image, at;             // image of the workgroup, first channel in the row of its block
    bool there;
    int valid, valid_last;     // elements of its vector in a row, and in the image's last row
};
template <int V>
__device__ __forceinline__ NormLane norm_lane(const NormArgs& p, int first_image, int block) {
    NormLane l;
    uint32_t column, at;
    l.row = p.by_all.by(threadIdx.x, column);
    l.image = p.by_width.by(column, at);
    l.at = at * V;
    const int channels = min(p.groups, p.G - block * p.groups) * p.D, length = p.pixels * channels;
    l.there = l.row < p.lanes_row && first_image + l.image < p.N && l.at < length;
    l.valid = max(0, min(V, length - l.at));
    l.valid_last = max(0, min(V, (p.P - (p.rows - 1) * p.pixels) * channels - l.at));
    return l;
}

// N elements, put at AT of a vector.
template <int AT, int N, class vec, class T>
__device__ __forceinline__ void norm_piece(vec& r, const T* from) {
    typedef T piece __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    const piece q = *reinterpret_cast<const piece*>(from);
#pragma unroll
    for (int i = 0; i < N; ++i) r[AT + i] = q[i];
}
// V adjacent elements, zeros from `valid` on; `from` is not read where that is 0.  What is less than a vector comes in pieces of four, two and one.
template <class X, bool FULL>
__device__ __forceinline__ typename NormVec<X>::type norm_load(const X* from, int valid) {
    using vec = typename NormVec<X>::type;
    constexpr int V = NormVec<X>::V;
    if (FULL || valid == V) return *reinterpret_cast<const vec*>(from);
    typedef X whole __attribute__((ext_vector_type(V)));
    whole r = {};
    if (V == 8 && valid & 4) {
        norm_piece<0, 4>(r, from);
        if (valid & 2) norm_piece<V == 8 ? 4 : 0, 2>(r, from + 4);
        if (valid == 7) norm_piece<V == 8 ? 6 : 0, 1>(r, from + 6);
        if (valid == 5) norm_piece<V == 8 ? 4 : 0, 1>(r, from + 4);
    } else {
        if (valid & 2) norm_piece<0, 2>(r, from);
        if (valid == 3) norm_piece<2, 1>(r, from + 2);
        if (valid == 1) norm_piece<0, 1>(r, from);
    }
    return r;
}

// What a lane leaves of its V elements for the sums of their groups: an entry for all of them where a vector is of one group (kNormOne), two where groups are as wide as a
// vector or wider (kNormTwo: what belongs to the first element's group, and what to the next), else one for each.
enum NormKind { kNormOne, kNormTwo, kNormEach };
template <NormKind KIND, int V>
constexpr int kNormEntries = KIND == kNormOne ? 1 : KIND == kNormTwo ? 2 : V;

// f(index, whether there is one) for the entries of group q of the workgroup that belong to one of the lanes that add it up.  A row's entries are adjacent; a group has p.size of
// them at most, once for each pixel of a row.
template <int V, NormKind KIND, class F>
__device__ __forceinline__ void norm_entries(const NormArgs& p, int q, int lane, F f) {
    constexpr int E = kNormEntries<KIND, V>;
    const int image = p.images > 1 ? q / (unsigned)p.groups : 0, first = (q - image * p.groups) * p.D;
    const int length = p.images * p.width * E, base = image * p.width * E;
    uint32_t begin;
    int r = p.by_size.by(lane, begin), d = begin;
    const int total = (p.lanes_row << p.log_pixels) * p.size, lanes = 1 << p.log_lanes;
#pragma unroll 4
    for (int left = (total - lane + lanes - 1) >> p.log_lanes; left > 0; --left) {
        const int row = r >> p.log_pixels, from = first + (r - (row << p.log_pixels)) * p.C;         // the group's first element in the row
        bool there = true;
        int e;
        if (KIND == kNormTwo) {
            const int vector = from / V + d;
            there = vector * V < from + p.D;
            e = there ? row * length + base + 2 * vector + (vector * V < from) : 0;
        } else {
            e = row * length + base + (KIND == kNormOne ? from / V : from) + d;
        }
        f(e, there);
        d += p.step_d;
        r += p.step_r + (d >= p.size);
        d -= d >= p.size ? p.size : 0;
    }
}
// A lane's entries of V values; `cut`: how many belong to the first element's group.
template <int V, NormKind KIND>
__device__ __forceinline__ void norm_fold(const float (&v)[KIND == kNormOne ? 1 : V], int cut, float* to) {
    if (KIND == kNormTwo) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a += i < cut ? v[i] : 0.f;
            b += i < cut ? 0.f : v[i];
        }
        to[0] = a;
        to[1] = b;
    } else {
#pragma unroll
        for (int i = 0; i < kNormEntries<KIND, V>; ++i) to[i] = v[i];
    }
}
// Sum over the 2^log_lanes lanes that share a group, the same in all of them.  Within 16 lanes by their neighbours' registers, then between quarters and halves of the
// wave; through LDS each step would wait for it.
template <int CTRL>
__device__ __forceinline__ float norm_dpp(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float norm_lanes_sum(float v, int log_lanes) {
    if (log_lanes > 0) v = norm_dpp<0xb1>(v);             // quad_perm 1 0 3 2
    if (log_lanes > 1) v = norm_dpp<0x4e>(v);             // quad_perm 2 3 0 1
    if (log_lanes > 2) v = norm_dpp<0x141>(v);            // row_half_mirror: the other four of eight
    if (log_lanes > 3) v = norm_dpp<0x140>(v);            // row_mirror: the other eight of 16
    if (log_lanes > 4) {
        const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
        v = __builtin_bit_cast(float, (int)s[0]) + __builtin_bit_cast(float, (int)s[1]);
    }
    if (log_lanes > 5) {
        const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
        v = __builtin_bit_cast(float, (int)s[0]) + __builtin_bit_cast(float, (int)s[1]);
    }
    return v;
}

// The groups of a lane's elements in the workgroup, their channels in the image, and how many are of the first one's group.
template <int V, bool ONE>
__device__ __forceinline__ int norm_channels(const NormArgs& p, const NormLane& l, int block, int (&group)[ONE ? 1 : V], uint32_t (&channel)[V]) {
    int c = p.pixels > 1 ? l.at % (unsigned)p.C : l.at;
    uint32_t in;
    int g = p.by_D.by(c, in), d = in;
    const int own = min(p.groups, p.G - block * p.groups), first = block * p.groups * p.D, cut = min(V, p.D - d);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        channel[i] = first + min(c, own * p.D - 1);
        if (!ONE || i == 0) group[ONE ? 0 : i] = l.image * p.groups + min(g, own - 1);
        ++c;
        if (++d == p.D) d = 0, ++g;
        if (p.pixels > 1 && c == p.C) c = 0, g = 0, d = 0;
    }
    return cut;
}

// The weights or biases of a lane's channels; `none` where there are none.
template <int V>
struct NormHalves {
    typedef half_t type __attribute__((ext_vector_type(V), aligned(2)));
};
template <int V>
__device__ __forceinline__ typename NormHalves<V>::type norm_per_channel(const half_t* from, float none, const uint32_t (&channel)[V], bool adjacent) {
    typename NormHalves<V>::type r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (half_t)none;
    if (from) {
        if (adjacent) {
            r = *reinterpret_cast<const typename NormHalves<V>::type*>(from + channel[0]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) r[i] = from[channel[i]];
        }
    }
    return r;
}

template <class O, int V>
__device__ __forceinline__ void norm_store(O* to, const float (&v)[V], int valid, bool stream) {
    typedef O vec __attribute__((ext_vector_type(V), aligned(sizeof(O))));
    if (valid == V) {
        vec q;
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = (O)v[i];
        if (stream) __builtin_nontemporal_store(q, reinterpret_cast<vec*>(to));
        else *reinterpret_cast<vec*>(to) = q;
    } else {                                              // in pieces of four, two and one
        auto piece = [&](auto at, auto n) HB_INLINE {
            constexpr int AT = decltype(at)::value, N = decltype(n)::value;
            typedef O part __attribute__((ext_vector_type(N), aligned(sizeof(O))));
            part q;
#pragma unroll
            for (int i = 0; i < N; ++i) q[i] = (O)v[AT + i];
            *reinterpret_cast<part*>(to + AT) = q;
        };
        constexpr int H = V == 8 ? 4 : 0;
        if (V == 8 && valid & 4) {
            piece(TkInt<0>{}, TkInt<4>{});
            if (valid & 2) piece(TkInt<H>{}, TkInt<2>{});
            if (valid == 7) piece(TkInt<H + 2>{}, TkInt<1>{});
            if (valid == 5) piece(TkInt<H>{}, TkInt<1>{});
        } else {
            if (valid & 2) piece(TkInt<0>{}, TkInt<2>{});
            if (valid == 3) piece(TkInt<2>{}, TkInt<1>{});
            if (valid == 1) piece(TkInt<0>{}, TkInt<1>{});
        }
    }
}
// f(activation) with the call's activation: one branch for all that f does.
template <class F>
__device__ __forceinline__ void norm_with(int act, F f) {
    switch (act) {
        case HB_ACT_RELU: return f([](float v) HB_INLINE { return linear_act(v, HB_ACT_RELU); });
        case HB_ACT_GELU: return f([](float v) HB_INLINE { return linear_act(v, HB_ACT_GELU); });
        case HB_ACT_GELU_TANH: return f([](float v) HB_INLINE { return linear_act(v, HB_ACT_GELU_TANH); });
        case HB_ACT_SILU: return f([](float v) HB_INLINE { return linear_act(v, HB_ACT_SILU); });
        default: return f([](float v) HB_INLINE { return v; });
    }
}

// ---------------------------------------------------------------------------
// Groups whose pixels fit the registers of a workgroup: x is read once, the mean and then the squares of the differences from it are added up in registers, over
// the lanes through LDS, and the results leave.
// 8 x 4096 x 1024 in 32 groups, 256 slabs of 256 KB, one to a compute unit: 32.8 us, 4.1 TB/s (fp32 results 54 us, 3.7); all of them read (13 us), then all write (11).  Slabs that share a compute unit
// overlap the two, but a group is not divided: what is joined over workgroups is read twice.  1 x 64 x 512, silu: 4.4 us, the launch and a chain of latencies.
template <class X, class O, int SLOTS, bool FULL, NormKind KIND>
__global__ void __launch_bounds__(kNormThreads) norm_slab_kernel(NormArgs p) {
    using vec = typename NormVec<X>::type;
    constexpr int V = NormVec<X>::V, E = kNormEntries<KIND, V>;
    constexpr bool ONE = KIND == kNormOne;
    constexpr int S = ONE ? 1 : V;                        // sums of a lane
    extern __shared__ float s_norm[];
    const int nT = blockDim.x, nG = p.images * p.groups;
    float *const s_a = s_norm, *const s_b = s_a + nT * E, *const s_mean = s_b + nT * E, *const s_rstd = s_mean + nG;
    uint32_t block_;
    const int first_image = (int)p.by_blocks.by(xcd_blocked(blockIdx.x, gridDim.x, 8), block_) * p.images, block = block_;
    const NormLane l = norm_lane<V>(p, first_image, block);
    const int n = min(first_image + l.image, p.N - 1);
    const int offset = block * p.groups * p.D + (l.there ? l.at : 0);
    const X* const x = static_cast<const X*>(p.x) + n * p.x_image + offset;

    // Slot i of a lane is its row l.row + i * lanes_row: all there but for the last slot, and the image's last row is in that.
    const int last_row = l.row + (p.passes - 1) * p.lanes_row;
    const int valid = l.there ? l.valid : 0, last = !l.there || last_row >= p.rows ? 0 : last_row == p.rows - 1 ? l.valid_last : l.valid;
    vec held[SLOTS];
    {
        const X* from = x + (int64_t)min(l.row, p.rows - 1) * p.x_row;
        const int64_t step = (int64_t)p.lanes_row * p.x_row;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
            if (i < p.passes) {
                if (i > 0) from = i == p.passes - 1 ? x + (int64_t)min(last_row, p.rows - 1) * p.x_row : from + step;
                held[i] = norm_load<X, FULL>(from, i == p.passes - 1 ? last : valid);
            }
    }
    int group[S];
    uint32_t channel[V];
    const int cut = norm_channels<V, ONE>(p, l, block, group, channel);
    const auto weight = norm_per_channel<V>(p.weight, 1.f, channel, p.pixels == 1 && l.valid == V), bias = norm_per_channel<V>(p.bias, 0.f, channel, p.pixels == 1 && l.valid == V);
    // f(vector, its slot, what of it counts) for each of them
    auto rows = [&](auto f) HB_INLINE {
        int some = valid, end = last, passes = p.passes;
        asm volatile("" : "+v"(some), "+v"(end), "+s"(passes));              // or what each slot compares would be kept from one use to the next, in registers that there are not
        tk_for<SLOTS>([&](auto index) HB_INLINE {
            constexpr int i = decltype(index)::value;
            if (i < passes) {
                const int counts = i == passes - 1 ? end : some;
                if (counts > 0) f(held[i], i, FULL ? V : counts);
                __builtin_amdgcn_sched_barrier(0);        // one vector's values at a time: several would not fit the registers
            }
        });
    };
    const float count = (float)p.P * (float)p.D;
    const int lane = threadIdx.x & ((1 << p.log_lanes) - 1);

    // About the mean of the first vectors, while the others are on their way.
    float a[S] = {}, b[S] = {};
    if ((p.passes == 1 ? last : valid) > 0) {             // what is not valid is zero
#pragma unroll
        for (int i = 0; i < V; ++i) a[ONE ? 0 : i] += (float)held[0][i];
    }
    norm_fold<V, KIND>(a, cut, s_a + threadIdx.x * E);
    lds_barrier();
    const float first = p.passes == 1 ? count : (float)p.lanes_row * (float)p.pixels * (float)p.D;
    for (int q = threadIdx.x >> p.log_lanes; q < nG; q += nT >> p.log_lanes) {
        float sum = 0.f;
        norm_entries<V, KIND>(p, q, lane, [&](int e, bool there) HB_INLINE { sum += there ? s_a[e] : 0.f; });
        sum = norm_lanes_sum(sum, p.log_lanes);
        if (lane == 0) s_mean[q] = sum / first;
    }
    lds_barrier();
    // The first vectors are at least a 16th of all: where their mean is off by e, that is a difference between them and the others that is in the variance too, 15 var >= e^2, and
    // the squares about it are at most 16 times those about the mean.
    float mean[S];
#pragma unroll
    for (int i = 0; i < S; ++i) mean[i] = s_mean[group[i]], a[i] = 0.f;
    rows([&](const vec& v, int, int valid) HB_INLINE {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = FULL || i < valid ? (float)v[i] - mean[ONE ? 0 : i] : 0.f;
            a[ONE ? 0 : i] += d;
            b[ONE ? 0 : i] = fmaf(d, d, b[ONE ? 0 : i]);
        }
    });
    norm_fold<V, KIND>(a, cut, s_a + threadIdx.x * E);
    norm_fold<V, KIND>(b, cut, s_b + threadIdx.x * E);
    __syncthreads();
    for (int q = threadIdx.x >> p.log_lanes; q < nG; q += nT >> p.log_lanes) {
        float left = 0.f, squares = 0.f;
        norm_entries<V, KIND>(p, q, lane, [&](int e, bool there) HB_INLINE {
            left += there ? s_a[e] : 0.f;
            squares += there ? s_b[e] : 0.f;
        });
        left = norm_lanes_sum(left, p.log_lanes) / count;
        squares = norm_lanes_sum(squares, p.log_lanes) / count;
        if (lane == 0) {
            s_mean[q] += left;
            const float var = squares - left * left;      // a NaN, as an infinity makes of it, stays one
            s_rstd[q] = 1.f / sqrtf((var < 0.f ? 0.f : var) + p.eps);
        }
    }
    __syncthreads();
    float scale[V];
#pragma unroll
    for (int i = 0; i < S; ++i) mean[i] = s_mean[group[i]];
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] = s_rstd[group[ONE ? 0 : i]] * (float)weight[i];
    O* out = static_cast<O*>(p.out) + n * p.out_image + offset + l.row * p.out_row;
    const int64_t step = (int64_t)p.lanes_row * p.out_row;
    norm_with(p.act, [&](auto act) HB_INLINE {
        rows([&](const vec& v, int slot, int valid) HB_INLINE {
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = act(fmaf((float)v[i] - mean[ONE ? 0 : i], scale[i], (float)bias[i]));
            norm_store<O, V>(out + slot * step, y, FULL ? V : valid, p.stream);
        });
    });
}

// ---------------------------------------------------------------------------
// Larger groups.  A workgroup reads a chunk of rows and leaves mean and sum of squared differences of each of its groups; the chunks of a group are joined, by a wave of a launch
// of its own or, where they are few, by every workgroup of the next; and the rows are read once more.  Every joining takes the means first and the squares about the joint
// mean, so that no digits are lost where a mean is far from zero.
// Bound by memory: 1 x 2^20 x 64 in 32 groups, silu, 84.3 us: 40 for the first reading (29 where no results of a call before it are still on their way to memory), 5 for the joining, 41 for
// the second reading and the results, 6.2 TB/s.  fp32 to fp32 163 us; 8 x 4096 x 1024, of which no group fits in fp32, 80 us.  Small maps by the latencies of two launches: 3 x 1079 x 180 fp32, 12 groups, 10.1 us.

// U rows of a lane from `row` on, as many as there are before `end`: their vectors, and how many.
template <class X, bool FULL, int U>
__device__ __forceinline__ int norm_batch(const NormArgs& p, const X* x, int row, int end, const NormLane& l, typename NormVec<X>::type (&v)[U]) {
    int have = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int at = row + u * p.lanes_row;
        have += at < end;
        const int from = min(at, end - 1);                // what is not there is loaded from what is
        v[u] = norm_load<X, FULL>(x + (int64_t)from * p.x_row, from == p.rows - 1 ? l.valid_last : l.valid);
    }
    return have;
}

template <class X, bool FULL, NormKind KIND, int MOST>
__global__ void __launch_bounds__(MOST) norm_stats_kernel(NormArgs p) {
    using vec = typename NormVec<X>::type;
    constexpr int V = NormVec<X>::V, E = kNormEntries<KIND, V>, U = FULL && MOST < kNormThreads ? kNormBatch : kNormBatch / 2;
    constexpr bool ONE = KIND == kNormOne;
    extern __shared__ float s_norm[];
    const int nT = blockDim.x;
    float *const s_count = s_norm, *const s_mean = s_count + nT * E, *const s_squares = s_mean + nT * E;
    uint32_t chunk_, block_;
    const int n = p.by_blocks.by(p.by_chunks.by(blockIdx.x, chunk_), block_), block = block_, chunk = chunk_;
    const NormLane l = norm_lane<V>(p, n, block);
    const X* const x = static_cast<const X*>(p.x) + n * p.x_image + block * p.groups * p.D + (l.there ? l.at : 0);
    // a last row that is shorter than the others comes by itself
    const bool ragged = !FULL && ((int64_t)p.rows << p.log_pixels) > p.P;
    const int begin = chunk * p.chunk, end = min(begin + p.chunk, p.rows - ragged);
    float count = 0.f, mean[V] = {}, squares[V] = {};
    float extra[V] = {};       // elements of the short row
    if (l.there) {
        int row = begin + l.row;
        if (row < end) {
            vec v[U];
            int have = norm_batch<X, FULL, U>(p, x, row, end, l, v);
            for (;;) {
                vec next[U];
                int have_next = 0;
                row += U * p.lanes_row;
                if (row < end) have_next = norm_batch<X, FULL, U>(p, x, row, end, l, next);
                const float more = (float)have, inverse = 1.f / more, f = more / (count + more), g = count * f;
                auto join = [&](auto whole) HB_INLINE {
                    constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float m = 0.f, s = 0.f;
#pragma unroll
                        for (int u = 0; u < U; ++u) m += WHOLE || u < have ? (float)v[u][i] : 0.f;
                        m *= inverse;
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const float d = WHOLE || u < have ? (float)v[u][i] - m : 0.f;
                            s = fmaf(d, d, s);
                        }
                        const float d = m - mean[i];
                        mean[i] = fmaf(d, f, mean[i]);
                        squares[i] += fmaf(d * g, d, s);                     // g is 0 ahead of a lane's first batch, and d the whole mean: its square may pass fp32
                    }
                };
                if (have == U) join(TkInt<1>{});
                else join(TkInt<0>{});
                count += more;
                if (have_next == 0) break;
                have = have_next;
                tk_for<U>([&](auto u) HB_INLINE { v[decltype(u)::value] = next[decltype(u)::value]; });
            }
        }
        if (!FULL && ragged && chunk == p.chunks - 1 && (p.rows - 1 - begin) % p.lanes_row == l.row) {
            const vec v = norm_load<X, FULL>(x + (int64_t)(p.rows - 1) * p.x_row, l.valid_last);
            const float f = 1.f / (count + 1.f);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < l.valid_last) {
                    const float d = (float)v[i] - mean[i];
                    mean[i] = fmaf(d, f, mean[i]);
                    squares[i] = fmaf(d * (count * f), d, squares[i]);       // as above
                    extra[i] = 1.f;
                }
        }
    }
    // elements from `from` on, `n` of them, as one entry
    int group[ONE ? 1 : V];
    uint32_t channel[V];
    const int cut = norm_channels<V, ONE>(p, l, block, group, channel);
    auto entry = [&](int e, auto in) HB_INLINE {
        float c = 0.f, m = 0.f, left = 0.f, s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            c += in(i) ? count + extra[i] : 0.f;
            m += in(i) ? (count + extra[i]) * mean[i] : 0.f;                 // what is behind the row may be anything
        }
        const float inverse = c > 0.f ? 1.f / c : 0.f;
        m *= inverse;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float k = count + extra[i], d = mean[i] - m;
            left += in(i) ? k * d : 0.f;
            s += in(i) ? fmaf(k * d, d, squares[i]) : 0.f;
        }
        left *= inverse;
        s_count[threadIdx.x * E + e] = c;
        s_mean[threadIdx.x * E + e] = m + left;
        s_squares[threadIdx.x * E + e] = fmaf(-c * left, left, s);
    };
    if (KIND == kNormOne) {
        entry(0, [](int) HB_INLINE { return true; });
    } else if (KIND == kNormTwo) {
        entry(0, [&](int i) HB_INLINE { return i < cut; });
        entry(1, [&](int i) HB_INLINE { return i >= cut; });
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s_count[threadIdx.x * E + i] = count + extra[i];
            s_mean[threadIdx.x * E + i] = mean[i];
            s_squares[threadIdx.x * E + i] = squares[i];
        }
    }
    __syncthreads();
    const int lane = threadIdx.x & ((1 << p.log_lanes) - 1);
    const float c = (float)(min((begin + p.chunk) << p.log_pixels, p.P) - (begin << p.log_pixels)) * (float)p.D, inverse_c = 1.f / c;     // elements of a group in the chunk
    for (int q = threadIdx.x >> p.log_lanes; q < p.groups; q += nT >> p.log_lanes) {
        float m = 0.f;
        norm_entries<V, KIND>(p, q, lane, [&](int e, bool there) HB_INLINE { m += there ? s_count[e] * s_mean[e] : 0.f; });
        m = norm_lanes_sum(m, p.log_lanes) * inverse_c;
        float left = 0.f, s = 0.f;
        norm_entries<V, KIND>(p, q, lane, [&](int e, bool there) HB_INLINE {
            const float d = s_mean[e] - m, cd = s_count[e] * d;
            left += there ? cd : 0.f;
            s += there ? fmaf(cd, d, s_squares[e]) : 0.f;
        });
        left = norm_lanes_sum(left, p.log_lanes) * inverse_c;
        s = norm_lanes_sum(s, p.log_lanes);
        const int g = block * p.groups + q;
        if (lane == 0 && g < p.G) p.parts[((int64_t)n * p.G + g) * p.chunks + chunk] = float2{m + left, fmaf(-c * left, left, s)};
    }
}

// Mean and 1 / sqrt(var + eps) of a group from its chunks, at most kNormJoin of a lane's, by 2^log_lanes lanes; the same in all of them.  In 64 bits: nothing here is on
// the path of an element.
__device__ __forceinline__ float2 norm_join(const NormArgs& p, const float2* parts, int lane, int log_lanes) {
    float2 part[kNormJoin];
    int at[kNormJoin];
#pragma unroll
    for (int i = 0; i < kNormJoin; ++i) {
        at[i] = lane + (i << log_lanes);
        part[i] = parts[min(at[i], p.chunks - 1)];
    }
    const int span = p.chunk << p.log_pixels;
    const double most = (double)span, least = (double)(p.P - (int64_t)(p.chunks - 1) * span);      // pixels of a chunk, and of the last
    auto pixels = [&](int i) HB_INLINE { return at[i] < p.chunks - 1 ? most : at[i] == p.chunks - 1 ? least : 0.0; };
    auto all = [&](double v) HB_INLINE {
        for (int m = 1 << log_lanes >> 1; m > 0; m >>= 1) v += __shfl_xor(v, m);
        return v;
    };
    double mean = 0.0, squares = 0.0;
#pragma unroll
    for (int i = 0; i < kNormJoin; ++i) mean += pixels(i) * (double)part[i].x;
    mean = all(mean) * p.inverse_P;
#pragma unroll
    for (int i = 0; i < kNormJoin; ++i) {
        const double d = (double)part[i].x - mean;
        squares += (at[i] < p.chunks ? (double)part[i].y : 0.0) + pixels(i) * p.D * d * d;
    }
    squares = all(squares) * p.inverse_P / (float)p.D;
    return float2{(float)mean, 1.f / sqrtf((squares < 0.0 ? 0.f : (float)squares) + p.eps)};
}
__global__ void __launch_bounds__(64) norm_join_kernel(NormArgs p) {
    const int64_t q = blockIdx.x;
    const float2 r = norm_join(p, p.parts + q * p.chunks, threadIdx.x, 6);
    if (threadIdx.x == 0) p.stats[q] = r;
}

template <class X, class O, bool FULL, bool ONE, bool JOINED>
__global__ void __launch_bounds__(kNormThreads) norm_apply_kernel(NormArgs p) {
    using vec = typename NormVec<X>::type;
    constexpr int V = NormVec<X>::V, S = ONE ? 1 : V, U = kNormBatch / 2;
    extern __shared__ float s_norm[];
    uint32_t chunk_, block_;
    const int n = p.by_blocks.by(p.by_apply_chunks.by(blockIdx.x, chunk_), block_), block = block_, chunk = chunk_;
    const NormLane l = norm_lane<V>(p, n, block);
    const int offset = block * p.groups * p.D + (l.there ? l.at : 0);
    const X* const x = static_cast<const X*>(p.x) + n * p.x_image + offset;
    O* const out = static_cast<O*>(p.out) + n * p.out_image + offset;
    const int begin = chunk * p.apply_chunk, end = min(begin + p.apply_chunk, p.rows);
    int row = begin + l.row, have = 0;
    vec v[U];
    if (l.there && row < end) have = norm_batch<X, FULL, U>(p, x, row, end, l, v);
    int group[S];
    uint32_t channel[V];
    norm_channels<V, ONE>(p, l, block, group, channel);
    const auto weight = norm_per_channel<V>(p.weight, 1.f, channel, p.pixels == 1 && l.valid == V), bias = norm_per_channel<V>(p.bias, 0.f, channel, p.pixels == 1 && l.valid == V);
    float mean[S], scale[V];
    if (JOINED) {
        const float2* stats = p.stats + (int64_t)n * p.G + block * p.groups;
#pragma unroll
        for (int i = 0; i < S; ++i) mean[i] = stats[group[i]].x;
#pragma unroll
        for (int i = 0; i < V; ++i) scale[i] = stats[group[ONE ? 0 : i]].y * (float)weight[i];
    } else {
        float2* const s_stats = reinterpret_cast<float2*>(s_norm);
        const int lane = threadIdx.x & ((1 << p.log_lanes) - 1), own = min(p.groups, p.G - block * p.groups);
        for (int q = threadIdx.x >> p.log_lanes; q < own; q += blockDim.x >> p.log_lanes) {
            const float2 r = norm_join(p, p.parts + ((int64_t)n * p.G + block * p.groups + q) * p.chunks, lane, p.log_lanes);
            if (lane == 0) s_stats[q] = r;
        }
        lds_barrier();
#pragma unroll
        for (int i = 0; i < S; ++i) mean[i] = s_stats[group[i]].x;
#pragma unroll
        for (int i = 0; i < V; ++i) scale[i] = s_stats[group[ONE ? 0 : i]].y * (float)weight[i];
    }
    if (have == 0) return;
    norm_with(p.act, [&](auto act) HB_INLINE {
        for (;;) {
            vec next[U];
            int have_next = 0;
            const int here = row;
            row += U * p.lanes_row;
            if (row < end) have_next = norm_batch<X, FULL, U>(p, x, row, end, l, next);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < have) {
                    const int at = here + u * p.lanes_row;
                    float y[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) y[i] = act(fmaf((float)v[u][i] - mean[ONE ? 0 : i], scale[i], (float)bias[i]));
                    norm_store<O, V>(out + (int64_t)at * p.out_row, y, FULL ? V : at == p.rows - 1 ? l.valid_last : l.valid, p.stream);
                    __builtin_amdgcn_sched_barrier(0);
                }
            if (have_next == 0) break;
            have = have_next;
            tk_for<U>([&](auto u) HB_INLINE { v[decltype(u)::value] = next[decltype(u)::value]; });
        }
    });
}

// ---------------------------------------------------------------------------
template <class X, class O, bool FULL, NormKind KIND>
static hb_status norm_launch(const NormArgs& a, const NormPlan& plan, hipStream_t st) {
    constexpr int E = kNormEntries<KIND, NormVec<X>::V>;
    constexpr bool ONE = KIND == kNormOne;
    if (plan.slab) {
        const int lds = (2 * plan.threads * E + 2 * plan.images * plan.groups) * 4;
        auto kernel = plan.passes <= 1 ? norm_slab_kernel<X, O, 1, FULL, KIND> : plan.passes <= 4 ? norm_slab_kernel<X, O, 4, FULL, KIND> : norm_slab_kernel<X, O, norm_slots(NormVec<X>::V, ONE), FULL, KIND>;
        if (lds > 65536)
            if (hb_status s = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds)) return s;
        // a launch has fewer than 2^32 lanes: so many images
        const int64_t most = 0xffffffffll / plan.threads / plan.blocks * plan.images;
        if (most < 1) return HB_ERR_UNSUPPORTED;
        for (int64_t n = 0; n < a.N; n += most) {
            NormArgs part = a;
            part.x = static_cast<const X*>(a.x) + n * a.x_image;
            part.out = static_cast<O*>(a.out) + n * a.out_image;
            part.N = (int)(a.N - n < most ? a.N - n : most);
            hipLaunchKernelGGL(kernel, dim3((unsigned)(((part.N - 1) / plan.images + 1) * plan.blocks)), dim3(plan.threads), lds, st, part);
            if (hb_status s = launch_status()) return s;
        }
        return HB_OK;
    }
    const int64_t wgs = (int64_t)a.N * plan.blocks * plan.chunks, apply_wgs = (int64_t)a.N * plan.blocks * plan.apply_chunks;
    if (!launch_holds((double)wgs, plan.threads) || !launch_holds((double)apply_wgs, plan.threads) || (plan.join && !launch_holds((double)a.N * a.G, 64))) return HB_ERR_UNSUPPORTED;
    const int lds = 3 * plan.threads * E * 4;
    auto stats = plan.threads <= 256 ? norm_stats_kernel<X, FULL, KIND, 256> : norm_stats_kernel<X, FULL, KIND, kNormThreads>;
    if (lds > 65536)
        if (hb_status s = allow_dynamic_lds(reinterpret_cast<const void*>(stats), lds)) return s;
    hipLaunchKernelGGL(stats, dim3((unsigned)wgs), dim3(plan.threads), lds, st, a);
    if (plan.join) {
        hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(a.N * a.G)), dim3(64), 0, st, a);
        hipLaunchKernelGGL((norm_apply_kernel<X, O, FULL, ONE, true>), dim3((unsigned)apply_wgs), dim3(plan.threads), 0, st, a);
    } else {
        hipLaunchKernelGGL((norm_apply_kernel<X, O, FULL, ONE, false>), dim3((unsigned)apply_wgs), dim3(plan.threads), 8 * plan.groups, st, a);
    }
    return launch_status();
}

template <class X, class O>
static hb_status norm_call(NormArgs a, int64_t x_pixel, int64_t out_pixel, void* workspace, size_t workspace_bytes, hipStream_t st) {
    constexpr int V = NormVec<X>::V;
    const NormPlan plan = norm_plan(a.N, a.P, a.C, a.G, V, x_pixel == a.C && out_pixel == a.C);
    if (const size_t need = norm_workspace(a.N, a.P, a.C, a.G)) {
        if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < need) return HB_ERR_WORKSPACE;
        a.parts = static_cast<float2*>(workspace);
        a.stats = a.parts + (int64_t)a.N * a.G * plan.chunks;
    }
    a.pixels = plan.pixels;
    a.groups = plan.groups;
    a.images = plan.images;
    a.width = plan.width;
    a.rows = plan.rows;
    a.blocks = plan.blocks;
    a.passes = plan.passes;
    a.chunk = plan.chunk;
    a.chunks = plan.chunks;
    a.apply_chunk = plan.apply_chunk;
    a.apply_chunks = plan.apply_chunks;
    while (1 << a.log_pixels < plan.pixels) ++a.log_pixels;                 // 1, 2, 4 or 8
    a.x_row = plan.pixels * x_pixel;
    a.out_row = plan.pixels * out_pixel;
    a.lanes_row = plan.threads / (plan.images * plan.width);
    const bool one = a.D % V == 0, full = plan.pixels * (int64_t)a.groups * a.D % V == 0 && (int64_t)a.G * a.D * plan.pixels % V == 0 && a.P % plan.pixels == 0;
    a.log_lanes = plan.log_lanes;
    a.size = one ? a.D / V : a.D >= V ? (a.D - 2) / V + 2 : a.D;
    a.step_d = (1 << a.log_lanes) % a.size;
    a.step_r = (1 << a.log_lanes) / a.size;
    a.by_all = norm_div(plan.images * plan.width);
    a.by_width = norm_div(plan.width);
    a.by_size = norm_div(a.size);
    a.by_D = norm_div(a.D);
    a.by_blocks = norm_div(plan.blocks);
    if (!plan.slab) {
        a.by_chunks = norm_div(plan.chunks);
        a.by_apply_chunks = norm_div(plan.apply_chunks);
        a.inverse_P = 1.0 / a.P;
    }
    a.stream = sizeof(O) <= sizeof(X) && (int64_t)a.groups * a.D * sizeof(O) % 128 == 0 && a.out_row * sizeof(O) % 128 == 0 && a.out_image * sizeof(O) % 128 == 0 && aligned_to(a.out, 128);
    if (one) return norm_launch<X, O, true, kNormOne>(a, plan, st);
    if (a.D >= V) return full ? norm_launch<X, O, true, kNormTwo>(a, plan, st) : norm_launch<X, O, false, kNormTwo>(a, plan, st);
    return full ? norm_launch<X, O, true, kNormEach>(a, plan, st) : norm_launch<X, O, false, kNormEach>(a, plan, st);
}

}  // namespace hb

extern "C" size_t hb_group_norm_workspace_size(int N, int P, int C, int groups) {
    if (N < 1 || P < 1 || C < 1 || groups < 1 || C % groups || C / groups > HB_GROUP_NORM_MAX_CHANNELS) return 0;
    return hb::norm_workspace(N, P, C, groups);
}

extern "C" hb_status hb_group_norm(const void* x, hb_type x_type, const hb_half* weight, const hb_half* bias, void* out, hb_type out_type,
                                   hb_act act, float eps, int N, int P, int C, int groups, int64_t x_image, int64_t x_pixel,
                                   int64_t out_image, int64_t out_pixel, void* workspace, size_t workspace_bytes, hb_stream stream) {
    using namespace hb;
    if (!x || !out || N < 1 || P < 1 || C < 1 || groups < 1 || C % groups) return HB_ERR_INVALID_ARG;
    if ((x_type != HB_F16 && x_type != HB_F32) || (out_type != HB_F16 && out_type != HB_F32) || act < HB_ACT_NONE || act > HB_ACT_SILU) return HB_ERR_INVALID_ARG;
    if (!(eps > 0.f) || isinf(eps)) return HB_ERR_INVALID_ARG;
    if (!aligned_to(x, x_type == HB_F32 ? 4 : 2) || !aligned_to(out, out_type == HB_F32 ? 4 : 2) || !aligned_to(weight, 2) || !aligned_to(bias, 2)) return HB_ERR_INVALID_ARG;
    // the stride of a single image or pixel has no meaning
    if (P == 1) x_pixel = out_pixel = C;
    if (N == 1) x_image = out_image = C;
    if (x_pixel < C || out_pixel < C || x_image < C || out_image < C) return HB_ERR_INVALID_ARG;
    if (C / groups > HB_GROUP_NORM_MAX_CHANNELS || P >= 1 << 30 || (int64_t)N * groups >= 1 << 30) return HB_ERR_UNSUPPORTED;
    NormArgs a = {};
    a.x = x;
    a.out = out;
    a.weight = reinterpret_cast<const half_t*>(weight);
    a.bias = reinterpret_cast<const half_t*>(bias);
    a.eps = eps;
    a.act = act;
    a.N = N;
    a.P = P;
    a.C = C;
    a.G = groups;
    a.D = C / groups;
    a.x_image = x_image;
    a.out_image = out_image;
    const auto st = reinterpret_cast<hipStream_t>(stream);
    if (x_type == HB_F32) {
        return out_type == HB_F32 ? norm_call<float, float>(a, x_pixel, out_pixel, workspace, workspace_bytes, st) : norm_call<float, half_t>(a, x_pixel, out_pixel, workspace, workspace_bytes, st);
    }
    return out_type == HB_F32 ? norm_call<half_t, float>(a, x_pixel, out_pixel, workspace, workspace_bytes, st) : norm_call<half_t, half_t>(a, x_pixel, out_pixel, workspace, workspace_bytes, st);
}
