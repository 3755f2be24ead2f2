// hb_group_norm: group norm with an activation, channels last.
#include <math.h>

#include "group_norm_plan.hpp"
#include "hb_device.hpp"
#include "hb_host.hpp"
#include "token_epilogue.hpp"

namespace hb {

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
    int lanes_row;             // rows side by side in a workgroup
    int log_lanes;             // lanes that add up a group: 2^this
    int step_d, step_r;        // these lanes in entries of a group's row, and in rows
    int stream;                // results past the caches
};

template <class X>
struct NormVec {
    static constexpr int V = 16 / sizeof(X);
    typedef X type __attribute__((ext_vector_type(V), aligned(sizeof(X))));
};

// Where a lane stands.
struct NormLane {
    int row, column;           // of the workgroup; columns are vectors
    int image, at;             // image of the workgroup, first channel in the row of its block
    bool there;
    int valid, valid_last;     // elements of its vector in a row, and in the image's last row
};
template <int V>
__device__ __forceinline__ NormLane norm_lane(const NormArgs& p, int first_image, int block) {
    NormLane l;
    const int all = p.images * p.width;
    l.row = threadIdx.x / (unsigned)all;
    l.column = threadIdx.x - l.row * all;
    l.image = l.column / (unsigned)p.width;
    l.at = (l.column - l.image * p.width) * V;
    const int channels = min(p.groups, p.G - block * p.groups) * p.D, length = p.pixels * channels;
    l.there = l.row < p.lanes_row && first_image + l.image < p.N && l.at < length;
    l.valid = max(0, min(V, length - l.at));
    l.valid_last = max(0, min(V, (p.P - (p.rows - 1) * p.pixels) * channels - l.at));
    return l;
}

// V adjacent elements, zeros from `valid` on; `from` is not read where that is 0.
template <class X, bool FULL>
__device__ __forceinline__ typename NormVec<X>::type norm_load(const X* from, int valid) {
    using vec = typename NormVec<X>::type;
    if (FULL || valid == NormVec<X>::V) return *reinterpret_cast<const vec*>(from);
    vec r = {};
#pragma unroll
    for (int i = 0; i < NormVec<X>::V; ++i)
        if (i < valid) r[i] = from[i];
    return r;
}

// The entries of group q of the workgroup that belong to one of the lanes that add it up: f(index).  An entry is an element of a lane, or, where a vector
// is of one group (ONE), a lane; entries of a row are adjacent, a group's are D (or D / V) of them, once for each pixel of a row.
template <int V, bool ONE, class F>
__device__ __forceinline__ void norm_entries(const NormArgs& p, int q, int lane, F f) {
    const int per = ONE ? 1 : V, size = ONE ? p.D / V : p.D, length = p.images * p.width * per;
    const int image = q / (unsigned)p.groups, first = image * p.width * per + (q - image * p.groups) * size;
    int r = lane / (unsigned)size, d = lane - r * size;
    if (p.pixels == 1) {
        for (; r < p.lanes_row;) {
            f(r * length + first + d);
            d += p.step_d;
            r += p.step_r + (d >= size);
            d -= d >= size ? size : 0;
        }
    } else {
        for (; r < p.lanes_row * p.pixels;) {
            const int row = r / (unsigned)p.pixels;
            f(row * length + (r - row * p.pixels) * p.C + first + d);
            d += p.step_d;
            r += p.step_r + (d >= size);
            d -= d >= size ? size : 0;
        }
    }
}
// Sum over the lanes that share a group, the same in all of them.
__device__ __forceinline__ float norm_lanes_sum(float v, int log_lanes) {
    for (int m = 1 << log_lanes >> 1; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// The groups of a lane's elements in the workgroup, and their channels in the image.
template <int V, bool ONE>
__device__ __forceinline__ void norm_channels(const NormArgs& p, const NormLane& l, int block, int (&group)[ONE ? 1 : V], uint32_t (&channel)[V]) {
    int c = p.pixels > 1 ? l.at % (unsigned)p.C : l.at, g = c / (unsigned)p.D, d = c - g * p.D;
    const int own = min(p.groups, p.G - block * p.groups), first = block * p.groups * p.D;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        channel[i] = first + min(c, own * p.D - 1);
        if (!ONE || i == 0) group[ONE ? 0 : i] = l.image * p.groups + min(g, own - 1);
        ++c;
        if (++d == p.D) d = 0, ++g;
        if (p.pixels > 1 && c == p.C) c = 0, g = 0, d = 0;
    }
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
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < valid) to[i] = (O)v[i];
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
template <class X, class O, int SLOTS, bool FULL, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_slab_kernel(NormArgs p) {
    using vec = typename NormVec<X>::type;
    constexpr int V = NormVec<X>::V, E = ONE ? 1 : V;
    extern __shared__ float s_norm[];
    const int nT = blockDim.x, nG = p.images * p.groups;
    float *const s_a = s_norm, *const s_b = s_a + nT * E, *const s_mean = s_b + nT * E, *const s_rstd = s_mean + nG;
    const int id = xcd_blocked(blockIdx.x, gridDim.x, 8), block = id % p.blocks, first_image = id / p.blocks * p.images;
    const NormLane l = norm_lane<V>(p, first_image, block);
    const int n = min(first_image + l.image, p.N - 1);
    const int offset = block * p.groups * p.D + (l.there ? l.at : 0);
    const X* const x = static_cast<const X*>(p.x) + n * p.x_image + offset;

    vec held[SLOTS];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i)
        if (i < p.passes) {
            const int row = min(l.row + i * p.lanes_row, p.rows - 1);
            held[i] = norm_load<X, FULL>(x + row * p.x_row, !l.there ? 0 : row == p.rows - 1 ? l.valid_last : l.valid);
        }
    int group[E];
    uint32_t channel[V];
    norm_channels<V, ONE>(p, l, block, group, channel);
    const auto weight = norm_per_channel<V>(p.weight, 1.f, channel, p.pixels == 1 && l.valid == V), bias = norm_per_channel<V>(p.bias, 0.f, channel, p.pixels == 1 && l.valid == V);
    // rows of this lane, and what of its vector counts in each
    auto rows = [&](auto f) HB_INLINE {
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
            if (i < p.passes) {
                const int row = l.row + i * p.lanes_row;
                if (l.there && row < p.rows) f(held[i], row, FULL ? V : row == p.rows - 1 ? l.valid_last : l.valid);
                __builtin_amdgcn_sched_barrier(0);        // one vector's values at a time: several would not fit the registers
            }
    };
    const float count = (float)p.P * (float)p.D;
    const int lane = threadIdx.x & ((1 << p.log_lanes) - 1);

    float a[E] = {}, b[E] = {};
    rows([&](const vec& v, int, int) HB_INLINE {          // what is not valid is zero
#pragma unroll
        for (int i = 0; i < V; ++i) a[ONE ? 0 : i] += (float)v[i];
    });
#pragma unroll
    for (int i = 0; i < E; ++i) s_a[threadIdx.x * E + i] = a[i];
    __syncthreads();
    for (int q = threadIdx.x >> p.log_lanes; q < nG; q += nT >> p.log_lanes) {
        float sum = 0.f;
        norm_entries<V, ONE>(p, q, lane, [&](int e) HB_INLINE { sum += s_a[e]; });
        sum = norm_lanes_sum(sum, p.log_lanes);
        if (lane == 0) s_mean[q] = sum / count;
    }
    __syncthreads();
    float mean[E];
#pragma unroll
    for (int i = 0; i < E; ++i) mean[i] = s_mean[group[i]], a[i] = 0.f;
    rows([&](const vec& v, int, int valid) HB_INLINE {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = i < valid ? (float)v[i] - mean[ONE ? 0 : i] : 0.f;
            a[ONE ? 0 : i] += d;
            b[ONE ? 0 : i] = fmaf(d, d, b[ONE ? 0 : i]);
        }
    });
#pragma unroll
    for (int i = 0; i < E; ++i) {
        s_a[threadIdx.x * E + i] = a[i];
        s_b[threadIdx.x * E + i] = b[i];
    }
    __syncthreads();
    for (int q = threadIdx.x >> p.log_lanes; q < nG; q += nT >> p.log_lanes) {
        float left = 0.f, squares = 0.f;
        norm_entries<V, ONE>(p, q, lane, [&](int e) HB_INLINE {
            left += s_a[e];
            squares += s_b[e];
        });
        left = norm_lanes_sum(left, p.log_lanes) / count;                    // what the rounded sum left of the mean
        squares = norm_lanes_sum(squares, p.log_lanes) / count;
        if (lane == 0) {
            s_mean[q] += left;
            s_rstd[q] = 1.f / sqrtf(fmaxf(squares - left * left, 0.f) + p.eps);
        }
    }
    __syncthreads();
    float scale[V];
#pragma unroll
    for (int i = 0; i < E; ++i) mean[i] = s_mean[group[i]];
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] = s_rstd[group[ONE ? 0 : i]] * (float)weight[i];
    O* const out = static_cast<O*>(p.out) + n * p.out_image + offset;
    norm_with(p.act, [&](auto act) HB_INLINE {
        rows([&](const vec& v, int row, int valid) HB_INLINE {
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = act(fmaf((float)v[i] - mean[ONE ? 0 : i], scale[i], (float)bias[i]));
            norm_store<O, V>(out + row * p.out_row, y, FULL ? V : valid, p.stream);
        });
    });
}

// ---------------------------------------------------------------------------
// Larger groups.  A workgroup reads a chunk of rows and leaves mean and sum of squared differences of each of its groups; a wave joins the chunks of a group; and
// the rows are read once more.  Every joining takes the means first and the squares about the joint mean, so that no digits are lost where a mean is far from zero.
template <class X, bool FULL, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_stats_kernel(NormArgs p) {
    using vec = typename NormVec<X>::type;
    constexpr int V = NormVec<X>::V, E = ONE ? 1 : V, U = kNormBatch;
    extern __shared__ float s_norm[];
    const int nT = blockDim.x;
    float *const s_count = s_norm, *const s_mean = s_count + nT * E, *const s_squares = s_mean + nT * E;
    const int chunk = blockIdx.x % (unsigned)p.chunks, rest = blockIdx.x / (unsigned)p.chunks, block = rest % p.blocks, n = rest / p.blocks;
    const NormLane l = norm_lane<V>(p, n, block);
    const X* const x = static_cast<const X*>(p.x) + n * p.x_image + block * p.groups * p.D + (l.there ? l.at : 0);
    // a last row that is shorter than the others comes by itself
    const bool ragged = !FULL && (int64_t)p.rows * p.pixels > p.P;
    const int begin = chunk * p.chunk, end = min(begin + p.chunk, p.rows - ragged);
    float count = 0.f, mean[V] = {}, squares[V] = {};
    auto join = [&](float more, const float (&m)[V], const float (&s)[V]) HB_INLINE {
        const float f = more / (count + more), g = count * f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = m[i] - mean[i];
            mean[i] = fmaf(d, f, mean[i]);
            squares[i] += fmaf(d * d, g, s[i]);
        }
        count += more;
    };
    float extra[V] = {};       // elements of the short row
    if (l.there) {
        int row = begin + l.row;
        const X* from = x + row * p.x_row;
        for (; row + (U - 1) * p.lanes_row < end; row += U * p.lanes_row) {
            vec v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = norm_load<X, FULL>(from + (int64_t)(u * p.lanes_row) * p.x_row, l.valid);
            from += (int64_t)(U * p.lanes_row) * p.x_row;
            float m[V], s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                m[i] = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u) m[i] += (float)v[u][i];
                m[i] *= 1.f / U;
                s[i] = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float d = (float)v[u][i] - m[i];
                    s[i] = fmaf(d, d, s[i]);
                }
            }
            join((float)U, m, s);
        }
        for (; row < end; row += p.lanes_row) {
            const vec v = norm_load<X, FULL>(x + row * p.x_row, l.valid);
            float m[V], s[V] = {};
#pragma unroll
            for (int i = 0; i < V; ++i) m[i] = (float)v[i];
            join(1.f, m, s);
        }
        if (!FULL && ragged && row == p.rows - 1 && row < begin + p.chunk) {
            const vec v = norm_load<X, FULL>(x + row * p.x_row, l.valid_last);
            const float f = 1.f / (count + 1.f);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < l.valid_last) {
                    const float d = (float)v[i] - mean[i];
                    mean[i] = fmaf(d, f, mean[i]);
                    squares[i] = fmaf(d * d, count * f, squares[i]);
                    extra[i] = 1.f;
                }
        }
    }
    if (ONE) {                                            // the lane's elements are of one group
        float m = 0.f, left = 0.f, s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) m += mean[i];
        m *= 1.f / V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = mean[i] - m;
            left += d;
            s += fmaf(d * d, count, squares[i]);
        }
        left *= 1.f / V;
        s_count[threadIdx.x] = V * count;
        s_mean[threadIdx.x] = m + left;
        s_squares[threadIdx.x] = fmaxf(fmaf(-V * count * left, left, s), 0.f);
        if (s != s) s_squares[threadIdx.x] = s;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s_count[threadIdx.x * V + i] = count + extra[i];
            s_mean[threadIdx.x * V + i] = mean[i];
            s_squares[threadIdx.x * V + i] = squares[i];
        }
    }
    __syncthreads();
    const int lane = threadIdx.x & ((1 << p.log_lanes) - 1);
    for (int q = threadIdx.x >> p.log_lanes; q < p.groups; q += nT >> p.log_lanes) {
        float c = 0.f, m = 0.f;
        norm_entries<V, ONE>(p, q, lane, [&](int e) HB_INLINE {
            c += s_count[e];
            m = fmaf(s_count[e], s_mean[e], m);
        });
        c = norm_lanes_sum(c, p.log_lanes);
        m = norm_lanes_sum(m, p.log_lanes) / c;
        float left = 0.f, s = 0.f;
        norm_entries<V, ONE>(p, q, lane, [&](int e) HB_INLINE {
            const float d = s_mean[e] - m, cd = s_count[e] * d;
            left += cd;
            s += fmaf(cd, d, s_squares[e]);
        });
        left = norm_lanes_sum(left, p.log_lanes) / c;
        s = norm_lanes_sum(s, p.log_lanes);
        const int g = block * p.groups + q;
        if (lane == 0 && g < p.G) p.parts[((int64_t)n * p.G + g) * p.chunks + chunk] = float2{m + left, fmaf(-c * left, left, s)};
    }
}

// A wave per group of an image.  In 64 bits: nothing here is on the path of an element.
__global__ void __launch_bounds__(64) norm_join_kernel(NormArgs p) {
    const int64_t q = blockIdx.x;
    const float2* parts = p.parts + q * p.chunks;
    auto pixels = [&](int chunk) HB_INLINE {
        const int64_t span = (int64_t)p.chunk * p.pixels, begin = chunk * span;
        return (double)(begin + span < p.P ? span : p.P - begin);
    };
    auto all = [&](double v) HB_INLINE {
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
        return v;
    };
    double mean = 0.0, squares = 0.0;
    for (int i = threadIdx.x; i < p.chunks; i += 64) mean += pixels(i) * (double)parts[i].x;
    mean = all(mean) / (double)p.P;
    for (int i = threadIdx.x; i < p.chunks; i += 64) {
        const double d = (double)parts[i].x - mean;
        squares += (double)parts[i].y + pixels(i) * p.D * d * d;
    }
    squares = all(squares) / ((double)p.P * p.D);
    if (threadIdx.x == 0) p.stats[q] = float2{(float)mean, 1.f / sqrtf((squares < 0.0 ? 0.f : (float)squares) + p.eps)};
}

template <class X, class O, bool FULL, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_apply_kernel(NormArgs p) {
    using vec = typename NormVec<X>::type;
    constexpr int V = NormVec<X>::V, E = ONE ? 1 : V, U = kNormBatch;
    const int chunk = blockIdx.x % (unsigned)p.chunks, rest = blockIdx.x / (unsigned)p.chunks, block = rest % p.blocks, n = rest / p.blocks;
    const NormLane l = norm_lane<V>(p, n, block);
    if (!l.there) return;
    const int offset = block * p.groups * p.D + l.at;
    const X* const x = static_cast<const X*>(p.x) + n * p.x_image + offset;
    O* const out = static_cast<O*>(p.out) + n * p.out_image + offset;
    int group[E];
    uint32_t channel[V];
    norm_channels<V, ONE>(p, l, block, group, channel);
    float mean[E], scale[V], shift[V];
    const float2* stats = p.stats + (int64_t)n * p.G + block * p.groups;
#pragma unroll
    for (int i = 0; i < E; ++i) mean[i] = stats[group[i]].x;
    const auto weight = norm_per_channel<V>(p.weight, 1.f, channel, p.pixels == 1 && l.valid == V), bias = norm_per_channel<V>(p.bias, 0.f, channel, p.pixels == 1 && l.valid == V);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        scale[i] = stats[group[ONE ? 0 : i]].y * (float)weight[i];
        shift[i] = (float)bias[i];
    }
    const int begin = chunk * p.chunk, end = min(begin + p.chunk, p.rows);
    norm_with(p.act, [&](auto act) HB_INLINE {
        auto store = [&](const vec& v, int row, int valid) HB_INLINE {
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = act(fmaf((float)v[i] - mean[ONE ? 0 : i], scale[i], shift[i]));
            norm_store<O, V>(out + row * p.out_row, y, valid, p.stream);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto valid = [&](int row) HB_INLINE { return FULL ? V : row == p.rows - 1 ? l.valid_last : l.valid; };
        int row = begin + l.row;
        for (; row + (U - 1) * p.lanes_row < end; row += U * p.lanes_row) {
            vec v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = norm_load<X, FULL>(x + (int64_t)(row + u * p.lanes_row) * p.x_row, valid(row + u * p.lanes_row));
#pragma unroll
            for (int u = 0; u < U; ++u) store(v[u], row + u * p.lanes_row, valid(row + u * p.lanes_row));
        }
        for (; row < end; row += p.lanes_row) store(norm_load<X, FULL>(x + (int64_t)row * p.x_row, valid(row)), row, valid(row));
    });
}

// ---------------------------------------------------------------------------
template <class X, class O, bool FULL, bool ONE>
static hb_status norm_launch(const NormArgs& a, const NormPlan& plan, hipStream_t st) {
    constexpr int E = ONE ? 1 : NormVec<X>::V;
    if (plan.slab) {
        const int64_t wgs = (int64_t)((a.N - 1) / plan.images + 1) * plan.blocks;
        if (!launch_holds((double)wgs, plan.threads)) return HB_ERR_UNSUPPORTED;
        const int lds = (2 * plan.threads * E + 2 * plan.images * plan.groups) * 4;
        auto kernel = plan.passes <= 1 ? norm_slab_kernel<X, O, 1, FULL, ONE> : plan.passes <= 4 ? norm_slab_kernel<X, O, 4, FULL, ONE> : norm_slab_kernel<X, O, kNormSlots, FULL, ONE>;
        if (lds > 65536)
            if (hb_status s = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds)) return s;
        hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(plan.threads), lds, st, a);
        return launch_status();
    }
    const int64_t wgs = (int64_t)a.N * plan.blocks * plan.chunks;
    if (!launch_holds((double)wgs, plan.threads) || !launch_holds((double)a.N * a.G, 64)) return HB_ERR_UNSUPPORTED;
    const int lds = 3 * plan.threads * E * 4;
    auto stats = norm_stats_kernel<X, FULL, ONE>;
    if (lds > 65536)
        if (hb_status s = allow_dynamic_lds(reinterpret_cast<const void*>(stats), lds)) return s;
    hipLaunchKernelGGL(stats, dim3((unsigned)wgs), dim3(plan.threads), lds, st, a);
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(a.N * a.G)), dim3(64), 0, st, a);
    hipLaunchKernelGGL((norm_apply_kernel<X, O, FULL, ONE>), dim3((unsigned)wgs), dim3(plan.threads), 0, st, a);
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
    a.x_row = plan.pixels * x_pixel;
    a.out_row = plan.pixels * out_pixel;
    a.lanes_row = plan.threads / (plan.images * plan.width);
    const bool one = a.D % V == 0, full = plan.pixels * (int64_t)a.groups * a.D % V == 0 && (int64_t)a.G * a.D * plan.pixels % V == 0 && a.P % plan.pixels == 0;
    // as many lanes to a group as there are, up to a wave
    const int groups = plan.images * plan.groups;
    while (a.log_lanes < 6 && (groups << a.log_lanes) < plan.threads) ++a.log_lanes;
    const int size = one ? a.D / V : a.D;
    a.step_d = (1 << a.log_lanes) % size;
    a.step_r = (1 << a.log_lanes) / size;
    a.stream = sizeof(O) <= sizeof(X) && (int64_t)a.groups * a.D * sizeof(O) % 128 == 0 && a.out_row * sizeof(O) % 128 == 0 && a.out_image * sizeof(O) % 128 == 0 && aligned_to(a.out, 128);
    if (one) return norm_launch<X, O, true, true>(a, plan, st);
    return full ? norm_launch<X, O, true, false>(a, plan, st) : norm_launch<X, O, false, false>(a, plan, st);
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
