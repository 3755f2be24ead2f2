// hb_group_norm: how a call's pixels and channels are dealt to workgroups; host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace hb {

constexpr int kNormThreads = 1024;        // most of a workgroup
constexpr int kNormSlots = 16;            // most vectors of a lane that stay in registers: 256 KB of a workgroup
constexpr int kNormBatch = 8;             // vectors of a lane under way at one time where pixels stream

// Rows are pixels, or, where pixels are no whole vectors and stand without gaps, so many pixels that they are (`pixels` of them; their channels repeat).  A workgroup
// takes `groups` neighbouring groups of channels, `width` vectors, of `images` images; its lanes stand side by side along them and in `threads` /
// (images * width) rows.
struct NormPlan {
    bool slab;                            // all rows of the groups stay in the workgroup's registers; else they stream by, twice
    int pixels, groups, images, width, threads;
    int rows;                             // of an image
    int blocks;                           // of groups
    int passes;                           // slab: vectors of a lane
    int chunk, chunks;                    // else: rows of a workgroup, workgroups along them
};

inline int norm_gcd(int a, int b) { return b ? norm_gcd(b, a % b) : a; }

// V: elements of a vector; dense: no gaps between the pixels of x and of out.
inline NormPlan norm_plan(int N, int P, int C, int G, int V, bool dense) {
    const int D = C / G, size = 16 / V;
    NormPlan p = {};
    p.images = 1;
    p.pixels = C % V && dense && C / norm_gcd(C, V) <= kNormThreads && P >= V / norm_gcd(C, V) ? V / norm_gcd(C, V) : 1;
    p.rows = (P - 1) / p.pixels + 1;
    const auto width = [&](int groups) { return (int)(((int64_t)p.pixels * groups * D - 1) / V + 1); };
    // blocks of whole vectors where there are any that are not too wide; all groups where pixels share a row
    int least = p.pixels > 1 ? G : C % V ? 1 : V / norm_gcd(D, V);
    if (width(least) > kNormThreads) least = 1;
    const auto fits = [&](int groups) { return width(groups) <= kNormThreads && (int64_t)((p.rows - 1) / (kNormThreads / width(groups)) + 1) <= kNormSlots; };
    p.groups = least;
    if (fits(least)) {
        p.slab = true;
        const auto wgs = [&](int groups) { return (int64_t)N * ((G - 1) / groups + 1); };
        while (p.groups < G) {
            const int next = p.groups * 2 < G ? p.groups * 2 : G;
            if (!fits(next)) break;
            const bool lines = (int64_t)p.groups * D * size < 128 && wgs(next) >= 64;
            const bool small = (int64_t)width(p.groups) * p.rows < 2048 && wgs(next) >= 1024;
            if (!lines && !small) break;
            p.groups = next;
        }
        if (p.groups == G)
            while ((int64_t)width(G) * p.rows * p.images < 512 && 2 * p.images * width(G) <= 256 && N / (2 * p.images) >= 1024) p.images *= 2;
        p.width = width(p.groups);
        const int all = p.images * p.width;
        for (p.threads = 64; p.threads < kNormThreads; p.threads *= 2)
            if (all <= p.threads && (p.rows - 1) / (p.threads / all) + 1 <= 4) break;
        p.passes = (p.rows - 1) / (p.threads / all) + 1;
        p.blocks = (G - 1) / p.groups + 1;
        return p;
    }
    p.threads = 256;
    while (width(p.groups) > p.threads) p.threads *= 2;
    while (p.groups < G) {
        const int next = p.groups * 2 < G ? p.groups * 2 : G;
        if (width(next) > p.threads) break;
        p.groups = next;
    }
    p.width = width(p.groups);
    p.blocks = (G - 1) / p.groups + 1;
    const int batch = p.threads / p.width * kNormBatch;
    const int64_t others = (int64_t)N * p.blocks, wanted = others >= 2048 ? 1 : 2048 / others, most = (p.rows - 1) / batch + 1;
    const int64_t chunks = wanted < most ? wanted : most;
    p.chunk = (int)((((p.rows - 1) / chunks) / batch + 1) * batch);
    p.chunks = (p.rows - 1) / p.chunk + 1;
    return p;
}

// Bytes for the chunks' statistics and what becomes of them, whatever the types and strides.
inline size_t norm_workspace(int N, int P, int C, int G) {
    size_t most = 0;
    for (int V : {4, 8})
        for (bool dense : {false, true}) {
            const NormPlan p = norm_plan(N, P, C, G, V, dense);
            const size_t need = p.slab ? 0 : ((size_t)N * G * (p.chunks + 1) * 8 + 255) / 256 * 256;
            most = need > most ? need : most;
        }
    return most;
}

}  // namespace hb
