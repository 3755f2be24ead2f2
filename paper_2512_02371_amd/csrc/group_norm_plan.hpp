// hb_group_norm: how a call's pixels and channels are dealt to workgroups; host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace hb {

constexpr int kNormThreads = 1024;        // most of a workgroup
// Most vectors of a lane that stay in registers, 256 KB of a workgroup of 1024; fewer where each element of a vector of 8 has sums of its own.
constexpr int norm_slots(int V, bool one) { return V == 8 && !one ? 14 : 16; }
constexpr int kNormWorkgroups = 512;      // that read chunks of streaming rows
constexpr int kNormJoin = 8;              // chunks of a lane that joins them
constexpr int kNormFewChunks = 64;        // of a group, that need no launch to be joined
static_assert(kNormWorkgroups <= 64 * kNormJoin, "a wave joins them");
constexpr int kNormBatch = 8;             // vectors of a lane under way at one time where pixels stream

// Rows are pixels, or, where pixels are no whole vectors and stand without gaps, so many pixels that they are (`pixels` of them; their channels repeat).  A workgroup
// takes `groups` neighbouring groups of channels, `width` vectors, of `images` images; its lanes stand side by side along them and in `threads` /
// (images * width) rows.
struct NormPlan {
    bool slab;                            // all rows of the groups stay in the workgroup's registers; else they stream by, twice
    int pixels, groups, images, width, threads;
    int rows;                             // of an image
    int blocks;                           // of groups
    int log_lanes;                        // 2^this lanes add up a group
    int passes;                           // slab: vectors of a lane
    int chunk, chunks;                    // else: rows of a workgroup, workgroups along them
    int apply_chunk, apply_chunks;        // and of those that read the rows again
    bool join;                            // the chunks of a group are joined by a launch of its own
};

// As many lanes to a group as there are, up to a wave.
inline int norm_log_lanes(int groups, int threads) {
    int n = 0;
    while (n < 6 && groups << n < threads) ++n;
    return n;
}
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
    const auto fits = [&](int groups) { return width(groups) <= kNormThreads && (int64_t)((p.rows - 1) / (kNormThreads / width(groups)) + 1) <= norm_slots(V, D % V == 0); };
    p.groups = least;
    // A slab's time is that of its workgroup, whose one compute unit has some 0.07 us of arithmetic and transfers for a KB (0.13 where the elements of a vector have sums of their
    // own), or that of all the bytes, 0.42 us a MB, and 5 us besides; reading twice takes 10 us and 0.52 a MB.  Fitted to 30 calls, silu, of 1 x 64 x 512 to 8 x 4096 x 1024
    // in 32 groups; 2 x 1024 x 640 14.3 us as slabs of 80 KB and 10.6 read twice, 16 x 256 x 1280 9.9 of 20 KB and 14.5, 1 x 16384 x 256 48 and 12.8.
    const double all_MB = (double)N * P * C * size / 1e6;
    const auto slab = [&](int groups) {
        const double kb = (double)width(groups) * p.rows * 0.016, alone = 5.0 + kb * (D % V == 0 ? 0.065 : 0.125), all = 5.5 + 0.42 * all_MB;
        return alone > all ? alone : all;
    };
    if (fits(least) && slab(least) <= 10.2 + 0.52 * all_MB) {
        p.slab = true;
        const auto wgs = [&](int groups) { return (int64_t)N * ((G - 1) / groups + 1); };
        // whole lines where there are workgroups enough, and not too small ones where there are many
        while (p.groups < G) {
            const int next = p.groups * 2 < G ? p.groups * 2 : G;
            if (!fits(next) || slab(next) > 1.1 * slab(p.groups)) break;
            const bool lines = (int64_t)p.groups * D * size < 128 && wgs(next) >= 64;
            const bool small = (int64_t)width(p.groups) * p.rows < 2048 && wgs(next) >= 1024;
            if (!lines && !small) break;
            p.groups = next;
        }
        if (p.groups == G)
            while ((int64_t)width(G) * p.rows * p.images < 512 && 2 * p.images * width(G) <= 256 && N / (2 * p.images) >= 1024) p.images *= 2;
        p.width = width(p.groups);
        const int all = p.images * p.width;
        // where workgroups are many, few lanes with many vectors each, so that several workgroups share a compute unit, some reading while others write (64 images
        // of 512 x 1024, 1024 workgroups: 43 us with 1024 lanes, 32 with 256); else many lanes, which are done sooner
        const int most = ((int64_t)(N - 1) / p.images + 1) * ((G - 1) / p.groups + 1) >= 512 ? norm_slots(V, D % V == 0) : 4;
        for (p.threads = 64; p.threads < kNormThreads; p.threads *= 2)
            if (all <= p.threads && (p.rows - 1) / (p.threads / all) + 1 <= most) break;
        p.passes = (p.rows - 1) / (p.threads / all) + 1;
        p.blocks = (G - 1) / p.groups + 1;
        p.log_lanes = norm_log_lanes(p.images * p.groups, p.threads);
        return p;
    }
    p.threads = 256;
    while (width(p.groups) > p.threads) p.threads *= 2;
    const auto others = [&](int groups) { return (int64_t)N * ((G - 1) / groups + 1); };
    // as wide as a workgroup, but whole lines alone while that leaves too few workgroups with few chunks to join
    while (p.groups < G) {
        const int next = p.groups * 2 < G ? p.groups * 2 : G;
        if (width(next) > p.threads || ((int64_t)p.groups * D * size >= 128 && others(next) * kNormFewChunks < kNormWorkgroups / 2)) break;
        p.groups = next;
    }
    p.width = width(p.groups);
    p.blocks = (G - 1) / p.groups + 1;
    const int across = p.threads / p.width;
    const auto share = [&](int batch, int wgs, int& chunk, int& chunks) {
        const int64_t wanted = others(p.groups) >= wgs ? 1 : wgs / others(p.groups), most = (p.rows - 1) / (across * batch) + 1;
        const int64_t parts = wanted < most ? wanted : most;
        chunk = (int)((((p.rows - 1) / parts) / across + 1) * across);
        chunks = (p.rows - 1) / chunk + 1;
    };
    // a workgroup to a compute unit, so that few parts are joined, where that is a large part of the time (1 x 16384 x 256 12.8 us, with twice as many 14.1, with twice and eight times as
    // many 14.8; 8 x 4096 x 320 21.8, 22.1, 25.7); else enough for some to read while others write (2^20 x 64 with 512 and 2048 4 % faster than with 256 and 1024)
    const bool many = all_MB >= 64;
    share(2, many ? kNormWorkgroups : kNormWorkgroups / 2, p.chunk, p.chunks);
    share(2, many ? 4 * kNormWorkgroups : kNormWorkgroups / 2, p.apply_chunk, p.apply_chunks);
    p.log_lanes = norm_log_lanes(p.groups, p.threads);
    p.join = p.chunks > kNormFewChunks || p.chunks > kNormJoin << p.log_lanes;
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
