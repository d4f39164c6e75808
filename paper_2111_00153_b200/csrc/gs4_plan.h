// What the products of group-scaled layers (gs4_product.cu, gs4_tensor.cu) are launched with, from sizes, types and alignment alone: host arithmetic
// without CUDA, so that a test can ask which form a shape gets.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>
#include "../../include/rmsmp.h"

#ifdef __CUDACC__
#define RMSMP_HOST_DEVICE __host__ __device__
#else
#define RMSMP_HOST_DEVICE
#endif

namespace rmsmp {

struct Gs4Sizes {
    int64_t R;                           // rows of y
    int E, tiles, Kp, sums, block_bytes; // of the layer
    int x_type;
    bool experts, in_order, x_vec;       // rows by offsets; without an index; rows of x 16-byte aligned
    int sms;
};

constexpr int kGs4MostSmem = 226 * 1024;

// ---- which kernel
// Up to eight columns (an fp32 token is two) by the few-token kernel, more on tcgen05; of experts, which have tiles enough for every SM, up to 24 on average.
// (8192 x 8192, 8 and 16 bf16 tokens: 16 and 26 us by the one, 31 and 31 by the other; 4096 x 4096: 9.3 and 11.2, 11.0 and 11.2; 1024 x 1024: 5.1 and 5.6,
// 5.2 and 5.2.  64 experts of 1408 x 2048, 16, 24 and 25 tokens each: 56 by the one and 109 by the other, 78 by the one, 96 by the other; eight of 4096 x 4096: 65 and 65, 88 and 66; 256 of 256 x 256, 16: 12 and 30.
// One number of columns for all sizes takes the slower of the two for 9 to 16 tokens of 8192 x 8192, and for 17 to 24 an expert of eight large ones.)
inline bool gs4_many_tokens(int64_t R, int E, int x_type, bool experts)
{
    const int64_t tokens = experts ? (R + E - 1) / E : R;
    return tokens * (x_type == RMSMP_F32 ? 2 : 1) > (experts ? 24 : 8);
}

// ---- few tokens
constexpr int kGs4FewWarps = 8;
constexpr int kGs4FewRing = 2;           // copies that a warp has in flight or at hand
// Blocks of a copy.  With sixteen columns, which many short CTAs of experts have, two CTAs fit on an SM if it is one (64 experts of 1408 x 2048, 16 tokens each:
// 56 us, 70 with two; eight of 4096 x 4096, where one fits at most: 69 and 65); with eight they fit, and more in flight is better (2 tokens each: 21 us, 26 with one).
RMSMP_HOST_DEVICE constexpr int gs4_few_chunk(int nt) { return nt == 1 ? 2 : 1; }
constexpr int kGs4FewRed = 36;           // floats between columns of a block's partial sums (32 rows, padded against bank conflicts)

struct Gs4FewPlan {
    int wr, wk, split;                   // row blocks x input shares of a CTA's warps; CTAs of a cluster
    int per, groups;                     // row blocks of a CTA (a multiple of wr); CTAs (clusters) that share a matrix's rows
    int slice, slab;                     // inputs of a CTA, and of one stage of x in shared memory (multiples of 128)
    int alone;                           // a warp has all inputs of its row blocks (wk = split = 1, one stage): it stores its sums itself
    int single;                          // ... of its one row block, sixteen columns: they pass through its ring, which nothing comes into any more
    int tokens, parts;                   // tokens of one pass over the weights; columns of a token
    int nt;                              // columns / 8
    size_t smem;
    int64_t grid;
};

inline Gs4FewPlan gs4_plan_few(const Gs4Sizes& a)
{
    Gs4FewPlan p = {};
    p.parts = a.x_type == RMSMP_F32 ? 2 : 1;
    const int64_t expect = a.experts ? std::max<int64_t>(1, (a.R + a.E - 1) / a.E) : a.R;      // tokens of a matrix
    // (64 experts of 1408 x 2048, 4 tokens each on average: 35 us eight columns at a time, 40 sixteen; 16 tokens: 81 and 71, and 56 with what gs4_few_chunk does.)
    const int nt = p.nt = expect * p.parts <= 8 ? 1 : 2;
    p.tokens = 8 * nt / p.parts;
    if (!a.experts) p.tokens = (int)std::min<int64_t>(p.tokens, a.R);
    const int64_t busy = a.experts ? std::min<int64_t>(a.E, a.R) : 1;                          // matrices with tokens, at most
    const int cols = p.tokens * p.parts, units = a.Kp / 128, sms = a.sms;
    const size_t ring = (size_t)kGs4FewWarps * kGs4FewRing * gs4_few_chunk(nt) * a.block_bytes;
    const size_t column = 2, factor = a.x_type == RMSMP_F16 ? 0 : (size_t)a.sums * 8 * nt * sizeof(float);      // bytes: of an input and column; of 128 inputs
    // Which rows and inputs a warp, a CTA and a cluster take: the least of an estimate in microseconds.  An SM streams 44 KB a microsecond, a warp alone a block in
    // 0.4; a CTA takes 4 to start, find its tokens and end, x comes in at 10 KB a microsecond, behind the weights' first copies, a cluster's join takes 2.
    // (8192 x 8192, one bf16 token: 13.1 us with whole rows a CTA, 12.7 with quarters; 1024 x 1024: 3.5 and 4.3; eight tokens, 16384 x 8192: quarters 22.9 us, halves 24.6, whole
    // rows 37; 32768 x 4096: whole rows 25, eighths with several row blocks a warp 56.  64 experts of 1408 x 2048, 4 tokens each: eight row blocks a CTA 33 us,
    // four 35, two 46; 8 tokens of 8: two 8.3, four 8.0, eight 11; eight experts of 4096 x 4096, 4 tokens: 24.3, halved in a cluster 23.4.)
    float best = 1e30f;
    for (int wr = 1; wr <= kGs4FewWarps; wr *= 2)
        for (int split = 1; split <= 8 && split <= units; split *= 2) {
            const int wk = kGs4FewWarps / wr, slice = (units + split - 1) / split;
            const size_t shared_by_all = ring + cols * 64, stage = slice * (128 * column * cols + factor), sums = (size_t)wr * wk * 8 * nt * kGs4FewRed * sizeof(float);
            const bool alone = wk == 1 && split == 1 && shared_by_all + sums + stage <= (size_t)kGs4MostSmem, single = alone && nt == 2;      // (only experts have sixteen columns)
            // Row blocks of a warp: as many as make one wave, half of them, or one.  (Experts' tokens differ: more and shorter CTAs even out; `single` relies on it.)
            int64_t most = a.experts ? 1 : std::max<int64_t>(1, (a.tiles * split + 2 * sms * wr - 1) / (2 * (int64_t)sms * wr));
            if (!alone) most = std::min<int64_t>(most, 8);
            most = std::min<int64_t>(most, (a.tiles + wr - 1) / wr);
            for (int64_t rounds = most; rounds > 0; rounds = rounds == 1 ? 0 : rounds == most ? (most + 1) / 2 : 1) {
                const int per = (int)rounds * wr;
                const size_t whole = shared_by_all + (single ? 0 : alone ? sums : sums * rounds), need = whole + stage;
                const int64_t ctas = (a.tiles + per - 1) / per * busy * split, at_once = need <= (size_t)kGs4MostSmem / 2 ? 2 : 1;
                const int blocks = (slice + wk - 1) / wk * (int)rounds;
                // (waves: whole ones; of experts, whose CTAs differ, as many as they fill and half a one for the last)
                const int64_t slots = std::max<int64_t>(1, at_once * sms * (split >= 4 ? 7 : 8) / 8);      // (clusters of four and eight leave SMs over)
                const float full = (float)ctas / slots, block_us = std::max(0.4f, std::min(1.0f, full) * at_once * kGs4FewWarps * (a.block_bytes / 44e3f));
                const float waves = full <= 1 ? 1.0f : a.experts ? full + 0.5f : (float)((ctas + slots - 1) / slots);
                const float t = waves * (blocks * block_us + 4.0f + slice * 256e-4f * std::min<int64_t>(p.tokens, expect) * p.parts + (split > 1 ? 2.0f : 0.0f));
                if (t >= best || whole + 128 * column * cols + factor > (size_t)kGs4MostSmem) continue;
                best = t;
                p.wr = wr; p.wk = wk; p.split = split; p.per = per; p.alone = alone; p.single = single;
                p.groups = (a.tiles + per - 1) / per;
                p.slice = slice * 128;
                p.slab = (int)std::min<int64_t>(p.slice, (int64_t)((kGs4MostSmem - whole) / (128 * column * cols + factor)) * 128);
                p.smem = whole + p.slab * column * cols + p.slab / 128 * factor;
            }
        }
    // Passes over the weights: a matrix's last is not full.  (All of 512 tokens with one of 64 experts of 1408 x 2048: 40 us, by CTAs that each go through
    // all of a matrix's tokens 589; where experts have 0 to 14 each, 35.6 and 42.9.)  CTAs behind the last pass there is find nothing to do.
    const int64_t passes = a.experts ? busy + (a.R - busy) / p.tokens : 1;
    p.grid = passes * p.groups * p.split;
    return p;
}

// ---- many tokens
struct Gs4ManyPlan {
    int bn;                              // tokens of a tile
    int split, units;                    // CTAs of a cluster; blocks of 128 inputs of each
    int mtiles;                          // row tiles
    int64_t ntiles;                      // token tiles (experts: as many as there can be)
};

inline Gs4ManyPlan gs4_plan_many(const Gs4Sizes& a)
{
    Gs4ManyPlan p = {};
    p.mtiles = (a.tiles + 3) / 4;
    p.bn = 16;
    const int units = a.Kp / 128;
    const int64_t expect = a.experts ? std::max<int64_t>(1, (a.R + a.E - 1) / a.E) : a.R;      // tokens of a matrix
    const int64_t busy = a.experts ? std::min<int64_t>(a.E, a.R) : 1;
    // Tokens of a tile and CTAs of a cluster: the least of an estimate.  A CTA takes `pace` microseconds for 128 inputs (measured: 4096 x 4096; `bulk`: x by tensor
    // copies), 2.5 to start and to end, a cluster's join another; every SM has one CTA.
    static constexpr struct { int bn; float pace, bulk; } kTiles[] = {{16, 0.75f, 0.72f}, {32, 0.78f, 0.75f}, {64, 0.83f, 0.8f}, {128, 1.05f, 0.95f}, {192, 1.35f, 1.07f}, {256, 1.7f, 1.25f}};
    const bool bulk = a.in_order && a.x_vec;
    float best = 1e30f;
    for (const auto& tile : kTiles) {
        if (tile.bn > 64 && a.x_type == RMSMP_F32) break;
        // (experts' last tiles are half empty on average)
        const float per = a.experts ? std::max(1.0f, (float)expect / tile.bn + 0.5f) : (float)((expect + tile.bn - 1) / tile.bn);
        const int64_t tiles = (int64_t)(busy * per * p.mtiles);
        for (int split = 1; split <= 4 && split <= units; split *= 2) {         // (clusters of eight wait for room: 1024 x 1024, 32 tokens 10.9 us, fours 5.5)
            const float t = (float)((tiles * split + a.sms - 1) / a.sms) * ((units + split - 1) / split * (bulk ? tile.bulk : tile.pace) * (a.x_type == RMSMP_F32 ? 1.8f : 1.0f) + 2.5f + (split > 1 ? 1.0f : 0.0f));
            if (t < best) { best = t; p.bn = tile.bn; p.split = split; }
        }
        if (tile.bn >= (a.experts ? 4 : 1) * expect) break;
    }
    p.ntiles = (a.R + p.bn - 1) / p.bn + (a.experts ? busy : 0);
    p.units = (units + p.split - 1) / p.split;
    return p;
}

}  // namespace rmsmp
