// How a product of 8-bit matrices (matmul.cu) is cut into tiles and parts of sums: sizes of the device and of the product
// in, a plan out. No CUDA in here: the host compiles it too.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace mbscan {

constexpr int kGroups = 2;           // of four warps that move sums, chunks in turn
constexpr int kFeatures = 128;       // output features of a tile: lanes of tensor memory
constexpr int kMaxRows = 224;        // rows of a tile: two sums and two sets of scales fit 512 columns
constexpr int kK = 128;              // columns of the sum in a block, which share a scale
constexpr int kMaxStages = 12;
constexpr int kSlots = 4;            // of the ring of scales
constexpr int kSlotBytes = 512 + 1024;                                       // a tile's features, then 256 rows
static_assert(kSlots * kSlotBytes % 1024 == 0, "what follows is swizzled");
constexpr int kScaleColumns = 4 + 8; // of one slot; two sets take turns
constexpr int kPairRows = 64;        // more may be for pairs of CTAs
constexpr int kMaxSplit = 8;
constexpr int kChunk = 32;           // rows of a sum that are moved at a time
constexpr int kBarrierBytes = 360;   // of static shared memory

struct Tiles {
    int features, rows;       // tiles across
    int band;                 // rows of tiles that are taken together, all of them for one column of tiles before the next
    int height;               // rows of a tile, a multiple of 16
    int blocks;               // 128-column blocks of the sum
    int deep;                 // blocks of a stage: 1, 2 or 4
    int split, stages;
    int held;                 // chunks that a group of warps holds in shared memory at a time
    int sums;                 // in tensor memory: two, or one where no CTA has more than a tile
    uint32_t ring;            // bytes of the ring of stages
    uint32_t columns;         // of tensor memory
};
struct MatmulLimits {
    int sms;
    size_t smem_sm, smem_reserved, smem_optin;   // of an SM, of it for each CTA, a CTA's most
};
struct MatmulPlan {
    Tiles t;
    int ctas;                 // 1, or 2: pairs of CTAs share a tile
    int team;                 // CTAs of a cluster: of a pair, or of the parts of a sum
    int64_t teams;
    size_t smem;
};

// clusters(n): clusters of n CTAs that fit the device side by side, with all the shared memory they can have (0: none can
// be launched). rows, n_out, width > 0.
template <typename Clusters>
MatmulPlan plan_matmul(int64_t p_rows, int64_t n_out, int64_t width, bool out_bf16, const MatmulLimits &lim,
                       const Clusters &clusters) {
    MatmulPlan plan;
    Tiles &t = plan.t;
    t.features = (int)((n_out + kFeatures - 1) / kFeatures);
    t.blocks = (int)((width + kK - 1) / kK);
    // rows by 32, so that the stores of a tile end in it, or 16 rows alone
    const int fewest = (int)((p_rows + kMaxRows - 1) / kMaxRows), most_rows = (int)((p_rows + kChunk - 1) / kChunk);
    const auto height = [&](int rows) { return p_rows <= 16 ? 16 : (int)((((p_rows + rows - 1) / rows) + kChunk - 1) / kChunk * kChunk); };
    // Rows of a tile and parts of a sum, where there are fewer tiles than SMs, by what they cost. The unit is a row of one of
    // the operands that a CTA loads for a block of the sum (128 bytes, two cycles, some 1 ns); what a cluster costs over
    // single CTAs, what adding up costs for a row, and what it costs that the clusters do not fit the GPU side by side are
    // fitted to the times of whole products. Microseconds (launches one after the other in a graph) with the fewest tiles
    // and no parts, with the parts that the rule would take of those, with what it takes: 1 x 2048 x 1024 4.6, 3.6, 3.6;
    // 256 x 1024 x 2304 4.9, 4.9, 4.3; 200 x 4608 x 2304 16.1, 11.5, 9.4; 384 x 4608 x 2304 15.8, 12.3, 10.6;
    // 128 x 2304 x 4608 7.4, 7.4, 6.2.
    t.rows = fewest;
    t.split = 1;
    const auto cost = [&](int rows, int split) {
        return (int64_t)((t.blocks + split - 1) / split) * (kFeatures + height(rows)) + (split > 1 ? 1000 + 19 * height(rows) : 0) +
               (split > 2 && t.features * rows > clusters(split) ? 2000 : 0);
    };
    const bool round = (int64_t)t.features * fewest <= lim.sms;   // all tiles at once
    for (int rows = fewest; round && rows <= most_rows && t.features * rows <= lim.sms; ++rows)
        for (int split = 1; split <= kMaxSplit && t.features * rows * split <= lim.sms && 4 * split <= std::max(t.blocks, 4); split *= 2)
            if ((split <= 2 || clusters(split) > 0) && cost(rows, split) < cost(t.rows, t.split)) t.rows = rows, t.split = split;
    // Pairs of CTAs load half of a tile's rows each, but wait for one another: 2800 of those units, fitted in the same way.
    // Microseconds of single CTAs and pairs: 1024 x 2304 x 2304 8.1, 10.1; 256 x 2304 x 9216 8.5, 10.4; 2048 x 4608 x 1024
    // 12.7, 14.7; 4096 x 4608 x 768 17.5, 16.6. Tiles in several rounds: 200 x 2304 x 32000 24.2, 20.4; 64 x 1024 x 32000
    // 8.6, 10.6.
    const int pairs = (t.features + 1) / 2, pair_rows = std::max(fewest, std::min(most_rows, lim.sms / 2 / pairs));
    const bool pair = n_out > kFeatures && p_rows > kPairRows &&
                      (!round || cost(t.rows, t.split) > (int64_t)t.blocks * (kFeatures + height(pair_rows) / 2) + 2800);
    if (pair) {
        t.features = pairs;
        t.rows = pair_rows;
        t.split = 1;
    }
    plan.ctas = pair ? 2 : 1;
    t.height = height(t.rows);
    t.rows = (int)((p_rows + t.height - 1) / t.height);
    t.band = t.rows > 16 ? 4 : 1;   // 65536 x 1024 x 4096: 190 us, with 1 204
    const int64_t tiles = (int64_t)t.features * t.rows;
    plan.team = pair ? 2 : t.split;
    const bool one = tiles <= lim.sms / plan.team;   // tile to a CTA (or team)
    const int unit = (kFeatures + t.height / plan.ctas) * kK;
    const bool tight = t.split > 2 && tiles > clusters(t.split);
    // What a stage costs the warp that issues its products, some 250 cycles beside them, is little next to 4 x 128 columns of
    // few rows (1 x 2304 x 9216: 7.8 us, of two 6.0, of four 5.3; 256 x 2304 x 9216: 9.9, of two 8.6); a pair's products hide it.
    t.deep = pair || tight ? 1 : unit <= 20 * 1024 ? 4 : unit <= 32 * 1024 ? 2 : 1;
    const int stage = t.deep * unit, share = ((t.blocks + t.deep - 1) / t.deep + t.split - 1) / t.split;   // stages of a tile
    const int chunk = kChunk * kFeatures * (out_bf16 ? 2 : 4);
    const int halves = ((t.height + kChunk - 1) / kChunk + kGroups - 1) / kGroups;   // chunks of a group of warps
    // Of several tiles to a CTA all that a group moves of a sum in bf16 is held beside the ring, in fp32 half of it.
    t.sums = one ? 1 : 2;
    t.held = one || out_bf16 ? halves : (halves + 1) / 2;
    const size_t fixed = 1024 + kSlots * kSlotBytes + (one ? 0 : (size_t)kGroups * t.held * chunk);
    const size_t most = lim.smem_optin - kBarrierBytes, beside = lim.smem_sm / 2 - lim.smem_reserved - kBarrierBytes;
    // as deep as it may be (256 x 2304 x 9216: three stages of two blocks 8.5 us, two 10.0), but where the clusters would not
    // fit the GPU side by side then, two CTAs to an SM
    t.stages = std::min((int)(((tight ? beside : most) - fixed) / stage), kMaxStages);
    if (one) t.stages = std::min(t.stages, share);
    const size_t parts = one ? std::max((size_t)kGroups * t.held * chunk, t.split > 1 ? (size_t)t.height * kFeatures * 4 : 0) : 0;
    t.ring = (uint32_t)((std::max((size_t)t.stages * stage, parts) + 1023) / 1024 * 1024);
    // never three to an SM: half of its tensor memory each, CTAs of one tile never wait for columns while others of their
    // cluster wait for them
    plan.smem = std::max(fixed + t.ring, lim.smem_sm / 3);
    for (t.columns = 32; (int)t.columns < t.sums * t.height + 2 * kScaleColumns; t.columns *= 2) {}
    plan.teams = one ? tiles : lim.sms / plan.team;
    return plan;
}

}  // namespace mbscan
