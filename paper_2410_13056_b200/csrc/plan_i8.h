// How a product of 8-bit codes is covered, chosen from sizes: host code without CUDA.
#pragma once

#include <algorithm>
#include <cstdint>

namespace cmpq {

struct ProductSize {
    int64_t n, cols;  // tokens; rows of weights (of a gated product those of both projections)
    int64_t kblocks;  // 128-byte blocks of the sum
    int64_t sms;
};

struct ProductPlan {
    bool pair;      // pairs of CTAs on tiles of 256 tokens, or tiles of 128
    int bn, rows;   // columns of a tile; token rows that a box brings
    int parts;      // CTAs of a cluster that share a tile's sum
    int slices;     // of a tile's sum, over an instruction
    int per_stage;  // tiles of 128: blocks of the sum in a stage
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int tile_rows(const ProductSize& p) { return (int)std::min<int64_t>(128, ceil_div(p.n, 8) * 8); }

// Cycles that a way to cover the product takes, from sizes: rounds of blocks over the SMs, in each the blocks of the sum
// at the pace of the products or of the loads (64 bytes a cycle and SM), and what a round or launch costs besides; not
// less than the weights' way from memory (3400 bytes a cycle).  Fitted to sweeps of bn over 1 to 512 tokens and layers of
// 4096 x 4096 to 8192 x 28672, where the choice is within 3 % of the best; e.g. 256 x 4096 x 11008: bn = 160 17.4 us, 176 17.7,
// pairs of 160 17.2; 512 tokens: pairs of 160 24.3, 192 25.7, 256 29.9.
inline int64_t tile_cycles(const ProductSize& p, int bn) {
    const int64_t rounds = ceil_div(ceil_div(p.n, 128) * ceil_div(p.cols, bn), p.sms);
    const int64_t pace = std::max<int64_t>(4 * std::max(32, bn / 2), (bn + std::min<int64_t>(p.n, 128)) * 2);
    return std::max(rounds * p.kblocks * pace, p.kblocks * 128 * p.cols / 3400) + rounds * (9000 + 8 * bn);
}
inline int64_t pair_cycles(const ProductSize& p, int bn) {
    return ceil_div(ceil_div(p.n, 256) * ceil_div(p.cols, bn), std::max<int64_t>(1, p.sms / 2)) * p.kblocks * (600 * (256 + bn) / 512) + 14000;  // the pace is that of the loads
}

// Slices of a tile's sum, for products that no cluster shares.  Shorter sums are not worth the adding up, and wider tiles wait for
// memory: 32 tokens 2048 -> 2048 6.0 -> 6.6 us with four slices, 53 tokens 4096 -> 4096 9.2 -> 9.5 and 28672 -> 8192 45.8 -> 46.9
// with two.
inline int slices_of(const ProductSize& p, int bn) {
    const int rows = tile_rows(p);
    return bn > 32 ? 1 : rows <= 32 && p.kblocks > 16 ? 4 : rows <= 64 && p.kblocks > 32 ? 2 : 1;
}

// The same with `parts` CTAs of a cluster to a tile, or one, to compare the two.  Here the loads' way from L2 and the weights' from
// memory delay one another, and a cluster pays 3300 cycles for its two barriers and for sums that cross it.  Fitted to 600 calls
// of 5 to 512 tokens, 2304 x 512 to 28672 x 12288: what it chooses is 1 % slower than the best of them in the mean (14 % at most).
// Over 166 calls that it gave to clusters, they took 0.78 of the time that tiles and pairs had taken (0.54 to 1.02).
inline int64_t parts_cycles(const ProductSize& p, int parts, int bn, int slots) {
    const int64_t rounds = ceil_div(ceil_div(p.n, 128) * ceil_div(p.cols, bn), slots);
    const int rows = tile_rows(p), slices = parts > 1 ? 1 : slices_of(p, bn);
    const int64_t loads = rounds * ceil_div(p.kblocks, parts) * std::max(2 * std::max(64, bn) / slices, (bn + rows) * 2);
    const int64_t memory = p.kblocks * 128 * p.cols / 3400;
    return std::max(loads, memory) + std::min(loads, memory) * 2 / 5 + rounds * (10000 + 7 * bn) + (slices > 1 ? 2000 : 0) +
           (parts > 1 ? 3300 + rows * (bn - bn / parts) * 2 / 5 : 0);
}

// Whether a stage of a tile holds one block of the sum.  Stages of several are for long sums in narrow tiles, whose weights memory
// brings faster the more of a row is asked for at a time (5 tokens 13824 -> 5120, 48 channels to a tile: 22.8 us with one block, 18.8
// with 64 KB; 28672 -> 8192, 64 channels 48.3 and 42.5); else the first products wait for more bytes than they need, and stages are few
// (4096 -> 4096, 320 tokens, 96 channels 11.3 and 12.6; 8192 -> 8192, 80 tokens, 64 channels 16.7 and 18.5; 11008 -> 4096, 512 tokens,
// 112 channels 25.6 and 28.7).  From 302 calls of 5 to 2048 tokens in tiles, 512 -> 1408 to 28672 -> 8192.
inline bool stage_of_one(const ProductSize& p, int bn) { return (bn - 16) * (bn - 16) > 32 * p.kblocks; }

// Tokens up to which clusters take the place of pairs.  Past the calls of the fit they do not pay: where the model would choose them for
// 513 to 4400 tokens, 11008 -> 4096 to 28672 -> 8192, they took 0.98 to 1.39 times as long as pairs (1.19 in the mean of 50 calls), in
// long streams 1.04 to 1.31 (1.17 of 68; 28672 -> 8192, 4200 tokens 923 us and 727; 11008 -> 4096, 1408 tokens 80 and 59).  A CTA of a split
// tile loads 48 KB for what one of a pair gets from 32.
constexpr int kClusterTokens = 512;

// slots(parts): clusters of so many CTAs that run at once, 0 where there are none.
template <class Slots>
inline ProductPlan plan_product(const ProductSize& p, Slots slots) {
    ProductPlan a = {};
    int64_t tile = INT64_MAX, pair = INT64_MAX, widest = INT64_MAX;
    int wide = 0;
    for (int bn = 32; bn <= 256; bn += 16)
        if (const int64_t cycles = tile_cycles(p, bn); cycles < tile) tile = cycles, a.bn = bn;
    for (int bn = 256; p.n > 128 && bn >= 128; bn -= 32)  // narrower where that fills the last round better
        if (const int64_t cycles = pair_cycles(p, bn); cycles < pair) pair = cycles, wide = bn, widest = bn == 256 ? cycles : widest;
    // The pace of narrow pairs is right beside wide ones, but a little too good beside tiles: where it promised less than 4 %, they took
    // 0.99 to 1.09 times as long (12288 -> 2304, 900 tokens 29.5 us in tiles and 32.1, 8192 -> 1024, 2900 tokens 30.0 and 31.8).
    a.pair = widest < tile || (p.n > 128 && pair + pair / 20 < tile);
    if (a.pair) a.bn = wide;
    // A few wide tiles with long sums: two or four CTAs to a tile.  A CTA finishes whole groups of eight channels.
    a.parts = 1;
    if (p.kblocks > 16 && (!a.pair || p.n <= kClusterTokens)) {
        int64_t least = a.pair ? (pair - 14000) * 14 / 10 + 14200 : parts_cycles(p, 1, a.bn, (int)p.sms);  // pairs by the same fit
        // which had stages of several blocks everywhere: without this, clusters were up to 6 % slower (11008 -> 4096, 384 tokens)
        if (!a.pair && slices_of(p, a.bn) == 1 && stage_of_one(p, a.bn)) least = least * 14 / 15;
        for (int c = 2; c <= 4; c *= 2) {
            const int at_once = slots(c);
            for (int bn = 16 * c; at_once > 0 && bn <= 256; bn += 16 * c)
                if (const int64_t cycles = parts_cycles(p, c, bn, at_once); cycles < least) least = cycles, a.bn = bn, a.parts = c, a.pair = false;
        }
    }
    a.rows = a.pair ? 128 : tile_rows(p);
    a.slices = a.pair || a.parts > 1 ? 1 : slices_of(p, a.bn);
    // wide tiles of clusters have more rows of weights on the way at once: 100 tokens 28672 -> 8192 47.9 -> 46.9 us with 48 KB, but
    // 20480 -> 5120, in tiles of 96 channels, 26.8 -> 29.2
    const int block = a.slices * (a.rows + a.bn) * 128, stage = p.n > 32 && (a.parts == 1 || a.bn < 128) ? 64 << 10 : 48 << 10;
    a.per_stage = (int)std::max<int64_t>(1, std::min<int64_t>(stage / block, ceil_div(p.kblocks, a.parts * a.slices)));
    if (a.parts == 1 && a.slices == 1 && stage_of_one(p, a.bn)) a.per_stage = 1;
    return a;
}

}  // namespace cmpq
