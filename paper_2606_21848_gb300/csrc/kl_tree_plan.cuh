// Launch layout of the tree attention, chosen on the host from sizes alone (plain C++, no CUDA).
#pragma once

#include <stdint.h>

namespace kl {

struct TreePlan {
    int hp;       // heads of a value head's group in a block of 128 rows
    int rpb;      // drafts per block: 128 / hp
    int blocks;   // blocks per (sequence, value head): blocks of heads x blocks of drafts
    int S;        // CTAs that a block's cache tiles are cut over
    int chunk;    // tokens per CTA (a multiple of 128)
};

constexpr int kTreeRows = 128;      // rows of a block
constexpr int kTreeTile = 128;      // cache rows of a tile
// A CTA's set-up, first tiles and epilogue take about as long as this many tiles.
constexpr int kTreeFixedTiles = 6;
// fp32 outputs: the tensor core's adds truncate, so a run's sum in tensor memory covers at most this
// many tokens (error about 2.7e-6 of the result after 4096; the runs are merged in rounded fp32).
constexpr int kTreeMaxChunkFp32 = 4096;

// B sequences, Hkv value heads of G query heads, at most max_q drafts each, tables of max_tokens tokens,
// num_splits CTAs per block (0: chosen here), sms multiprocessors (one CTA each).
inline TreePlan plan_tree(int B, int Hkv, int G, int max_q, int64_t max_tokens, int num_splits, bool fp32,
                          int sms) {
    TreePlan p{1, kTreeRows, 1, 1, 0};
    const auto blocks_of = [&](int hp) {
        const int rpb = kTreeRows / hp;
        return (int64_t)((G + hp - 1) / hp) * ((max_q + rpb - 1) / rpb);
    };
    // the fewest blocks, and the fewest heads per block among equals
    for (int hp = 2; hp <= G && hp <= kTreeRows; ++hp)
        if (blocks_of(hp) < blocks_of(p.hp)) p.hp = hp;
    p.rpb = kTreeRows / p.hp;
    p.blocks = (int)blocks_of(p.hp);

    const int64_t tiles = (max_tokens + kTreeTile - 1) / kTreeTile;
    int64_t S = num_splits;
    if (S == 0) {
        // the split count with the shortest estimate: waves of CTAs x (tiles of a CTA + its fixed cost)
        const int64_t units = (int64_t)(B > 0 ? B : 1) * Hkv * p.blocks;
        int64_t best = -1;
        for (int64_t s = 1; s <= 256 && s <= tiles; ++s) {
            const int64_t waves = (units * s + sms - 1) / sms;
            const int64_t cost = waves * ((tiles + s - 1) / s + kTreeFixedTiles);
            if (best < 0 || cost < best) {
                best = cost;
                S = s;
            }
            if (units * s > 8 * (int64_t)sms) break;
        }
    }
    int64_t per = (tiles + S - 1) / S;                       // tiles per CTA
    if (per < 1) per = 1;
    if (fp32 && per > kTreeMaxChunkFp32 / kTreeTile) per = kTreeMaxChunkFp32 / kTreeTile;
    p.chunk = (int)(per * kTreeTile);
    p.S = (int)((tiles + per - 1) / per);
    if (p.S < 1) p.S = 1;
    return p;
}

}  // namespace kl
