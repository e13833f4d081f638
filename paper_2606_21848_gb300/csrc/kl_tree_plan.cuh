// Launch layout of the tree attention, chosen on the host from sizes alone (plain C++, no CUDA).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace kl {

struct TreePlan {
    int hp;       // heads of a value head's group in a block of 128 rows
    int rpb;      // drafts per block: 128 / hp
    int blocks;   // blocks per (sequence, value head), at most: blocks of heads x blocks of drafts
    int ctas;     // runs that the units' tiles are cut into, at most
    int start;    // what starting a segment takes, in tiles, in the runs' shares
    int run;      // there are no more runs than units or shares of `run` tiles
    int whole;    // units of up to this many tiles are not cut
};

constexpr int kTreeRows = 128;      // rows of a block
constexpr int kTreeTile = 128;      // cache rows of a tile
// A part costs a start (about 5 us), a state and the merge (3 to 5 us). A tile takes 1 us with bf16 outputs, 2.7
// with fp32 outputs. Cuts fall on multiples of kTreeCut tiles. (32 / 8 heads, bf16: one sequence of 4096 tokens,
// 16 drafts, with runs of 8 tiles and more 23.9 us, of 2 19.4; 4 of 1000 tokens in one part each 16.2, cut 20.5.
// fp32: one of 4096 tokens, 16 drafts, with runs of 8 tiles 42.9 us, of 4 33.3, of 2 25.8; one of 700, 4
// drafts, in one part 24.3, cut 22.8; 64 of 1000 114 and 117.)
constexpr int kTreeCut = 2, kTreeRun = 2;
constexpr int kTreeStart = 5, kTreeWhole = 8;
constexpr int kTreeStartFp32 = 2, kTreeWholeFp32 = 4;
constexpr int kTreeMaxRuns = 512;   // (one per SM; the merge lists a unit's parts in shared memory)
// A part's state: O [32][128 rows] float4 and {m, l} [128 rows]. Every run has up to two parts.
constexpr size_t kTreeStateBytes = kTreeRows * 128 * sizeof(float) + kTreeRows * 2 * sizeof(float);

// B sequences, Hkv value heads of G query heads, at most max_q drafts each, tables of max_tokens tokens,
// sms multiprocessors (one CTA each), outputs in fp32 or bf16.
inline TreePlan plan_tree(int B, int Hkv, int G, int max_q, int64_t max_tokens, int sms,
                          bool fp32 = false) {
    TreePlan p{1, kTreeRows, 1, 1, fp32 ? kTreeStartFp32 : kTreeStart, kTreeRun,
               fp32 ? kTreeWholeFp32 : kTreeWhole};
    const auto blocks_of = [&](int hp) {
        const int rpb = kTreeRows / hp;
        return (int64_t)((G + hp - 1) / hp) * ((max_q + rpb - 1) / rpb);
    };
    // the fewest blocks, and the fewest heads per block among equals
    for (int hp = 2; hp <= G && hp <= kTreeRows; ++hp)
        if (blocks_of(hp) < blocks_of(p.hp)) p.hp = hp;
    p.rpb = kTreeRows / p.hp;
    p.blocks = (int)blocks_of(p.hp);
    const int64_t units = (int64_t)(B > 0 ? B : 1) * Hkv * p.blocks;
    const int64_t shared = ((max_tokens + kTreeTile - 1) / kTreeTile + p.start) * units / (p.run + p.start);
    const int64_t most = shared > units ? shared : units;
    const int64_t top = sms < kTreeMaxRuns ? sms : kTreeMaxRuns;
    p.ctas = (int)(most < 1 ? 1 : most < top ? most : top);
    return p;
}

}  // namespace kl
