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
// A part costs a start (about 5 us), a state and the merge (3 to 5 us). A tile takes 1.2 us with bf16 outputs, 2.7
// with fp32 outputs. Cuts fall on multiples of kTreeCut tiles. (32 / 8 heads, bf16, at 1 us per tile: one sequence
// of 4096 tokens, 16 drafts, with runs of 8 tiles and more 23.9 us, of 2 19.4; 4 of 1000 tokens in one part each
// 16.2, cut 20.5. fp32: one of 4096 tokens, 16 drafts, with runs of 8 tiles 42.9 us, of 4 33.3, of 2 25.8; one of 700, 4
// drafts, in one part 24.3, cut 22.8; 64 of 1000 114 and 117.)
constexpr int kTreeCut = 2, kTreeRun = 2;
constexpr int kTreeStart = 5, kTreeWhole = 8;
constexpr int kTreeStartFp32 = 2, kTreeWholeFp32 = 4;
constexpr int kTreeMaxRuns = 512;   // (one per SM; the merge lists a unit's parts in shared memory)
// The pipeline of a segment: softmax groups (half tile u is group u % kTreeGroups'), buffers of scores with bf16
// and with fp32 outputs, and with fp32 outputs the half tiles between two moves of O to its sum and the barriers
// on which the references are announced (half tile u's on u % kTreeTurns, phase u / kTreeTurns). A wait by parity
// holds only while its barrier is in that phase or the next one: with a barrier per group the softmax could
// pass two half tiles, and with them two phases, before the warps that move O came to wait for the first.
constexpr int kTreeGroups = 2, kTreeSub = 3, kTreeSubFp32 = 2, kTreeFold = 2, kTreeTurns = 4;
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

// How a call with `rows` rows per value head (drafts x heads of a group) over `units` (sequence, value head) pairs
// of up to `tiles` tiles runs: in blocks of 128 rows (0, kl_tree_tc.cu), or on the wide decode's kernel in one
// block of 16 or 32 rows (1) or two of 16 (2). `per_qh`: W^R per query head.
// - Two blocks of 16: three terms, or the routing by a W^R per query head, leave no tensor memory for 32 rows. Else
//   a tile takes a block of 32 0.87 us and one of 16 0.62, but the block of 32 starts 4 us later, so while
//   every CTA has an SM and few tiles. (bf16, 8 drafts of 32 / 8 heads: one sequence of 300 tokens in two blocks
//   9.5 us, in one 13.3; of 131072 78.5 and 60.7; 8 of 4096 25.3 and 26.5; 16 of 4096 45 and 35. W^R per query
//   head, in two blocks and in 128 rows: 8 of 4096 26.2 and 38.9, one of 131072 80.3 and 78.9, 64 of 1000 72.3 and
//   69.1; fp32 8 of 4096 26.5 and 59.)
// - Blocks of 128 rows for many short units, whose starts a persistent CTA pays without a launch wave's rest (8
//   drafts of 32 / 8 heads in 128 rows and in one block: 64 of 500 tokens 47 and 58 us, of 1000 65.5 and 69.3, of
//   1500 85.6 and 82.1, of 2000 100 and 93, 32 of 1000 35.0 and 35.7, of 2000 61 and 47).
inline int tree_wide_blocks(int64_t units, int64_t tiles, int64_t rows, bool fp32, bool per_qh, int64_t sms) {
    if (rows > 32) return 0;
    if (rows <= 16) return 1;
    if (fp32 || (2 * units <= sms && units * tiles <= 16 * sms)) return 2;
    return per_qh || (units > sms && tiles <= 8) ? 0 : 1;
}

}  // namespace kl
