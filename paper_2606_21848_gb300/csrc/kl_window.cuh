// What consecutive query positions see under the causal mask with a sliding window and first tokens that
// stay visible: position p sees t <= p with t < sinks or t > p - window.
#pragma once

namespace kl {

// The cache tiles of 128 tokens that positions p0 .. p1 may see, laid end to end: those of the first tokens,
// then the window's. Token x of this line is token x of the sequence up to `first`, x + shift behind it.
struct WindowSpan {
    int first, shift, len;
};
__host__ __device__ inline WindowSpan window_span(int p0, int p1, int window, int sinks) {
    const int end = p1 + 1, head = ((sinks < end ? sinks : end) + 127) / 128;
    const int low = p0 - window + 1 > 0 ? (p0 - window + 1) / 128 : 0;
    WindowSpan s;
    s.first = head * 128;
    s.shift = low > head ? (low - head) * 128 : 0;
    s.len = end - s.shift;
    return s;
}

// Most tokens of that line for `rows` consecutive positions of a sequence of up to max_tokens tokens (window
// and sinks at most max_tokens): the window and the rows touch one tile more than they fill.
__host__ __device__ inline int64_t window_line(int64_t rows, int64_t window, int64_t sinks, int64_t max_tokens) {
    const int64_t n = ((sinks + 127) / 128 + (window + rows - 2) / 128 + 2) * 128;
    return n < max_tokens ? n : max_tokens;
}

// The rows of a block for max_q positions of G heads per value head: 16 or 32 on the wide decode's kernel, 0: 128 on
// the prefill's. Operands of three bf16 terms (`fine`), and a W^R per query head a place in tensor memory each, leave
// room for 16 there; the prefill's blocks hold one head's rows where each has its W^R.
inline int window_rows(int64_t G, int64_t max_q, bool fine, bool per_qh) {
    const int64_t rows = G * max_q;
    if (rows <= 16) return 16;
    if (per_qh ? max_q > 32 : rows > 32) return 0;
    return fine || per_qh ? 16 : 32;
}

// Most runs of a block: states that one CTA merges (their table and rows take the place of the ring's tiles).
constexpr int kCausalMostRuns = 256;

// How blocks of up to `tiles` tiles of 128 tokens are cut into runs, one per CTA.
struct CausalRuns {
    int splits;      // pieces of a line, of `chunk` tokens each
    int chunk;
    int spc;         // pieces per run
    int whole;       // the first units are one run each
};
// `units` blocks of rows on `slots` places; num_splits: most runs of a block, 0: chosen here; never more than most_states.
// A CTA costs 8 tiles' time by itself.
// - Fewer blocks than places: as many runs as fit one wave, or several waves of shorter runs where these are done a
//   tenth sooner.
// - More: the last wave's blocks alone are cut, where that is done sooner. (128 sequences with a window of 4160, 8 value
//   heads: 1024 blocks on 304 places, in 3.4 waves 197 us, 187 with the last wave cut; 512 blocks of 64 tiles with weights
//   on 152 places 243, 231.)
inline CausalRuns plan_runs(int64_t units, int64_t max_tokens, int num_splits, int64_t slots, int most_states) {
    const int64_t tiles = (max_tokens + 127) / 128;
    const auto cost = [&](int64_t n, int64_t runs) {
        return (n * runs + slots - 1) / slots * ((tiles + runs - 1) / runs + 8);
    };
    const auto cut = [&](int64_t runs, int64_t whole) {
        CausalRuns r;
        r.chunk = (int)((tiles + runs - 1) / runs * 128);
        r.splits = (int)((max_tokens + r.chunk - 1) / r.chunk);
        r.spc = 1;
        r.whole = (int)(r.splits > 1 ? whole : units);
        return r;
    };
    if (num_splits > 0) {
        // (no more than four waves of CTAs, each of which pays a start)
        int64_t runs = num_splits < tiles ? num_splits : tiles;
        if (runs > most_states) runs = most_states;
        while (runs > 1 && runs * units > 4 * slots) --runs;
        return cut(runs, 0);
    }
    const int64_t most = tiles / 2 < most_states ? tiles / 2 : most_states;
    int64_t best = 1;
    if (units < slots) {
        for (int64_t runs = 2; runs <= most && runs * units <= slots; ++runs) best = runs;
        const int64_t one_wave = cost(units, best);
        int64_t other = best;
        for (int64_t runs = best + 1; runs <= most && runs * units <= 4 * slots; ++runs)
            if (cost(units, runs) < cost(units, other)) other = runs;
        if (cost(units, other) * 10 < one_wave * 9) best = other;
        return cut(best, 0);
    }
    // long lines: runs of at most 8192 tokens while these are not too many, so that batches of any lengths balance
    const int64_t pieces = (max_tokens + 8191) / 8192, cap = pieces < most_states ? pieces : most_states;
    if (cap > 1) return cut(cap, 0);
    const int64_t rest = units % slots;
    for (int64_t runs = 2; runs <= 4 && runs <= most; ++runs)
        if (rest && cost(rest, runs) < cost(rest, best)) best = runs;
    return cut(best, units - rest);
}

}  // namespace kl
