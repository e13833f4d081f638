// Attention of a tree of drafted tokens with few rows per value head (drafts x heads of a group <= 32) on the
// wide decode's kernel (kl_decode_wide_kernel.cuh, kTree): there a tile costs what its 16 or 32 rows cost,
// where a block of kl_tree_tc.cu costs 128 rows, and the splits merge inside.
// fp32 outputs take operands of three bf16 terms (24 bits) in the place of two.
// Measured, 32 / 8 heads: 4 drafts on 700 tokens 10.3 us (13.6 in kl_tree_tc.cu; latency), with fp32 outputs 10.4
// (22.7); 8 sequences of 4096 tokens, 8 drafts 25.6 us (37; HBM 10, the rest the start-up and one run of 32 tiles
// in each of 128 CTAs), fp32 27 (59); 64 of 8192, 4 drafts 176 us (6130 GB/s), fp32 200 (520), 8 drafts 227 us
// (the tile chain of 32 rows); one of 131072, 8 drafts 61 us (HBM 40).
#include "kl_rows_wide.cuh"

namespace kl {
namespace {

// Splits per CTA of g.S splits of up to `tiles` tiles for `ctas` blocks (units times blocks of rows) on `slots`
// places.
inline int rows_splits_per_cta(const Geometry &g, int64_t tiles, int64_t ctas, int64_t slots) {
    int spc = splits_per_cta(g.S, ctas, slots);
    // That fits one wave where it can, even if it leaves places empty; shorter runs in several waves where they are
    // done a tenth sooner, a CTA costing 8 tiles' time by itself (10 sequences of 40000 tokens, 4 drafts of 64 / 8
    // heads 215 -> 168 us, 2 drafts 162 -> 140).
    const auto cost = [&](int n) {
        return (ctas * ((g.S + n - 1) / n) + slots - 1) / slots * ((tiles * n + g.S - 1) / g.S + 8);
    };
    int best = spc;
    for (int n = (g.S + kWideMaxRuns - 1) / kWideMaxRuns; n < spc; ++n)
        if (cost(n) < cost(best)) best = n;
    if (cost(best) * 10 < cost(spc) * 9) spc = best;
    // (and no more than four waves of CTAs, each of which pays a start: a split count of the caller's may ask for
    // any number of short runs)
    while (spc < g.S && (g.S + spc - 1) / spc * ctas > 4 * slots) ++spc;
    return spc;
}

template <int NH, int NG, int T>
cudaError_t launch_tree(const DecodeArgs &la, const CUtensorMap &vmap, const CUtensorMap &wmap,
                        const CUtensorMap &qmap) {
    return la.wait_ns < kExactWaitNs ? launch_kernel_wide<NH, NG, true, kForest, T>(la, vmap, wmap, qmap)
                                     : launch_kernel_wide<NH, NG, false, kForest, T>(la, vmap, wmap, qmap);
}

}  // namespace

cudaError_t launch_tree_wide(const DecodeArgs &a) {
    DecodeArgs la = a;
    Geometry &g = la.geo;
    const int rows = g.G * a.tree.max_q;
    const int64_t sms = device_sm_count(), units = (int64_t)g.B * g.Hkv;
    const bool fp32 = a.out_dtype == KL_FP32, w32 = rows > 16 && g.nhb == 1;
    // Two CTAs per SM as the decode's blocks of heads. With three terms these have rings of two tiles, which
    // suits short caches alone (fp32, 32 / 8 heads, two and one per SM: 64 sequences of 1000 tokens, 4 drafts 43.6
    // and 51.5 us, 16 of 4096, 8 drafts 54 and 70, 64 of 8192 208 and 196, of 64 / 8 heads 370 and 297).
    const int64_t tiles = ((int64_t)g.max_pages * g.P + 127) / 128;
    const bool two_per_sm = !w32 && units * g.nhb > sms && (!fp32 || tiles <= 32);
    g.qbox = rows;
    const int64_t slots = two_per_sm ? 2 * sms : sms, ctas = units * g.nhb;
    g.spc = rows_splits_per_cta(g, tiles, ctas, slots);
    CUtensorMap vmap, wmap, qmap;
    if (!rows_maps(a, g.G, a.tree.max_q, &vmap, &wmap, &qmap)) return cudaErrorInvalidValue;
    if (fp32)
        return two_per_sm ? launch_tree<16, 1, 3>(la, vmap, wmap, qmap) : launch_tree<16, 2, 3>(la, vmap, wmap, qmap);
    if (w32) return launch_tree<32, 2, 2>(la, vmap, wmap, qmap);
    return two_per_sm ? launch_tree<16, 1, 2>(la, vmap, wmap, qmap) : launch_tree<16, 2, 2>(la, vmap, wmap, qmap);
}

}  // namespace kl
