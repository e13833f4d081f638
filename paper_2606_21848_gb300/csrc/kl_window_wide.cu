// Attention of consecutive positions with a sliding window and first tokens that stay visible, on the wide
// decode's kernel (kl_decode_wide_kernel.cuh, kWindow): the last tokens of decoding, a few drafts in a row.
//
//   out_p = sum_t softmax(scale <q_p W^R, v_t>)_t v_t   over t <= p with t < sinks or t > p - window
//
// A block of up to 16 or 32 (position, head) rows reads the tiles that its positions see and no others, so a step
// costs what the window costs, however long the sequence. HBM bounds it: 256 bytes per visible token and value head.
// Measured: 128 sequences, 64 / 8 heads, window 4096 and 64 first tokens of 8192: 187 us (5.8 TB/s); 64 of 512 to 32768
// tokens, 1 to 4 new ones, 32 / 8 heads, window 2047, fp32 outputs 80 us; one sequence, window 1000: 10.7 us.
#include "kl_rows_wide.cuh"

namespace kl {
namespace {

template <int NH, int NG, int T>
cudaError_t launch_window(const DecodeArgs &la, const CUtensorMap &vmap, const CUtensorMap &wmap,
                          const CUtensorMap &qmap) {
    return la.wait_ns < kExactWaitNs ? launch_kernel_wide<NH, NG, true, kWindow, T>(la, vmap, wmap, qmap)
                                     : launch_kernel_wide<NH, NG, false, kWindow, T>(la, vmap, wmap, qmap);
}

}  // namespace

cudaError_t launch_window_wide(const DecodeArgs &a) {
    DecodeArgs la = a;
    Geometry &g = la.geo;
    const bool fp32 = a.out_dtype == KL_FP32, w32 = a.causal.hp * a.causal.rpb > 16, two_per_sm = a.causal.two_per_sm;
    g.qbox = a.causal.hp * a.causal.rpb;
    CUtensorMap vmap, wmap, qmap;
    if (!rows_maps(a, a.causal.hp, a.causal.rpb, &vmap, &wmap, &qmap)) return cudaErrorInvalidValue;
    if (fp32)
        return two_per_sm ? launch_window<16, 1, 3>(la, vmap, wmap, qmap)
                          : launch_window<16, 2, 3>(la, vmap, wmap, qmap);
    if (w32) return launch_window<32, 2, 2>(la, vmap, wmap, qmap);
    return two_per_sm ? launch_window<16, 1, 2>(la, vmap, wmap, qmap) : launch_window<16, 2, 2>(la, vmap, wmap, qmap);
}

}  // namespace kl
