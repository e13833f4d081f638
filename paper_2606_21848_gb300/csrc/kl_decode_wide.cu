// Tensor-core decode for groups of more than 8 query heads (kl_decode_wide_kernel.cuh): its layouts and launch.
#include "kl_decode_wide_kernel.cuh"

namespace kl {
namespace {

template <int NH, int NG>
cudaError_t launch_wide(const DecodeArgs &la, const CUtensorMap &vmap, const CUtensorMap &wmap,
                        const CUtensorMap &qmap) {
    return la.wait_ns < kExactWaitNs ? launch_kernel_wide<NH, NG, true, kHeads>(la, vmap, wmap, qmap)
                                     : launch_kernel_wide<NH, NG, false, kHeads>(la, vmap, wmap, qmap);
}

}  // namespace

cudaError_t launch_tc_wide(const DecodeArgs &a) {
    DecodeArgs la = a;
    Geometry &g = la.geo;
    const int64_t sms = device_sm_count();
    const auto per_cta = [&](int64_t units, int64_t slots) { return splits_per_cta(g.S, units, slots); };
    // Groups of 17 or more heads: CTAs of 32 heads (about 1200 cycles per tile where HBM does not set
    // the pace), unless CTAs of 16 (about 1000) have an SM each and not 6/5 as many splits to run.
    // (Group of 32, measured with CTAs of 16 and of 32: 104 sequences of 8192 tokens 67.7 and 51.4 us,
    // 77 68.1 and 49.8, 30 of 32768 in 4 splits 72.6 and 55.5, 20 of 40000 in 5 71.1 and 53.0, 150 of
    // 1000 in a group of 24 14.9 and 13.9; 52 sequences of 8192, one CTA of 16 on each of 104 SMs,
    // 39.1 and about 45.)
    const int64_t seq_heads = (int64_t)g.B * g.Hkv;
    const int64_t units32 = seq_heads * ((g.G + 31) / 32), units16 = seq_heads * ((g.G + 15) / 16);
    const bool w32 = g.G > 16 && (units16 > sms || 6 * per_cta(units32, sms) <=
                                                       5 * per_cta(units16, sms));
    const int NH = w32 ? 32 : 16;
    g.nhb = (g.G + NH - 1) / NH;
    g.qbox = g.G < NH ? g.G : NH;
    // Blocks of 16 heads that overflow one CTA per SM go two to an SM with one softmax group each:
    // their waves overlap, and the last one shares HBM evenly. (Within one wave, the
    // deeper ring and the two groups of a CTA that has its SM alone are faster.)
    const int64_t units = w32 ? units32 : units16;
    const bool two_per_sm = !w32 && units > sms;
    const int64_t slots = two_per_sm ? 2 * sms : sms;
    g.spc = per_cta(units, slots);
    CUtensorMap vmap, wmap, qmap;
    if (!make_map(&vmap, a.v_cache, kD, (uint64_t)g.num_pages * g.Hkv * g.P, (uint32_t)g.P))
        return cudaErrorInvalidValue;
    wmap = qmap = vmap;
    if (a.w_r) {
        const uint64_t hw = g.wr_per_qh ? (uint64_t)g.Hq : (uint64_t)g.Hkv;
        if (!make_map(&wmap, a.w_r, kD, hw * kD, (uint32_t)kD)) return cudaErrorInvalidValue;
        if (!make_map(&qmap, a.q, kD, (uint64_t)g.B * g.Hq, (uint32_t)g.qbox))
            return cudaErrorInvalidValue;
    }
    if (w32) return launch_wide<32, 2>(la, vmap, wmap, qmap);
    return two_per_sm ? launch_wide<16, 1>(la, vmap, wmap, qmap) : launch_wide<16, 2>(la, vmap, wmap, qmap);
}

}  // namespace kl
