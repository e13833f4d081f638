// Attention of a tree of drafted tokens with few rows per value head (drafts x heads of a group <= 32) on the
// wide decode's kernel (kl_decode_wide_kernel.cuh, kTree): there a tile costs what its 16 or 32 rows cost,
// where a block of kl_tree_tc.cu costs 128 rows, and the splits merge inside.
// fp32 outputs take operands of three bf16 terms (24 bits) in the place of two.
// Measured, 32 / 8 heads: 4 drafts on 700 tokens 9.7 us (13.6 in kl_tree_tc.cu; latency), with fp32 outputs 10.0
// (22.7); 8 sequences of 4096 tokens, 8 drafts 24.5 us (34.5; HBM 10, the rest the start-up and the splits'
// merge), fp32 26.5 (59); 64 of 8192, 4 drafts 172 us (6250 GB/s), fp32 197 (520), 8 drafts 223 us (the tile
// chain of 32 rows); one of 131072, 8 drafts 60 us (HBM 40).
#include "kl_decode_wide_kernel.cuh"

namespace kl {

cudaError_t launch_tree_wide(const DecodeArgs &a) {
    DecodeArgs la = a;
    Geometry &g = la.geo;
    const int rows = g.G * a.tree.max_q;
    const int64_t sms = device_sm_count(), units = (int64_t)g.B * g.Hkv;
    const bool fp32 = a.out_dtype == KL_FP32;
    // More than 16 rows: one block of 32, or two of 16. Three terms leave no tensor memory for 32. With two terms a
    // tile takes a block of 32 0.87 us and one of 16 0.62, but the block of 32 starts 4 us later: two blocks
    // while every CTA has an SM and few tiles. (One sequence of 300 tokens, 8 drafts of 32 / 8 heads: 9.3 us in two
    // blocks, 13.0 in one; of 16384 18.9 and 24.4; of 131072 75.6 and 60.5; 8 of 4096 24.5 and 26.8; 16 of 4096
    // 65 and 35; 8 of 16384, 6 drafts, 71 and 58.)
    const int64_t tiles = ((int64_t)g.max_pages * g.P + 127) / 128;
    const bool blocks = rows > 16 && (fp32 || (2 * units <= sms && units * tiles <= 16 * sms));
    const bool w32 = rows > 16 && !blocks;
    // (two CTAs per SM as the decode's blocks of heads; three terms leave no room for that)
    const bool two_per_sm = rows <= 16 && !fp32 && units > sms;
    g.nhb = blocks ? 2 : 1;
    g.qbox = rows;
    g.spc = splits_per_cta(g.S, units * g.nhb, two_per_sm ? 2 * sms : sms);
    CUtensorMap vmap, wmap, qmap;
    if (!make_map(&vmap, a.v_cache, kD, (uint64_t)g.num_pages * g.Hkv * g.P, (uint32_t)g.P))
        return cudaErrorInvalidValue;
    wmap = qmap = vmap;
    if (a.w_r) {
        if (!make_map(&wmap, a.w_r, kD, (uint64_t)g.Hkv * kD, (uint32_t)kD)) return cudaErrorInvalidValue;
        // q as [total_q][Hq][128], one box = max_q consecutive drafts of a group's heads (64 dims); rows past
        // total_q read as zeros
        auto fn = encode_fn();
        const cuuint64_t dims[3] = {kD, (cuuint64_t)g.Hq, (cuuint64_t)a.tree.total_q};
        const cuuint64_t strides[2] = {kD * 2, (cuuint64_t)g.Hq * kD * 2};
        const cuuint32_t box[3] = {64, (cuuint32_t)g.G, (cuuint32_t)a.tree.max_q}, estr[3] = {1, 1, 1};
        if (!fn || fn(&qmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t *>(a.q), dims, strides, box,
                      estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    if (fp32) return launch_kernel_wide<16, 2, false, true, 3>(la, vmap, wmap, qmap);
    if (w32) return launch_kernel_wide<32, 2, false, true>(la, vmap, wmap, qmap);
    return two_per_sm ? launch_kernel_wide<16, 1, false, true>(la, vmap, wmap, qmap)
                      : launch_kernel_wide<16, 2, false, true>(la, vmap, wmap, qmap);
}

}  // namespace kl
