// Launching of the wide decode's kernel on the rows of drafts or consecutive positions.
#pragma once

#include "kl_decode_wide_kernel.cuh"

namespace kl {
namespace {

// merge_states puts 12 bytes per row and state and a state's rows into the ring.
template <int NH, int NG, int T>
constexpr bool merge_fits = ((12u * NH * kCausalMostRuns + 1023) & ~1023u) + NH * kD * sizeof(float) <=
                            sizeof(WideSmem<NH, NG, T>::tiles);
static_assert(kCausalMostRuns == kWideMaxRuns && merge_fits<16, 1, 2> && merge_fits<16, 1, 3> && merge_fits<16, 2, 2> &&
                  merge_fits<16, 2, 3> && merge_fits<32, 2, 2>, "");

// The maps of the cache, of W^R and of the queries ([total_q][Hq][128], one box = `rows` consecutive rows of
// `heads` heads, 64 dims; rows past total_q and heads past Hq read as zeros).
inline bool rows_maps(const DecodeArgs &a, int heads, int rows, CUtensorMap *vmap, CUtensorMap *wmap,
                      CUtensorMap *qmap) {
    const Geometry &g = a.geo;
    if (!make_map(vmap, a.v_cache, kD, (uint64_t)g.num_pages * g.Hkv * g.P, (uint32_t)g.P)) return false;
    *wmap = *qmap = *vmap;
    if (!a.w_r) return true;
    const uint64_t hw = g.wr_per_qh ? g.Hq : g.Hkv;
    if (!make_map(wmap, a.w_r, kD, hw * kD, (uint32_t)kD)) return false;
    auto fn = encode_fn();
    const cuuint64_t dims[3] = {kD, (cuuint64_t)g.Hq, (cuuint64_t)a.tree.total_q};
    const cuuint64_t strides[2] = {kD * 2, (cuuint64_t)g.Hq * kD * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)rows}, estr[3] = {1, 1, 1};
    return fn && fn(qmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint16_t *>(a.q), dims, strides, box, estr,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace kl
