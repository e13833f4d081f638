// Causal attention that adds up the weight of each cached row (kl_weights.cu has the formulas), where a value head has
// more than 32 rows: blocks of 128 rows on the prefill's kernel (kl_prefill_tc_kernel.cuh, kWeights), which writes
// the scores, and a second kernel that adds the weights up.
//
// The scores lie as [block][tokens / 4][128 rows] float4: a warp of the attention writes 32 rows' four tokens as 512
// consecutive bytes, and here a warp reads them so: lane = row, and the lanes' sums of 32 tokens meet in one
// exchange of 31 shuffles. The order of all additions is fixed.
// Measured: 16 rows behind 4 prompts of 4001 to 6007 tokens, 32 / 8 heads 45 us, 37 of them the attention (as blocks of
// 16 rows on the wide decode's kernel 82).
#include "kl_prefill_tc_kernel.cuh"

namespace kl {
namespace {

constexpr int kSumWarps = 8, kSumTokens = 32 * kSumWarps;    // a warp adds up 32 tokens

// Lane l gets the sum over all lanes of x[l].
__device__ __forceinline__ float sum_lanes(float (&x)[32], int lane) {
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) {
        const bool upper = lane & w;
#pragma unroll
        for (int i = 0; i < w; ++i) {
            const float give = upper ? x[i] : x[i + w], keep = upper ? x[i + w] : x[i];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, w);
        }
    }
    return x[0];
}

// CTA (tokens, g, b). nm: blocks of positions; cs: CTAs that shared a block.
__global__ void __launch_bounds__(32 * kSumWarps) sum_weights_kernel(const PrefillArgs a, int hp, int rpb, int nm, int cs) {
    __shared__ float2 of[kBM];                               // rows' {maximum, 1 / sum}
    grid_dep_wait();
    grid_dep_launch();
    const Geometry &geo = a.geo;
    const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int q0 = a.cu_q[b], q1 = a.cu_q[b + 1], n = q1 - q0, L = a.seq_lens[b];
    if (q0 < 0 || n < 0 || q1 > a.total_q || n > a.max_q || L < n || L > a.stride || L > geo.max_pages * geo.P)
        return;                                              // (reported by the attention)
    if ((int)blockIdx.x * kSumTokens >= L) return;
    const int nhg = (geo.G + hp - 1) / hp, t0 = blockIdx.x * kSumTokens + 32 * warp;
    float sum[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) sum[i] = 0.f;
    const int blocks = nhg * ((n + rpb - 1) / rpb);
    for (int k = 0; k < blocks; ++k) {
        const int hg = k % nhg, m0 = k / nhg * rpb, hn = min(hp, geo.G - hg * hp), rows = min(rpb, n - m0);
        const size_t blk = ((size_t)(b * geo.Hkv + g) * nhg + hg) * nm + m0 / rpb;
        const int live = (rows - 1) * hp + hn, end = L - n + m0 + rows, stop = (end + 63) & ~63;
        const float4 *const s = a.scores + (blk * (a.pitch / 4) + t0 / 4) * kBM;
        // (scores behind a position's own token are -inf; behind the block's last half tile there are none)
        auto load = [&](int r, float4(&x)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                if (r < live && t0 + 4 * i < stop) x[i] = __ldcg(s + i * kBM + r);
            }
        };
        float4 x[8];
        load(lane, x);                                       // (on their way with the sums)
        if (k) __syncthreads();
        if (tid < live) {
            // every CTA's sum moves to the largest maximum
            const float2 *of_row = a.stats + (blk * kBM + tid) * 8;
            float2 y[8];
            float M = -INFINITY, z = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = make_float2(-INFINITY, 0.f);
                if (i < cs) y[i] = __ldcg(of_row + i);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) M = fmaxf(M, y[i].x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < cs) z += y[i].x == M ? y[i].y : y[i].y * ptx::ex2(y[i].x - M);
            // (heads past the group's have no scores: weight 0)
            of[tid] = tid % hp < hn ? make_float2(M, 1.f / z) : make_float2(INFINITY, 0.f);
        }
        __syncthreads();
        for (int r = lane; r < live; r += 32) {
            if (r != lane) load(r, x);
            const float2 m = of[r];
            if (m.x == INFINITY && m.y == 0.f) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[4 * i] += ptx::ex2(x[i].x - m.x) * m.y;
                sum[4 * i + 1] += ptx::ex2(x[i].y - m.x) * m.y;
                sum[4 * i + 2] += ptx::ex2(x[i].z - m.x) * m.y;
                sum[4 * i + 3] += ptx::ex2(x[i].w - m.x) * m.y;
            }
        }
    }
    __syncwarp();
    const float added = sum_lanes(sum, lane);
    const int t = t0 + lane;
    if (t < L) {
        const size_t at = ((size_t)b * geo.Hkv + g) * a.stride + t;
        a.new_weights[at] = a.decay != 0.f ? fmaf(a.decay, a.weights[at], added) : added;
    }
}

}  // namespace

cudaError_t launch_weights_tc(const PrefillArgs &a) {
    const Geometry &g = a.geo;
    const int64_t tokens = (int64_t)g.max_pages * g.P, longest = tokens < a.stride ? tokens : a.stride;
    int cs = 1;
    const cudaError_t e = a.out_dtype == KL_FP32 ? launch_rows<kModeWeights, 3, 3>(a, longest, &cs)
                                                 : launch_rows<kModeWeights, 3, 1>(a, longest, &cs);
    if (e != cudaSuccess) return e;
    const PrefillPlan p = plan_prefill(g.B, g.Hkv, g.G, a.max_q, longest, g.wr_per_qh != 0, device_sm_count());
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((longest + kSumTokens - 1) / kSumTokens), g.Hkv, g.B);
    cfg.blockDim = dim3(32 * kSumWarps);
    cfg.stream = a.stream;
    const OverlapAttr overlap(cfg);
    return cudaLaunchKernelEx(&cfg, sum_weights_kernel, a, p.hp, p.rpb, (a.max_q + p.rpb - 1) / p.rpb, cs);
}

}  // namespace kl
