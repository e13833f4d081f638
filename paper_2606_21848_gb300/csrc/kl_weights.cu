// Causal attention of a sequence's last rows that also adds up the weight that each cached row receives, for
// sm_103a; head_dim 128:
//
//   out as kl_window_attention without a window, and per sequence, value head and cached row
//   new_t = decay old_t + sum over the new rows r and the group's heads of softmax(s_r)_t
//
// The attention is the wide decode's kernel (kl_decode_wide_kernel.cuh, kWeights) in blocks of up to 16 (position,
// head) rows, with query and weights of three bf16 terms, since the weights are fp32 results whatever type the
// outputs have. A weight needs its row's whole softmax: the kernel writes the scores (4 bytes per row and token, 32
// per cached row of 256 where a group has 8 heads), and the last CTA of a value head reads them back, mostly from
// L2, with the runs' {maximum, sum}. Where a value head has several blocks of rows, a second kernel, the first's
// programmatic dependent, does that. Rows are added in their order: the sums are the same on every run.
// HBM bounds it (256 bytes per token and value head), then the tile's chain with three terms. Measured: 64 sequences of
// 8192 tokens, 64 / 8 heads 231 us (4.8 TB/s); 24 of 301 to 20011, 32 / 8 heads 129 us; one of 2000 11.5 us.
#include "kl_rows_wide.cuh"

namespace kl {
namespace {

constexpr int kAddThreads = 256;
constexpr int kAddRows = 256;                            // rows whose {maximum, 1 / sum} a CTA holds at a time
constexpr int kAddAhead = 8;                             // scores that a thread has on their way, times kAddPer

// CTA (tokens, g, b); kAddPer tokens per thread, kAddThreads apart.
template <int kAddPer>
__global__ void __launch_bounds__(kAddThreads) add_weights_kernel(const DecodeArgs a) {
    __shared__ float2 row[kAddRows];                     // {maximum, 1 / sum}
    constexpr int kAddTokens = kAddThreads * kAddPer;
    grid_dep_wait();
    grid_dep_launch();
    const Geometry &geo = a.geo;
    const auto &w = a.causal;
    const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const int q0 = a.tree.cu_q[b], q1 = a.tree.cu_q[b + 1], n = q1 - q0, L = a.seq_lens[b];
    if (q0 < 0 || n < 0 || q1 > a.tree.total_q || n > a.tree.max_q || L < n || L > a.causal.stride ||
        L > geo.max_pages * geo.P) {
        // (reported by the attention where there is one)
        if ((a.tree.total_q == 0 || a.tree.max_q == 0) && tid == 0 && blockIdx.x == 0 && g == 0)
            raise_flag(a.err, KL_FLAG_BAD_LENGTH);
        return;
    }
    const int t0 = blockIdx.x * kAddTokens + tid;
    if (blockIdx.x * kAddTokens >= L) return;
    const size_t unit = (size_t)b * geo.Hkv + g;
    const int hp = a.causal.hp, rpb = a.causal.rpb, nhg = a.causal.nhg;
    float old[kAddPer], sum[kAddPer];
#pragma unroll
    for (int k = 0; k < kAddPer; ++k) {
        const int t = t0 + k * kAddThreads;
        old[k] = w.decay != 0.f && t < L ? w.weights[unit * a.causal.stride + t] : 0.f;
        sum[k] = 0.f;
    }
    // rows in blocks as the attention's, kAddRows / 16 blocks at a time
    const int blocks = (n + rpb - 1) / rpb * nhg;
    constexpr int kBatch = kAddRows / 16;
    for (int k0 = 0; k0 < blocks; k0 += kBatch) {
        if (k0) __syncthreads();
        const int hb = k0 + tid / 16, r = tid & 15;      // (kAddThreads = kAddRows)
        if (hb < blocks) {
            const int m0 = hb / nhg * rpb, end = L - n + min(m0 + rpb, n);
            const int spc = (int)(unit * geo.nhb + hb) < a.causal.whole ? geo.S : geo.spc;
            const int runs = (end + geo.chunk * spc - 1) / (geo.chunk * spc);
            const int live = min(hp, geo.G - hb % nhg * hp) + (min(rpb, n - m0) - 1) * hp;
            if (r < live) {
                const float2 *s = a.causal.stats + ((unit * geo.nhb + hb) * 16 + r) * geo.S;
                float M = -INFINITY, z = 0.f;
                for (int i = 0; i < runs; ++i) {
                    const float2 x = __ldcg(s + i);
                    const float top = fmaxf(M, x.x);
                    // (a run of maximum -inf has sum 0, or NaN)
                    z = (M == top ? z : z * ptx::ex2(M - top)) + (x.x == top ? x.y : x.y * ptx::ex2(x.x - top));
                    M = top;
                }
                row[tid] = make_float2(M, 1.f / z);
            }
        }
        __syncthreads();
        for (int hb = k0; hb < min(blocks, k0 + kBatch); ++hb) {
            const int m0 = hb / nhg * rpb, live = min(hp, geo.G - hb % nhg * hp) + (min(rpb, n - m0) - 1) * hp;
            const float *s = a.causal.scores + (unit * geo.nhb + hb) * a.causal.rows * a.causal.pitch;
            const float2 *of = row + (hb - k0) * 16;
            const int p0 = L - n + m0;
            if ((int)(blockIdx.x + 1) * kAddTokens - 1 <= p0) {
                // all positions see all of these tokens
                s += t0;
                int r = 0;
                for (; r + kAddAhead <= live; r += kAddAhead) {
                    float x[kAddAhead][kAddPer];
#pragma unroll
                    for (int e = 0; e < kAddAhead; ++e)
#pragma unroll
                        for (int k = 0; k < kAddPer; ++k) x[e][k] = __ldcs(s + (r + e) * a.causal.pitch + k * kAddThreads);
#pragma unroll
                    for (int e = 0; e < kAddAhead; ++e) {
                        const float2 m = of[r + e];
#pragma unroll
                        for (int k = 0; k < kAddPer; ++k) sum[k] += ptx::ex2(x[e][k] - m.x) * m.y;
                    }
                }
                for (; r < live; ++r) {
                    const float2 m = of[r];
#pragma unroll
                    for (int k = 0; k < kAddPer; ++k)
                        sum[k] += ptx::ex2(__ldcs(s + r * a.causal.pitch + k * kAddThreads) - m.x) * m.y;
                }
            } else {
                // draft by draft; a position sees the tokens up to its own
                for (int r0 = 0, p = p0; r0 < live; r0 += hp, ++p)
#pragma unroll 4
                    for (int r = r0; r < min(r0 + hp, live); ++r) {
                        const float2 m = of[r];
#pragma unroll
                        for (int k = 0; k < kAddPer; ++k)
                            if (t0 + k * kAddThreads <= p)
                                sum[k] += ptx::ex2(__ldcs(s + r * a.causal.pitch + t0 + k * kAddThreads) - m.x) * m.y;
                    }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kAddPer; ++k) {
        const int t = t0 + k * kAddThreads;
        if (t < L) w.new_weights[unit * a.causal.stride + t] = w.decay != 0.f ? fmaf(w.decay, old[k], sum[k]) : sum[k];
    }
}

template <int NG>
cudaError_t launch_scores(const DecodeArgs &la, const CUtensorMap &vmap, const CUtensorMap &wmap,
                          const CUtensorMap &qmap) {
    return la.wait_ns < kExactWaitNs ? launch_kernel_wide<16, NG, true, kWeights, 3>(la, vmap, wmap, qmap)
                                     : launch_kernel_wide<16, NG, false, kWeights, 3>(la, vmap, wmap, qmap);
}

cudaError_t add_weights(const DecodeArgs &a) {
    const Geometry &g = a.geo;
    cudaLaunchConfig_t cfg = {};
    const int64_t longest = (int64_t)g.max_pages * g.P < a.causal.stride ? (int64_t)g.max_pages * g.P : a.causal.stride;
    // (one token per thread while that leaves places empty)
    const bool few = longest * g.Hkv * g.B <= 8 * kAddThreads * (int64_t)device_sm_count();
    const int tokens = kAddThreads * (few ? 1 : 4);
    cfg.gridDim = dim3((unsigned)((longest + tokens - 1) / tokens), g.Hkv, g.B);
    cfg.blockDim = dim3(kAddThreads);
    cfg.stream = a.stream;
    const OverlapAttr overlap(cfg);
    return cudaLaunchKernelEx(&cfg, few ? add_weights_kernel<1> : add_weights_kernel<4>, a);
}

}  // namespace

cudaError_t launch_attention_weights(const DecodeArgs &a) {
    DecodeArgs la = a;
    Geometry &g = la.geo;
    const bool two_per_sm = a.causal.two_per_sm;
    g.qbox = a.causal.hp * a.causal.rpb;
    CUtensorMap vmap, wmap, qmap;
    if (!rows_maps(a, a.causal.hp, a.causal.rpb, &vmap, &wmap, &qmap)) return cudaErrorInvalidValue;
    cudaError_t e = two_per_sm ? launch_scores<1>(la, vmap, wmap, qmap) : launch_scores<2>(la, vmap, wmap, qmap);
    return e != cudaSuccess || g.nhb == 1 ? e : add_weights(la);   // (one block per value head adds its weights itself)
}

cudaError_t launch_weights_fade(const DecodeArgs &a) { return add_weights(a); }

}  // namespace kl
