// Tensor-core chunked prefill (kl_prefill_tc_kernel.cuh), and the chunk append.
#include "kl_prefill_tc_kernel.cuh"

namespace kl {
namespace {

// Chunk append: row i of sequence b's chunk goes to position seq_lens[b] - n_b + i. One CTA per
// (16 chunk rows, sequence); 16-byte copies.
constexpr int kAppendRows = 16;

__global__ void __launch_bounds__(128) append_chunk_kernel(int Hkv, int D, int P, int num_pages,
                                                           int max_pages, int total_q,
                                                           const uint4 *v_new,
                                                           const int32_t *block_table,
                                                           const int32_t *seq_lens,
                                                           const int32_t *cu_q,
                                                           uint4 *v_cache, int32_t *err) {
    grid_dep_wait();
    grid_dep_launch();
    const int b = blockIdx.y;
    const int q0 = cu_q[b], n = cu_q[b + 1] - q0, L = seq_lens[b];
    if (q0 < 0 || n < 0 || q0 + n > total_q || L < n || L > max_pages * P) {
        if (threadIdx.x == 0 && blockIdx.x == 0) raise_flag(err, KL_FLAG_BAD_LENGTH);
        return;
    }
    const int i0 = blockIdx.x * kAppendRows;
    const int cpr = D / 8;   // 16-byte chunks per row
    const int per_row = Hkv * cpr;
    for (int k = threadIdx.x; k < kAppendRows * per_row; k += blockDim.x) {
        const int i = i0 + k / per_row;
        if (i >= n) break;
        const int gc = k % per_row, g = gc / cpr, c = gc % cpr;
        const int pos = L - n + i;
        const int page = block_table[(size_t)b * max_pages + pos / P];
        if (page < 0 || page >= num_pages) {
            raise_flag(err, KL_FLAG_BAD_PAGE);
            continue;
        }
        v_cache[(((size_t)page * Hkv + g) * P + pos % P) * cpr + c] =
            v_new[((size_t)(q0 + i) * Hkv + g) * cpr + c];
    }
}

}  // namespace

bool prefill_tc_supported(const Geometry &g) {
    if (g.D != kD) return false;
    if (g.P != 16 && g.P != 32 && g.P != 64 && g.P != 128) return false;
    if ((int64_t)g.num_pages * g.Hkv * g.P >= ((int64_t)1 << 31)) return false;
    int dev = 0, major = 0, minor = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
    return major == 10 && minor == 3;
}

cudaError_t launch_prefill_tc(const PrefillArgs &a) {
    return launch_rows<kModePrefill, 2, 1>(a, (int64_t)a.geo.max_pages * a.geo.P);
}

cudaError_t launch_append_chunk(const Geometry &g, int total_q, int max_q, const uint16_t *v_new,
                                const int32_t *block_table, const int32_t *seq_lens,
                                const int32_t *cu_q, uint16_t *v_cache, int32_t *err,
                                cudaStream_t stream) {
    if (g.B == 0 || total_q == 0 || max_q == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((max_q + kAppendRows - 1) / kAppendRows, g.B);
    cfg.blockDim = dim3(128);
    cfg.stream = stream;
    const OverlapAttr overlap(cfg);
    return cudaLaunchKernelEx(&cfg, append_chunk_kernel, g.Hkv, g.D, g.P, g.num_pages, g.max_pages,
                              total_q, reinterpret_cast<const uint4 *>(v_new), block_table, seq_lens,
                              cu_q, reinterpret_cast<uint4 *>(v_cache), err);
}

}  // namespace kl
