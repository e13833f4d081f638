// Eviction from the paged Value-Only Cache by accumulated attention weight, for sm_103a: of every sequence and
// value head the first `sinks` rows, the last `recent` and of those between the ones with the largest weight (ties:
// the lowest index) stay, `budget` in all; they move together in their order, and their weights with them.
//
// Two kernels. The selection: a cluster of CTAs per (sequence, value head), each with a piece of the weights in
// shared memory. The smallest weight that stays is found by four rounds over its bits, 8 at a time from the top: every
// CTA counts its piece's weights under the bits found so far, all add the counts up through distributed shared memory
// and find the same byte. Then each warp counts what stays of a stretch of the piece, the counts are summed before
// it, and it writes. (All weights are in shared memory before the first is written: weights may move in place.)
// The move: 512 bytes of traffic per row of 128 bf16 values. Rows only ever move down, row j to a place at most
// where it was, so in place a CTA takes (sequence, value head, a stretch of each row) from the first row on and reads
// a step ahead of what it writes: what it overwrites has been read. To other pages the rows are shared out.
#include "kl_internal.cuh"

namespace kl {
namespace {

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr int kBins = 256;
constexpr int kMostCluster = 8;

// What the move needs to know of a (sequence, value head): rows that stay (0: it is left alone) and whether its
// rows may move within their pages.
struct EvictUnit {
    int rows, in_place;
};
static_assert(sizeof(EvictUnit) == kEvictUnitBytes, "");

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The word at `p` of this CTA's shared memory in that of CTA `rank` of the cluster.
__device__ __forceinline__ int ld_cluster(const int *p, int rank) {
    uint32_t at;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(at)
                 : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// Weights in their order as whole numbers; what is not positive, and NaN, is 0.
__device__ __forceinline__ uint32_t weight_key(float w) { return w > 0.f ? __float_as_uint(w) : 0u; }

// Cluster (b, g), CTA `rank` of it: tokens rank * piece ...
__global__ void __launch_bounds__(kSelThreads) select_kernel(const EvictArgs a, EvictUnit *units, int cluster, int piece) {
    extern __shared__ float held[];                      // [piece]
    __shared__ int hist[2][kBins];
    __shared__ int count[2];                             // of this CTA's piece: above the border, on it
    __shared__ int warp_above[kSelWarps], warp_on[kSelWarps];
    __shared__ uint32_t border;
    __shared__ int wanted, bad, same;
    const Geometry &geo = a.geo;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0, unit = blockIdx.x / cluster;
    const int b = unit / geo.Hkv;
    grid_dep_wait();
    const int L = a.seq_lens[b], rows = min(L, a.budget);
    if (tid == 0) {
        bad = L < 0 || L > geo.max_pages * geo.P || L > a.stride ? KL_FLAG_BAD_LENGTH : 0;
        same = 0;
        border = 0;
        wanted = 0;
    }
    __syncthreads();
    grid_dep_launch();
    // every page of the sequence and of where it goes (the same answer in all CTAs of the sequence)
    const int32_t *from = a.block_table + (size_t)b * geo.max_pages, *to = a.new_table + (size_t)b * geo.max_pages;
    if (!bad) {
        const int pages = (L + geo.P - 1) / geo.P, new_pages = (rows + geo.P - 1) / geo.P;
        bool wrong = false, eq = false;
        for (int i = tid; i < pages; i += kSelThreads) {
            const int p = from[i];
            wrong |= p < 0 || p >= geo.num_pages;
            if (i < new_pages) {
                const int q = to[i];
                wrong |= q < 0 || q >= geo.num_pages;
                eq |= p == q;
            }
        }
        if (wrong) bad = KL_FLAG_BAD_PAGE;               // (any of them)
        if (eq) same = 1;
    }
    __syncthreads();
    const bool left = bad != 0;
    if (tid == 0 && rank == 0) {
        if (left && unit % geo.Hkv == 0) raise_flag(a.err, bad);
        units[unit] = EvictUnit{left ? -1 : rows, same};
    }
    if (left) return;                                    // (every CTA of the cluster)
    const float *w = a.weights + (size_t)unit * a.stride;
    const int t0 = min(rank * piece, L), t1 = min(t0 + piece, L);
    for (int t = t0 + tid; t < t1; t += kSelThreads) held[t - t0] = w[t];
    // the tokens between the first and the last ones, of which `want` stay
    const bool all = L <= a.budget;
    const int mid0 = a.sinks, mid1 = L - a.recent;
    int want = all ? 0 : a.budget - a.sinks - a.recent;
    uint32_t key = 0;
    for (int round = 0; round < 4 && want > 0; ++round) {
        const int shift = 24 - 8 * round;
        int *const h = hist[round & 1];
        if (tid < kBins) h[tid] = 0;
        __syncthreads();
        for (int base = t0; base < t1; base += kSelThreads) {
            const int t = base + tid;
            const uint32_t k = t < t1 ? weight_key(held[t - t0]) : 0;
            const bool in = t < t1 && t >= mid0 && t < mid1 && (round == 0 || (k >> (shift + 8)) == (key >> (shift + 8)));
            // (one addition per distinct byte of a warp: weights share their upper bits)
            const uint32_t bin = in ? (k >> shift) & 255u : kBins;
            const uint32_t mates = __match_any_sync(0xffffffffu, bin);
            if (in && lane == __ffs(mates) - 1) atomicAdd(h + bin, __popc(mates));
        }
        if (cluster > 1) cluster_sync();
        else __syncthreads();
        // the byte of the want-th largest: bins from the top, 8 per lane of one warp
        if (warp == 0) {
            int n[8], sum = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int bin = 255 - 8 * lane - e;
                n[e] = 0;
                if (cluster > 1)
                    for (int c = 0; c < cluster; ++c) n[e] += ld_cluster(h + bin, c);
                else n[e] = h[bin];
                sum += n[e];
            }
            int upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            int above = upto - sum;
            if (above < want && want <= upto) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (above < want && want <= above + n[e]) {
                        border = key | (uint32_t)(255 - 8 * lane - e) << shift;
                        wanted = want - above;
                    }
                    above += n[e];
                }
            }
        }
        __syncthreads();
        key = border;
        want = wanted;
    }
    // `want` of those on the border `key` stay, the first ones; with none wanted nothing between stays
    const bool none = !all && a.budget == a.sinks + a.recent;
    auto above = [&](int t) { return all || t < mid0 || t >= mid1 || (!none && weight_key(held[t - t0]) > key); };
    auto on = [&](int t) { return !all && !none && t >= mid0 && t < mid1 && weight_key(held[t - t0]) == key; };
    const int per = ((t1 - t0 + kSelWarps - 1) / kSelWarps + 31) & ~31;
    const int s0 = min(t0 + warp * per, t1), s1 = min(s0 + per, t1);
    if (want == 0 || all || none) __syncthreads();       // (held is complete)
    int na = 0, no = 0;
    for (int t = s0; t < s1; t += 32) {
        na += __popc(__ballot_sync(0xffffffffu, t + lane < s1 && above(t + lane)));
        no += __popc(__ballot_sync(0xffffffffu, t + lane < s1 && on(t + lane)));
    }
    if (lane == 0) {
        warp_above[warp] = na;
        warp_on[warp] = no;
    }
    __syncthreads();
    if (tid == 0) {
        int x = 0, y = 0;
        for (int i = 0; i < kSelWarps; ++i) {
            x += warp_above[i];
            y += warp_on[i];
        }
        count[0] = x;
        count[1] = y;
    }
    if (cluster > 1) cluster_sync();                     // (and every CTA holds its weights)
    else __syncthreads();
    int before = 0, on_before = 0;                       // this warp's stretch: above the border and on it before
    for (int c = 0; c < rank; ++c) {
        before += ld_cluster(count, c);
        on_before += ld_cluster(count + 1, c);
    }
    for (int i = 0; i < warp; ++i) {
        before += warp_above[i];
        on_before += warp_on[i];
    }
    int32_t *kept = a.kept + (size_t)unit * a.budget;
    float *nw = a.new_weights + (size_t)unit * a.stride;
    for (int t = s0; t < s1; t += 32) {
        const bool live = t + lane < s1, x = live && above(t + lane), y = live && on(t + lane);
        const uint32_t mx = __ballot_sync(0xffffffffu, x), my = __ballot_sync(0xffffffffu, y);
        const uint32_t under = (1u << lane) - 1;
        const int ox = before + __popc(mx & under), oy = on_before + __popc(my & under);
        if (x || (y && oy < want)) {
            const int at = ox + min(oy, want);
            kept[at] = t + lane;
            nw[at] = held[t + lane - t0];
        }
        before += __popc(mx);
        on_before += __popc(my);
    }
    // (the whole cluster writes the rest; nothing there is read again)
    for (int t = rows + rank * kSelThreads + tid; t < L; t += cluster * kSelThreads) nw[t] = 0.f;
    for (int t = rows + rank * kSelThreads + tid; t < a.budget; t += cluster * kSelThreads) kept[t] = -1;
    if (cluster > 1) cluster_sync();                     // (the counts are read)
}

constexpr int kMoveThreads = 256;
constexpr int kMoveDepth = 4;                            // 16-byte pieces per thread and step

// CTA (unit * slices + slice) * parts + part: a stretch of 2^cshift 16-byte pieces of every row.
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const EvictArgs a, const EvictUnit *units, int slices,
                                                            int cshift, int parts) {
    grid_dep_wait();
    grid_dep_launch();
    const Geometry &geo = a.geo;
    const int part = blockIdx.x % parts, slice = blockIdx.x / parts % slices, unit = blockIdx.x / parts / slices;
    const int tid = threadIdx.x;
    const int b = unit / geo.Hkv, g = unit % geo.Hkv, P = geo.P;
    const EvictUnit u = units[unit];
    if (u.rows < 0) return;
    if (g == 0 && slice == 0 && part == 0 && tid == 0) a.new_lens[b] = u.rows;
    int j0 = 0, j1 = u.rows;
    constexpr int kStep = kMoveThreads * kMoveDepth;
    const int step = kStep >> cshift;                    // rows per step
    if (u.in_place) {
        if (part > 0) return;
    } else {
        const int per = ((u.rows + parts - 1) / parts + step - 1) / step * step;
        j0 = min(part * per, u.rows);
        j1 = min(j0 + per, u.rows);
    }
    const int32_t *from = a.block_table + (size_t)b * geo.max_pages, *to = a.new_table + (size_t)b * geo.max_pages;
    const int32_t *kept = a.kept + (size_t)unit * a.budget;
    const int cpr = geo.D / 8, c = (slice << cshift) + (tid & ((1 << cshift) - 1)), r = tid >> cshift;
    const int rstep = kMoveThreads >> cshift;
    uint4 *const v = reinterpret_cast<uint4 *>(a.v_cache);
    auto piece = [&](const int32_t *table, int t) -> uint4 * {
        return v + (((int64_t)table[t / P] * geo.Hkv + g) * P + t % P) * cpr + c;
    };
    uint4 x[kMoveDepth], y[kMoveDepth];
    auto load = [&](int j, uint4 (&d)[kMoveDepth]) {
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k) {
            const int at = j + r + k * rstep;
            if (at < j1) d[k] = *piece(from, kept[at]);
        }
    };
    load(j0, x);
    for (int j = j0; j < j1; j += step) {
        load(j + step, y);
        if (u.in_place) __syncthreads();                 // this step's and the next one's rows have been read
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k) {
            const int at = j + r + k * rstep;
            if (at < j1) *piece(to, at) = x[k];
            x[k] = y[k];
        }
    }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs &a) {
    const Geometry &g = a.geo;
    const int units = g.B * g.Hkv, sms = device_sm_count();
    const int64_t longest = (int64_t)g.max_pages * g.P < a.stride ? (int64_t)g.max_pages * g.P : a.stride;
    // as many CTAs per unit as the GPU has room for, with pieces of 2048 weights and more
    int cluster = 1;
    while (cluster < kMostCluster &&
           ((longest > (int64_t)cluster * KL_EVICT_MAX_TOKENS / kMostCluster) ||
            (2 * (int64_t)units * cluster <= sms && longest >= 4096 * (int64_t)cluster)))
        cluster *= 2;
    const int piece = (int)((longest + cluster - 1) / cluster + 31) & ~31;
    EvictUnit *info = static_cast<EvictUnit *>(a.workspace);
    static PerDeviceOnce once;
    const cudaError_t e = once.run([&] {
        return cudaFuncSetAttribute(select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    KL_EVICT_MAX_TOKENS / kMostCluster * (int)sizeof(float));
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * cluster));
    cfg.blockDim = dim3(kSelThreads);
    cfg.dynamicSmemBytes = piece * sizeof(float);
    cfg.stream = a.stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t s = cudaLaunchKernelEx(&cfg, select_kernel, a, info, cluster, piece);
    if (s != cudaSuccess) return s;
    // 64-byte stretches where there are few units, whole rows where they fill the GPU
    const int cpr = g.D / 8;
    int cshift = 2;
    while ((1 << cshift) < cpr && (int64_t)units * (cpr >> (cshift + 1)) >= 2 * sms) ++cshift;
    const int slices = cpr >> cshift, step = kMoveThreads * kMoveDepth >> cshift;
    int64_t parts = (4 * (int64_t)sms + units * slices - 1) / ((int64_t)units * slices);
    const int64_t most = (a.budget + step - 1) / step;
    parts = parts > most ? most : parts;
    cudaLaunchConfig_t mv = {};
    parts = parts < 1 ? 1 : parts;
    mv.gridDim = dim3((unsigned)(parts * units * slices));
    mv.blockDim = dim3(kMoveThreads);
    mv.stream = a.stream;
    const OverlapAttr overlap(mv);
    return cudaLaunchKernelEx(&mv, move_kernel, a, (const EvictUnit *)info, slices, cshift, (int)parts);
}

}  // namespace kl
