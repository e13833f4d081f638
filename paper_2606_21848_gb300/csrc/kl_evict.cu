// Eviction from the paged Value-Only Cache by accumulated attention weight, for sm_103a: of every sequence and
// value head the first `sinks` rows, the last `recent` and of those between the ones with the largest weight (ties:
// the lowest index) stay, `budget` in all; they move together in their order, and their weights with them.
//
// Two kernels. The selection: a cluster of CTAs per (sequence, value head), each with a piece of the weights in
// shared memory. The smallest weight that stays is found by three rounds over its bits from the top, 11, 10 and 10
// (a positive fp32's order is that of its bits): every CTA counts its piece's weights that have the bits found so
// far by their next ones, all add the counts up through distributed shared memory and find the same bin. Few
// weights are left to count after the first round. Then each warp counts what stays of a stretch of the piece, the
// counts are summed before it, and it writes. (All weights are in shared memory before the first is written:
// weights may move in place.)
// The move: 512 bytes of traffic per row of 128 bf16 values, and HBM bounds it. Rows only ever move down: in place
// the CTAs of a cluster take turns of consecutive rows from the first on, read a turn ahead and meet between the
// reads and the writes of a turn; what they overwrite has been read by then. To other pages nothing waits.
#include "kl_internal.cuh"

namespace kl {
namespace {

constexpr int kBits0 = 11, kBits = 10;                   // of the first round, of the others
constexpr int kBins = 1 << kBits0;
constexpr int kPerThread = 4, kBinWarps = kBins / kPerThread / 32;   // the first warps find the bin
constexpr int kMostCluster = 8;

// What the move needs to know of a (sequence, value head): rows that stay (0: it is left alone) and whether its
// rows may move within their pages.
struct EvictUnit {
    int rows, in_place;
};
static_assert(sizeof(EvictUnit) == kEvictUnitBytes, "");

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
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

// Sums of the four words at `p` (16-byte aligned) over CTAs rank .. rank + 3 (those below `cluster`), all four loads
// on their way at once.
__device__ __forceinline__ void add_cluster(const int *p, int rank, int cluster, int (&n)[4]) {
    uint32_t at[4];
    int v[16];
#pragma unroll
    for (int c = 0; c < 4; ++c)
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                     : "=r"(at[c])
                     : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(min(rank + c, cluster - 1)));
    asm volatile(
        "ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%16];\n\t"
        "ld.shared::cluster.v4.b32 {%4, %5, %6, %7}, [%17];\n\t"
        "ld.shared::cluster.v4.b32 {%8, %9, %10, %11}, [%18];\n\t"
        "ld.shared::cluster.v4.b32 {%12, %13, %14, %15}, [%19];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(at[0]), "r"(at[1]), "r"(at[2]), "r"(at[3])
        : "memory");
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (rank + c < cluster)
#pragma unroll
            for (int e = 0; e < 4; ++e) n[e] += v[4 * c + e];
}

// Writes n to `p` (16-byte aligned) in the shared memory of CTA `rank`.
__device__ __forceinline__ void st_cluster(int *p, int rank, const int (&n)[4]) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(at)
                 : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(n[0]), "r"(n[1]), "r"(n[2]), "r"(n[3])
                 : "memory");
}

// Weights in their order as whole numbers; what is not positive, and NaN, is 0.
__device__ __forceinline__ uint32_t weight_key(float w) { return w > 0.f ? __float_as_uint(w) : 0u; }

// Cluster (b, g), CTA `rank` of it: tokens rank * piece ... kThreads: 512, of which an SM holds four CTAs, or 1024 where
// there are few units.
template <int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 4 : 1) select_kernel(const EvictArgs a, EvictUnit *units, int cluster, int piece) {
    constexpr int kSelWarps = kThreads / 32;
    extern __shared__ __align__(16) float held[];        // [piece]
    __shared__ __align__(16) int hist[kBins], sums[kBins];   // of this CTA, of the cluster
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
    const bool too_long = L < 0 || L > geo.max_pages * geo.P || L > a.stride;
    if (tid == 0) {
        border = 0;
        wanted = 0;
    }
    // The pages of the sequence and of where it goes, shared out over the cluster, while the weights are on their way
    const int32_t *from = a.block_table + (size_t)b * geo.max_pages, *to = a.new_table + (size_t)b * geo.max_pages;
    const float *w = a.weights + (size_t)unit * a.stride;
    const int t0 = too_long ? 0 : min(rank * piece, L), t1 = too_long ? 0 : min(t0 + piece, L);
    constexpr int kAhead = 8;
    float ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (t0 + tid + k * kThreads < t1) ahead[k] = w[t0 + tid + k * kThreads];
    int fault = too_long, eq = 0;
    if (!too_long) {
        const int pages = (L + geo.P - 1) / geo.P, new_pages = (rows + geo.P - 1) / geo.P;
#pragma unroll 2
        for (int i = rank * kThreads + tid; i < pages; i += cluster * kThreads) {
            const int p = from[i], q = i < new_pages ? to[i] : 0;
            if (p < 0 || p >= geo.num_pages || q < 0 || q >= geo.num_pages) fault = 1;
            if (i < new_pages && p == q) eq = 1;
        }
    }
    fault = __syncthreads_or(fault) ? (too_long ? KL_FLAG_BAD_LENGTH : KL_FLAG_BAD_PAGE) : 0;
    eq = __syncthreads_or(eq);
    if (cluster > 1) {
        if (tid == 0) {
            bad = fault;
            same = eq;
        }
        cluster_sync();
        fault = eq = 0;
#pragma unroll
        for (int c = 0; c < kMostCluster; ++c)
            if (c < cluster) {
                fault |= ld_cluster(&bad, c);
                eq |= ld_cluster(&same, c);
            }
    }
    if (tid == 0 && rank == 0) {
        if (fault && unit % geo.Hkv == 0) raise_flag(a.err, fault);
        units[unit] = EvictUnit{fault ? -1 : rows, eq};
    }
    if (fault) {                                         // (every CTA of the cluster, once all have read)
        if (cluster > 1) cluster_sync();
        return;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (t0 + tid + k * kThreads < t1) held[tid + k * kThreads] = ahead[k];
    for (int t = t0 + tid + kAhead * kThreads; t < t1; t += kAhead * kThreads) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (t + k * kThreads < t1) ahead[k] = w[t + k * kThreads];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (t + k * kThreads < t1) held[t - t0 + k * kThreads] = ahead[k];
    }
    // the tokens between the first and the last ones, of which `want` stay
    const bool all = L <= a.budget;
    const int mid0 = a.sinks, mid1 = L - a.recent;
    int want = all ? 0 : a.budget - a.sinks - a.recent;
    uint32_t key = 0;
    __shared__ int warp_sum[kBinWarps];
    int shift = 31;
    for (int round = 0; round < 3 && want > 0; ++round) {
        const int bits = round == 0 ? kBits0 : kBits;
        const uint32_t known = round == 0 ? 0u : ~0u << shift;   // bits found so far
        shift -= bits;
        int *const h = hist;
        for (int i = tid; i < kBins; i += kThreads) h[i] = 0;
        __syncthreads();
        // four consecutive weights per thread (those at the ends of the middle one by one)
        for (int at = 4 * tid; at < t1 - t0; at += 4 * kThreads) {
            const float4 x = *reinterpret_cast<const float4 *>(held + at);
            uint32_t k[4] = {weight_key(x.x), weight_key(x.y), weight_key(x.z), weight_key(x.w)};
            const int from_mid = t0 + at - mid0;
            const uint32_t mids = (uint32_t)(min(t1, mid1) - mid0);
            bool in[4], any = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                in[e] = ((k[e] ^ key) & known) == 0 && (uint32_t)(from_mid + e) < mids;
                any |= in[e];
            }
            if (any)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (in[e]) atomicAdd(h + ((k[e] >> shift) & ((1u << bits) - 1)), 1);
        }
        if (cluster > 1) {
            // each CTA adds up a share of the bins and gives it to all
            cluster_sync();
            const int share = kBins / cluster;
            if (4 * tid < share) {
                int *const mine = h + rank * share + 4 * tid;
                int n[4] = {0, 0, 0, 0};
                for (int c = 0; c < cluster; c += 4) add_cluster(mine, c, cluster, n);
                for (int c = 0; c < cluster; ++c) st_cluster(sums + (mine - h), c, n);
            }
            cluster_sync();
        } else {
            __syncthreads();
        }
        // the bin of the want-th largest: bins from the top, kPerThread per thread
        const int low = kBins - kPerThread * (tid + 1);          // its lowest bin
        int n[kPerThread] = {0, 0, 0, 0}, sum = 0, upto = 0;
        if (warp < kBinWarps) {
            const int4 x = *reinterpret_cast<const int4 *>((cluster > 1 ? sums : h) + low);
            n[0] = x.x;
            n[1] = x.y;
            n[2] = x.z;
            n[3] = x.w;
            sum = upto = n[0] + n[1] + n[2] + n[3];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            if (lane == 31) warp_sum[warp] = upto;
        }
        __syncthreads();
        if (warp < kBinWarps) {
            upto += __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane] : 0);
            int above = upto - sum;
            if (above < want && want <= upto) {
#pragma unroll
                for (int e = kPerThread - 1; e >= 0; --e) {
                    if (above < want && want <= above + n[e]) {
                        border = key | (uint32_t)(low + e) << shift;
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
    // Four consecutive tokens per lane and step: how many are above, and (<< 16) on the border; of which bits they are.
    auto look = [&](int t, uint32_t &bits) -> uint32_t {
        bits = 0;
        if (t >= t1) return 0;
        const float4 x = *reinterpret_cast<const float4 *>(held + (t - t0));
        const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (t + e >= t1) continue;
            const bool inner = !all && t + e >= mid0 && t + e < mid1;
            const uint32_t k = weight_key(xs[e]);
            if (!inner || (!none && k > key)) bits |= 1u << e;
            else if (!none && k == key) bits |= 16u << e;
        }
        return __popc(bits & 15u) | __popc(bits >> 4) << 16;
    };
    const int per = ((t1 - t0 + kSelWarps - 1) / kSelWarps + 127) & ~127;
    const int s0 = min(t0 + warp * per, t1), s1 = min(s0 + per, t1);
    if (want == 0 || all || none) __syncthreads();       // (held is complete)
    int na = 0, no = 0;
    for (int t = s0; t < s1; t += 128) {
        uint32_t bits;
        const uint32_t n = __reduce_add_sync(0xffffffffu, look(t + 4 * lane, bits));
        na += n & 0xffffu;
        no += n >> 16;
    }
    if (lane == 0) {
        warp_above[warp] = na;
        warp_on[warp] = no;
    }
    __syncthreads();
    if (warp == 0) {
        const int x = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? warp_above[lane] : 0);
        const int y = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? warp_on[lane] : 0);
        if (lane == 0) {
            count[0] = x;
            count[1] = y;
        }
    }
    if (cluster > 1) cluster_sync();                     // (and every CTA holds its weights)
    else __syncthreads();
    // above the border and on it before this warp's stretch
    int before = lane < warp ? warp_above[lane] : 0, on_before = lane < warp ? warp_on[lane] : 0;
    if (lane < rank) {
        before += ld_cluster(count, lane);
        on_before += ld_cluster(count + 1, lane);
    }
    before = __reduce_add_sync(0xffffffffu, before);
    on_before = __reduce_add_sync(0xffffffffu, on_before);
    grid_dep_launch();
    int32_t *kept = a.kept + (size_t)unit * a.budget;
    float *nw = a.new_weights + (size_t)unit * a.stride;
    for (int t = s0; t < s1; t += 128) {
        uint32_t bits, upto = look(t + 4 * lane, bits);
        const uint32_t mine = upto;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        int ox = before + (int)((upto - mine) & 0xffffu), oy = on_before + (int)((upto - mine) >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool x = bits >> e & 1, y = bits >> (4 + e) & 1;
            if (x || (y && oy < want)) {
                const int at = ox + min(oy, want);
                kept[at] = t + 4 * lane + e;
                nw[at] = held[t + 4 * lane + e - t0];
            }
            ox += x;
            oy += y;
        }
        const uint32_t total = __shfl_sync(0xffffffffu, upto, 31);
        before += total & 0xffffu;
        on_before += total >> 16;
    }
    // (the whole cluster writes the rest; nothing there is read again)
    for (int t = rows + rank * kThreads + tid; t < L; t += cluster * kThreads) nw[t] = 0.f;
    for (int t = rows + rank * kThreads + tid; t < a.budget; t += cluster * kThreads) kept[t] = -1;
    if (cluster > 1) cluster_sync();                     // (the counts are read)
}

constexpr int kMoveThreads = 128, kMoveCtas = 8;         // per SM
constexpr int64_t kEarlyBytes = 256 << 20;               // of rows: up to here the move starts early
constexpr int kMoveDepth = 4;                            // 16-byte pieces per thread and turn

// t / P and t % P: P a power of two (its shift), or any (shift -1).
struct Paging {
    int P, shift;
    __device__ __forceinline__ int page(int t) const { return shift >= 0 ? t >> shift : t / P; }
    __device__ __forceinline__ int row(int t) const { return shift >= 0 ? t & (P - 1) : t % P; }
};

// CTA ((unit * slices + slice) * groups + group) * cluster + rank: a stretch of 2^cshift 16-byte pieces of every row.
// In turn s of its group (groups * cluster of them share the rows that move to other pages) CTA `rank` takes
// `step` rows. Three turns ahead of the write it reads which rows, two ahead their pages, one ahead the rows.
__global__ void __launch_bounds__(kMoveThreads, kMoveCtas) move_kernel(const EvictArgs a, const EvictUnit *units, int slices,
                                                            int cshift, int groups, int cluster, const Paging pg) {
    grid_dep_wait();
    grid_dep_launch();
    const Geometry &geo = a.geo;
    const int rank = blockIdx.x % cluster, group = blockIdx.x / cluster % groups;
    const int slice = blockIdx.x / cluster / groups % slices, unit = blockIdx.x / cluster / groups / slices;
    const int tid = threadIdx.x;
    const int b = unit / geo.Hkv, g = unit % geo.Hkv;
    const EvictUnit u = units[unit];
    // (the whole cluster leaves)
    if (u.rows < 0) return;
    if (g == 0 && slice == 0 && group == 0 && rank == 0 && tid == 0) a.new_lens[b] = u.rows;
    if (u.in_place && group > 0) return;
    constexpr int kStep = kMoveThreads * kMoveDepth;
    const int step = kStep >> cshift;                    // rows of a CTA per turn
    const int turn = step * cluster * (u.in_place ? 1 : groups);
    const int32_t *from = a.block_table + (size_t)b * geo.max_pages, *to = a.new_table + (size_t)b * geo.max_pages;
    const int32_t *kept = a.kept + (size_t)unit * a.budget;
    const int cpr = geo.D / 8, c = (slice << cshift) + (tid & ((1 << cshift) - 1));
    const int rstep = kMoveThreads >> cshift;
    uint4 *const v = reinterpret_cast<uint4 *>(a.v_cache);
    auto piece = [&](int page, int t) -> uint4 * {
        return v + (((int64_t)page * geo.Hkv + g) * geo.P + pg.row(t)) * cpr + c;
    };
    const int first = (u.in_place ? rank : group * cluster + rank) * step + (tid >> cshift);
    // of this thread's kMoveDepth rows: which (of turn s + 2 at the loop's head), their pages and rows (s + 1)
    uint4 x[kMoveDepth], y[kMoveDepth];
    int id[kMoveDepth], page[kMoveDepth], next[kMoveDepth];
    auto each = [&](int j, auto &&f) {
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k)
            if (j + k * rstep < u.rows) f(k, j + k * rstep);
    };
    each(first, [&](int k, int at) { id[k] = kept[at]; });
    each(first + turn, [&](int k, int at) { next[k] = kept[at]; });
    each(first, [&](int k, int) { page[k] = from[pg.page(id[k])]; });
    each(first, [&](int k, int) { x[k] = *piece(page[k], id[k]); });
    each(first + turn, [&](int k, int) { page[k] = from[pg.page(next[k])]; id[k] = next[k]; });
    each(first + 2 * turn, [&](int k, int at) { next[k] = kept[at]; });
    const int turns = (u.rows + turn - 1) / turn;        // (as many in all CTAs: they meet)
    for (int s = 0, j = first; s < turns; ++s, j += turn) {
        each(j + turn, [&](int k, int) { y[k] = *piece(page[k], id[k]); });
        each(j + 2 * turn, [&](int k, int) { page[k] = from[pg.page(next[k])]; id[k] = next[k]; });
        each(j + 3 * turn, [&](int k, int at) { next[k] = kept[at]; });
        if (u.in_place) {                                // the rows of this turn and the next one have been read
            if (cluster > 1) cluster_sync();
            else __syncthreads();
        }
        each(j, [&](int k, int at) { *piece(to[pg.page(at)], at) = x[k]; });
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k) x[k] = y[k];
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
    const int piece = (int)((longest + cluster - 1) / cluster + 127) & ~127;
    EvictUnit *info = static_cast<EvictUnit *>(a.workspace);
    const bool few = units * cluster <= sms;
    const auto kernel = few ? select_kernel<1024> : select_kernel<512>;
    static PerDeviceOnce once[2];
    const cudaError_t e = once[few].run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    KL_EVICT_MAX_TOKENS / kMostCluster * (int)sizeof(float));
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * cluster));
    cfg.blockDim = dim3(few ? 1024 : 512);
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
    cudaError_t s = cudaLaunchKernelEx(&cfg, kernel, a, info, cluster, piece);
    if (s != cudaSuccess) return s;
    // As many CTAs as the GPU holds at a time, eight per SM: clusters of them while there are few units, then 64-byte
    // stretches instead of whole rows, then (to other pages) groups of clusters.
    const int cpr = g.D / 8;
    const int64_t wanted = kMoveCtas * sms;
    int team = 1, cshift = g.D == 128 ? 4 : 3;
    while (cshift > 3 && 2 * (int64_t)units * (cpr >> cshift) <= wanted) --cshift;
    while (team < kMostCluster && 2 * (int64_t)units * team * (cpr >> cshift) <= wanted && (kMoveThreads * kMoveDepth >> cshift) * team < a.budget) team *= 2;
    while (cshift > 2 && 2 * (int64_t)units * team * (cpr >> cshift) <= wanted) --cshift;
    const int slices = cpr >> cshift, step = kMoveThreads * kMoveDepth >> cshift;
    int64_t groups = wanted / ((int64_t)units * slices * team);
    const int64_t most = (a.budget + (int64_t)step * team - 1) / ((int64_t)step * team);
    groups = groups < 1 ? 1 : groups > most ? most : groups;
    int shift = 0;
    while (1 << shift < g.P) ++shift;
    const Paging pg{g.P, 1 << shift == g.P ? shift : -1};
    cudaLaunchConfig_t mv = {};
    mv.gridDim = dim3((unsigned)(groups * units * slices * team));
    mv.blockDim = dim3(kMoveThreads);
    mv.stream = a.stream;
    attr[1].val.clusterDim.x = team;
    // An early start saves a launch's latency, but the CTAs then crowd the SMs that the selection leaves first (64 x
    // 8192 rows to 4096, 8 heads, 1 GB of traffic: 242 us with it)
    if ((int64_t)units * (a.budget < longest ? a.budget : longest) * g.D * 4 > kEarlyBytes)
        attr[0].val.programmaticStreamSerializationAllowed = 0;
    mv.attrs = attr;
    mv.numAttrs = 2;
    return cudaLaunchKernelEx(&mv, move_kernel, a, (const EvictUnit *)info, slices, cshift, (int)groups, team, pg);
}

}  // namespace kl
