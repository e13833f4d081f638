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
// The move: 512 bytes of traffic per row of 128 bf16 values, and HBM bounds it. Rows only ever move down, so in place
// what a chunk of consecutive rows overwrites has been read once all chunks before it have been read.
// - Many (sequence, value head)s: one CTA per stretch of 128 bytes of their rows goes through the chunks and reads a
//   chunk ahead of what it writes (64 x 8192 rows to 4096, 8 heads: 163 us, 6.6 TB/s).
// - Fewer: a cluster of CTAs each, which meet between the reads and the writes of a turn (8 x 8 heads, 2048 of 2300 rows:
//   17 us).
// - Fewer than 48: as many CTAs as the GPU holds take the chunks in order, from a counter, announce each that they have
//   read, and ahead of a write wait for the chunks that read what it overwrites, whose number the selection has counted
//   (3 sequences of 90000 rows to 40821, 2 heads, 29 us, in clusters 103; one of 131072 rows to 65536, one head, 17 and 140;
//   88 units of 5300 rows to 3589 42 and 45, 64 of 2300 to 2048 36 and 17).
// To other pages nothing waits.
#include "kl_internal.cuh"

namespace kl {
namespace {

constexpr int kBits0 = 11, kBits = 10;                   // of the first round, of the others
constexpr int kBins = 1 << kBits0;
constexpr int kPerThread = 4, kBinWarps = kBins / kPerThread / 32;   // the first warps find the bin
constexpr int kMostCluster = 8;
constexpr int kMovePieces = 512;                         // 16-byte pieces of a chunk of rows: one CTA's turn of the move

// What the move needs to know of a (sequence, value head): rows that stay (-1: it is left alone), whether its rows
// may move within their pages, and the chunks that CTAs have taken.
struct EvictUnit {
    int rows, in_place, taken, spare;
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
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 4 : 1)
    select_kernel(const EvictArgs a, EvictUnit *units, uint4 *read, int32_t *need, int marks, int cluster, int piece) {
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
        units[unit] = EvictUnit{fault ? -1 : rows, eq, 0, 0};
    }
    for (int i = rank * kThreads + tid; i < marks; i += cluster * kThreads)      // (no chunk has been read)
        read[(size_t)unit * marks + i] = make_uint4(0u, 0u, 0u, 0u);
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
            const uint32_t mids = (uint32_t)max(min(t1, mid1) - mid0, 0);   // (0: the piece is all first tokens)
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
    const int chunk = kMovePieces * 8 / geo.D;           // rows (a power of two)
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
            // the rows that have to be read before the chunk that ends with this place is written
            const int t1e = t + 4 * lane + e + 1;
            if ((t1e & (chunk - 1)) == 0 && t1e <= rows && t1e <= t1) need[(size_t)unit * marks * 16 + t1e / chunk - 1] = ox + min(oy, want);
        }
        const uint32_t total = __shfl_sync(0xffffffffu, upto, 31);
        before += total & 0xffffu;
        on_before += total >> 16;
    }
    // (the whole cluster writes the rest; nothing there is read again)
    for (int t = rows + rank * kThreads + tid; t < L; t += cluster * kThreads) nw[t] = 0.f;
    for (uint32_t t = rows + rank * kThreads + tid; t < (uint32_t)a.budget; t += cluster * kThreads) kept[t] = -1;
    if (cluster > 1) cluster_sync();                     // (the counts are read)
}

constexpr int kMoveThreads = 128, kMoveCtas = 8;         // per SM
constexpr int64_t kEarlyBytes = 256 << 20;               // of rows: up to here the move starts early
constexpr uint64_t kMoveWaitNs = 1000000000ull;          // bound of a wait for other CTAs' reads
constexpr int kShareUnits = 48;                          // fewer units: share_kernel
constexpr int kMoveDepth = kMovePieces / kMoveThreads;                            // 16-byte pieces per thread and turn

__device__ __forceinline__ uint64_t global_timer() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Whether the first n (or all 16) bytes at `p` are 1.
__device__ __forceinline__ bool all_read(const uint4 *p, int n) {
    bool all = true;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t v;
        asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];"
                     : "=r"(v)
                     : "l"(reinterpret_cast<const uint32_t *>(p) + e)
                     : "memory");
        const int m = min(4, n - 4 * e);
        if (m > 0) all = all && ((v ^ 0x01010101u) & (0xffffffffu >> (32 - 8 * m))) == 0;
    }
    return all;
}

// t / P and t % P: P a power of two (its shift), or any (shift -1).
struct Paging {
    int P, shift;
    __device__ __forceinline__ int page(int t) const { return shift >= 0 ? t >> shift : t / P; }
    __device__ __forceinline__ int row(int t) const { return shift >= 0 ? t & (P - 1) : t % P; }
};

// What both forms share: this thread's pieces of the rows of a chunk.
struct Mover {
    const int32_t *from, *to, *kept;
    uint4 *v;
    int64_t page_pieces;     // 16-byte pieces of a page
    int head, cpr, c, first, rstep, rows;   // head: of the value head's first row in a page; c: of this thread in a row
    Paging pg;
    __device__ __forceinline__ uint4 *piece(int page, int t) const {
        return v + page * page_pieces + head + pg.row(t) * cpr + c;
    }
    // f(k, row) for this thread's rows of the chunk from row j on
    template <typename F>
    __device__ __forceinline__ void each(int j, F &&f) const {
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k)
            if (j + first + k * rstep < rows) f(k, j + first + k * rstep);
    }
    __device__ __forceinline__ void ids(int j, int (&id)[kMoveDepth]) const {
        each(j, [&](int k, int at) { id[k] = kept[at]; });
    }
    __device__ __forceinline__ void pages(int j, const int (&id)[kMoveDepth], int (&page)[kMoveDepth]) const {
        each(j, [&](int k, int) { page[k] = from[pg.page(id[k])]; });
    }
    __device__ __forceinline__ void load(int j, const int (&id)[kMoveDepth], const int (&page)[kMoveDepth],
                                         uint4 (&x)[kMoveDepth]) const {
        each(j, [&](int k, int) { x[k] = *piece(page[k], id[k]); });
    }
    __device__ __forceinline__ void store(int j, const uint4 (&x)[kMoveDepth]) const {
        each(j, [&](int k, int at) { *piece(to[pg.page(at)], at) = x[k]; });
    }
};
// A stretch of 2^cshift pieces, number `slice`, of the rows of a unit.
__device__ __forceinline__ Mover mover(const EvictArgs &a, int unit, int rows, int slice, int cshift, const Paging &pg) {
    const Geometry &geo = a.geo;
    const int b = unit / geo.Hkv, g = unit % geo.Hkv, tid = threadIdx.x;
    Mover m;
    m.from = a.block_table + (size_t)b * geo.max_pages;
    m.to = a.new_table + (size_t)b * geo.max_pages;
    m.kept = a.kept + (size_t)unit * a.budget;
    m.v = reinterpret_cast<uint4 *>(a.v_cache);
    m.cpr = geo.D / 8;
    m.page_pieces = (int64_t)geo.Hkv * geo.P * m.cpr;
    m.head = g * geo.P * m.cpr;
    m.c = (slice << cshift) + (tid & ((1 << cshift) - 1));
    m.first = tid >> cshift;
    m.rstep = kMoveThreads >> cshift;
    m.rows = rows;
    m.pg = pg;
    return m;
}

// CTA ((unit * slices + slice) * groups + group) * team + rank: a cluster of `team` CTAs takes its chunks in turns, chunk
// rank of each; `groups` of them share a unit that moves to other pages, in place the first does it alone. Three turns
// ahead of the write a CTA reads which rows, two ahead their pages, one ahead the rows.
__global__ void __launch_bounds__(kMoveThreads, kMoveCtas) move_kernel(const EvictArgs a, const EvictUnit *units, int slices,
                                                                       int cshift, int groups, int team, const Paging pg) {
    grid_dep_wait();
    grid_dep_launch();
    const int rank = blockIdx.x % team, group = blockIdx.x / team % groups;
    const int slice = blockIdx.x / team / groups % slices, unit = blockIdx.x / team / groups / slices;
    const EvictUnit u = units[unit];
    if (u.rows < 0) return;                              // (the whole cluster)
    if (unit % a.geo.Hkv == 0 && slice == 0 && group == 0 && rank == 0 && threadIdx.x == 0)
        a.new_lens[unit / a.geo.Hkv] = u.rows;
    if (u.in_place && group > 0) return;
    const Mover m = mover(a, unit, u.rows, slice, cshift, pg);
    const int chunk = kMovePieces >> cshift, step = chunk * team * (u.in_place ? 1 : groups);
    uint4 x[kMoveDepth], y[kMoveDepth];
    int id[kMoveDepth], page[kMoveDepth], next[kMoveDepth];
    int j = (u.in_place ? rank : group * team + rank) * chunk;
    m.ids(j, id);
    m.ids(j + step, next);
    m.pages(j, id, page);
    m.load(j, id, page, x);
    m.pages(j + step, next, page);
#pragma unroll
    for (int k = 0; k < kMoveDepth; ++k) id[k] = next[k];
    m.ids(j + 2 * step, next);
    const int turns = (u.rows + step - 1) / step;        // (as many in all CTAs: they meet)
    for (int s = 0; s < turns; ++s, j += step) {
        m.load(j + step, id, page, y);
        m.pages(j + 2 * step, next, page);
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k) id[k] = next[k];
        m.ids(j + 3 * step, next);
        if (u.in_place) {                                // this turn's and the next one's rows have been read
            if (team > 1) cluster_sync();
            else __syncthreads();
        }
        m.store(j, x);
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k) x[k] = y[k];
    }
}

// CTA unit * team + t, whole rows: the CTAs of a unit take its chunks in order, from a counter. read[unit][chunk]: bytes,
// 1 once its rows have been read (marks: 16 of them each); need[unit][chunk]: the first rows that have to be read before it
// is written. The last warp keeps the books: it takes tickets, announces chunks and looks at the other CTAs' while the
// movers' loads are on their way. A ticket is taken when there is room to read its chunk at once, so that no chunk waits
// for another's write before it is read: the chunks below one that waits are with CTAs that read them.
// The marks need no fences: what was announced has been read, since its values are here, and a write that follows a mark
// in the program cannot be ahead of it. (3 sequences of 90000 rows to 40821, 2 heads: with fences, which wait for the
// writes of all warps, 122 instead of 86 us; with a wait for all chunks ahead instead of those that are needed 86
// instead of 29; with chunks in turns of the whole team instead of tickets 36.)
constexpr int kShareThreads = kMoveThreads + 32, kShareCtas = 6;
constexpr uint32_t kBarTake = 1, kBarRead = 2, kBarWrite = 3;    // a ticket is here; a chunk is; its place may be written
__device__ __forceinline__ void bar(uint32_t id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kShareThreads) : "memory"); }

__global__ void __launch_bounds__(kShareThreads, kShareCtas) share_kernel(const EvictArgs a, EvictUnit *units, uint4 *read,
                                                                          const int32_t *need, int marks, int team, int cshift,
                                                                          const Paging pg) {
    __shared__ volatile int ticket, gone;
    grid_dep_wait();
    grid_dep_launch();
    const int unit = blockIdx.x / team, tid = threadIdx.x, lane = tid & 31;
    const int rows = units[unit].rows, in_place = units[unit].in_place;
    if (rows < 0) return;
    if (unit % a.geo.Hkv == 0 && blockIdx.x % team == 0 && tid == 0) a.new_lens[unit / a.geo.Hkv] = rows;
    const int chunk = kMovePieces >> cshift;
    if (tid >= kMoveThreads) {
        uint8_t *const mine = reinterpret_cast<uint8_t *>(read + (size_t)unit * marks);
        const int32_t *const first_rows = need + (size_t)unit * marks * 16;
        auto take = [&]() -> int {
            int c = 0;
            if (lane == 0) ticket = c = atomicAdd(&units[unit].taken, 1);
            return __shfl_sync(0xffffffffu, c, 0);
        };
        // chunk c may be written once those below this have been read
        auto limit = [&](int c) -> int {
            if (!in_place || c * chunk >= rows) return 0;
            return (c + 1) * chunk > rows ? c : min(c, (__ldcg(first_rows + c) + chunk - 1) / chunk);
        };
        if (lane == 0) gone = 0;
        int known = 0, c0 = take(), stop = limit(c0);    // known: all chunks below have been read
        bar(kBarTake);
        while (c0 * chunk < rows) {
            bar(kBarRead);
            if (in_place && lane == 0)
                asm volatile("st.relaxed.gpu.global.u8 [%0], %1;" ::"l"(mine + c0), "r"(1) : "memory");
            const int c1 = take();
            bar(kBarTake);
            const int next = limit(c1);
            const uint64_t t0 = global_timer();
            while (known < stop) {
                // 16 marks per lane from the last whole 16 on; as many as follow each other from there
                const int first = known & ~15, n = min(16, stop - first - 16 * lane);
                const bool ok = n <= 0 || all_read(reinterpret_cast<const uint4 *>(mine + first) + lane, n);
                const unsigned not_yet = ~__ballot_sync(0xffffffffu, ok);
                known = not_yet ? max(known, first + 16 * (__ffs(not_yet) - 1)) : min(stop, first + 512);
                if (known < stop && global_timer() - t0 > kMoveWaitNs) {
                    gone = 1;
                    break;
                }
            }
            __syncwarp();
            bar(kBarWrite);
            if (gone) {                                  // (rows that are still to be read may not be overwritten)
                if (lane == 0) raise_flag(a.err, KL_FLAG_TIMEOUT);
                return;
            }
            c0 = c1;
            stop = next;
        }
        return;
    }
    const Mover m = mover(a, unit, rows, 0, cshift, pg);
    uint4 x[kMoveDepth], y[kMoveDepth];
#pragma unroll
    for (int k = 0; k < kMoveDepth; ++k) x[k] = y[k] = make_uint4(0u, 0u, 0u, 0u);
    int id[kMoveDepth], page[kMoveDepth];
    bar(kBarTake);
    int c0 = ticket;
    m.ids(c0 * chunk, id);
    m.pages(c0 * chunk, id, page);
    m.load(c0 * chunk, id, page, x);
    while (c0 * chunk < rows) {
        // (a word of every load goes into a branch, so that the rows are here and not only on their way)
        if ((x[0].x ^ x[1].x ^ x[2].x ^ x[3].x) == 0x9e3779b9u) __nanosleep(0);
        bar(kBarRead);
        bar(kBarTake);
        const int c1 = ticket;
        m.ids(c1 * chunk, id);
        m.pages(c1 * chunk, id, page);
        m.load(c1 * chunk, id, page, y);
        bar(kBarWrite);
        if (gone) return;
        m.store(c0 * chunk, x);
#pragma unroll
        for (int k = 0; k < kMoveDepth; ++k) x[k] = y[k];
        c0 = c1;
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
    // (the marks first: they are read 16 at a time)
    const int marks = kl_evict_marks(a.budget);
    uint4 *read = static_cast<uint4 *>(a.workspace);
    int32_t *need = reinterpret_cast<int32_t *>(read + (size_t)units * marks);
    EvictUnit *info = reinterpret_cast<EvictUnit *>(need + (size_t)units * marks * 16);
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
    cudaError_t s = cudaLaunchKernelEx(&cfg, kernel, a, info, read, need, marks, cluster, piece);
    if (s != cudaSuccess) return s;
    int shift = 0;
    while (1 << shift < g.P) ++shift;
    const Paging pg{g.P, 1 << shift == g.P ? shift : -1};
    cudaLaunchConfig_t mv = {};
    mv.blockDim = dim3(kMoveThreads);
    mv.stream = a.stream;
    // An early start saves a launch's latency, but the CTAs then crowd the SMs that the selection leaves first (64 x
    // 8192 rows to 4096, 8 heads, 1 GB of traffic: 242 us with it)
    if ((int64_t)units * (a.budget < longest ? a.budget : longest) * g.D * 4 > kEarlyBytes)
        attr[0].val.programmaticStreamSerializationAllowed = 0;
    mv.attrs = attr;
    mv.numAttrs = 1;
    const int cpr = g.D / 8, wanted = kMoveCtas * sms;
    const int64_t most = a.budget < longest ? a.budget : longest;
    int cshift = g.D == 128 ? 4 : 3;
    if (units < kShareUnits) {
        const int chunks = (int)((most + (kMovePieces >> cshift) - 1) / (kMovePieces >> cshift));
        const int places = kShareCtas * sms / units, team = places < chunks ? places : chunks;
        mv.gridDim = dim3((unsigned)(units * team));
        mv.blockDim = dim3(kShareThreads);
        return cudaLaunchKernelEx(&mv, share_kernel, a, info, read, (const int32_t *)need, marks, team, cshift, pg);
    }
    // As many CTAs as the GPU holds at a time, eight per SM: 128-byte stretches, then clusters, then (to other pages)
    // groups of clusters
    while (cshift > 3 && 2 * (int64_t)units * (cpr >> cshift) <= wanted) --cshift;
    int team = 1;
    while (team < kMostCluster && 2 * (int64_t)units * team * (cpr >> cshift) <= wanted &&
           (int64_t)(kMovePieces >> cshift) * team < most)
        team *= 2;
    const int slices = cpr >> cshift;
    const int64_t turn = (int64_t)(kMovePieces >> cshift) * team, turns = (most + turn - 1) / turn;
    int64_t groups = wanted / ((int64_t)units * slices * team);
    groups = groups < 1 ? 1 : groups > turns ? turns : groups;
    mv.gridDim = dim3((unsigned)(groups * units * slices * team));
    attr[1].val.clusterDim.x = team;
    mv.numAttrs = 2;
    return cudaLaunchKernelEx(&mv, move_kernel, a, (const EvictUnit *)info, slices, cshift, (int)groups, team, pg);
}

}  // namespace kl
