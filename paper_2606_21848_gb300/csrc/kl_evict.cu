// Eviction from the paged Value-Only Cache by accumulated attention weight, for sm_103a: of every sequence and
// value head the first `sinks` rows, the last `recent` and of those between the ones with the largest weight (ties:
// the lowest index) stay, `budget` in all; they move together in their order, and their weights with them.
//
// Two kernels. The selection: a cluster of CTAs per (sequence, value head), each with a piece of the weights in
// shared memory. The smallest weight that stays is found by three rounds over its bits from the top, 11, 10 and 10
// (a positive fp32's order is that of its bits): every CTA counts its piece's weights that have the bits found so
// far by their next ones, and by 32 of these together; all meet, add up the coarse counts through distributed shared
// memory, then the 32 fine ones, and find the same bin. Few weights are left to count after the first round. Then each
// warp counts what stays of a stretch of the piece, the counts are summed before it, and it writes. (All weights are in shared memory before the first is written:
// weights may move in place.)
// The move: 512 bytes of traffic per row of 128 bf16 values, and HBM bounds it. Rows only ever move down, so in place
// what a chunk of consecutive rows overwrites has been read once all chunks before it have been read.
// - Many (sequence, value head)s: one CTA per stretch of 128 bytes of their rows goes through the chunks and reads a
//   chunk ahead of what it writes (64 x 8192 rows to 4096, 8 heads: 163 us, 6.6 TB/s).
// - Fewer: a cluster of CTAs each, which meet between the reads and the writes of a turn (8 x 8 heads, 2048 of 2300 rows:
//   17 us).
// - Fewer than 48: as many CTAs as the GPU holds take the chunks in order, from a counter, announce each that they have
//   read, and ahead of a write wait for the chunks that read what it overwrites, whose number the selection has counted
//   (3 sequences of 90000 rows to 40821, 2 heads, 35 us, in clusters 103; one of 131072 rows to 65536, one head, 16 and 140;
//   before the fences between reads and writes, which cost up to a tenth, 88 units of 5300 rows to 3589 42, in clusters 45,
//   64 of 2300 to 2048 36 and 17).
// To other pages nothing waits. In place, rows ahead of the first that goes are where they belong and are not touched (64
// sequences of 4096 rows within their budget, 8 heads: 18 us, all of it the selection; 182 to other pages).
#include "kl_internal.cuh"

namespace kl {
namespace {

constexpr int kBits0 = 11, kBits = 10;                   // of the first round, of the others
constexpr int kBins = 1 << kBits0;
constexpr int kMostCluster = 8;
constexpr int kMovePieces = 512;                         // 16-byte pieces of a chunk of rows: one CTA's turn of the move

// What the move needs to know of a (sequence, value head): rows that stay (-1: it is left alone), whether none, some or all
// of its pages stay, the chunks that CTAs have taken, and the first row that another row takes the place of.
enum { kElsewhere = 0, kMixed = 1, kInPlace = 2 };
struct EvictUnit {
    int rows, in_place, taken, gap;
    // the first row that has to be written (rows: none)
    __device__ __forceinline__ int first() const { return in_place == kInPlace ? min(gap, rows) : 0; }
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
// The two words at `p` (8-byte aligned) of this CTA's shared memory in that of CTA `rank` of the cluster, or the first.
__device__ __forceinline__ void ld_cluster(const int *p, int rank, int (&n)[2]) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(at)
                 : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v2.b32 {%0, %1}, [%2];" : "=r"(n[0]), "=r"(n[1]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ld_cluster(const int *p, int rank, int (&n)[1]) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(at)
                 : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(n[0]) : "r"(at) : "memory");
}
// Their sums over the cluster, eight loads on their way at once.
template <int kWords>
__device__ __forceinline__ void add_cluster(const int *p, int cluster, int (&n)[kWords]) {
#pragma unroll
    for (int e = 0; e < kWords; ++e) n[e] = cluster > 1 ? 0 : p[e];
    if (cluster == 1) return;
    for (int c0 = 0; c0 < cluster; c0 += 8) {
        int v[8][kWords];
#pragma unroll
        for (int c = 0; c < 8; ++c) ld_cluster(p, min(c0 + c, cluster - 1), v[c]);
#pragma unroll
        for (int e = 0; e < kWords; ++e)
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c0 + c < cluster) n[e] += v[c][e];
    }
}

// Writes x, y to `p` (8-byte aligned) in the shared memory of CTA `rank`.
__device__ __forceinline__ void st_cluster(int *p, int rank, int x, int y) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(at)
                 : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x), "r"(y) : "memory");
}

// Sums of n over lanes 0 .. lane.
__device__ __forceinline__ int upto_lane(int n, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, n, o);
        if (lane >= o) n += x;
    }
    return n;
}

// Weights in their order as whole numbers; what is not positive, and NaN, is 0.
__device__ __forceinline__ uint32_t weight_key(float w) { return w > 0.f ? __float_as_uint(w) : 0u; }

// Cluster (b, g), CTA `rank` of it: tokens rank * piece ... kThreads: 512, of which an SM holds four CTAs, or 1024 where
// there are few units. Shared memory: the piece's weights, and two bits for each of them (above the border, on it).
template <int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 4 : 1)
    select_kernel(const EvictArgs a, EvictUnit *units, uint32_t *read, int32_t *need, int marks, int cluster, int piece) {
    constexpr int kSelWarps = kThreads / 32;
    extern __shared__ __align__(16) float held[];        // [piece], then the bits
    // of this CTA: the bins, and sums of 32 of them; the rounds take turns, since the cluster still reads the last one's
    __shared__ __align__(16) int hists[2][kBins], coarse[2][kBins / 32];
    __shared__ __align__(8) int counts[kMostCluster][2]; // of the CTAs' pieces: above the border, on it
    __shared__ int warp_above[kSelWarps], warp_on[kSelWarps];
    __shared__ uint32_t border;
    __shared__ __align__(8) int found[2];                // pages outside the pool; 1: pages that stay, 2: that do not
    __shared__ int wanted, bad;
    uint2 *const sel = reinterpret_cast<uint2 *>(held + piece);
    const Geometry &geo = a.geo;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0, unit = blockIdx.x / cluster;
    const int b = unit / geo.Hkv;
    grid_dep_wait();
    const int L = a.seq_lens[b], rows = min(L, a.budget);
    const bool first = tid == 0 && rank == 0, tells = first && unit % geo.Hkv == 0;
    if (L < 0 || L > geo.max_pages * geo.P || L > a.stride) {    // (the whole cluster)
        if (tells) raise_flag(a.err, KL_FLAG_BAD_LENGTH);
        if (first) units[unit] = EvictUnit{-1, 0, 0, 0};
        return;
    }
    // The pages of the sequence and of where it goes, shared out over the cluster, while the weights are on their way
    const int32_t *from = a.block_table + (size_t)b * geo.max_pages, *to = a.new_table + (size_t)b * geo.max_pages;
    const float *w = a.weights + (size_t)unit * a.stride;
    const int t0 = min(rank * piece, L), t1 = min(t0 + piece, L);
    constexpr int kAhead = 8;
    float ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (t0 + tid + k * kThreads < t1) ahead[k] = w[t0 + tid + k * kThreads];
    unsigned seen = 0;                                   // 1: a page outside the pool, 2: one that stays, 4: one that does not
    {
        const int pages = (L + geo.P - 1) / geo.P, new_pages = (rows + geo.P - 1) / geo.P;
#pragma unroll 2
        for (int i = rank * kThreads + tid; i < pages; i += cluster * kThreads) {
            const int p = from[i], q = i < new_pages ? to[i] : 0;
            if (p < 0 || p >= geo.num_pages || q < 0 || q >= geo.num_pages) seen |= 1;
            if (i < new_pages) seen |= p == q ? 2 : 4;
        }
    }
    for (int i = rank * kThreads + tid; i < marks; i += cluster * kThreads)      // (no chunk has been read)
        read[(size_t)unit * marks + i] = 0u;
    {
        seen = __reduce_or_sync(0xffffffffu, seen);
        if (lane == 0) warp_on[warp] = seen;
        __syncthreads();
        if (warp == 0) {
            const unsigned any = __reduce_or_sync(0xffffffffu, lane < kSelWarps ? warp_on[lane] : 0);
            if (lane == 0) {
                found[0] = any & 1;
                found[1] = any >> 1;
            }
        }
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
    auto meet = [&] {
        if (cluster > 1) cluster_sync();
        else __syncthreads();
    };
    // Warp 0, behind the first meeting: what the CTAs have found out about the pages.
    auto look_around = [&] {
        int x[2] = {0, 0};
        if (lane < cluster) {
            if (cluster > 1) ld_cluster(found, lane, x);
            else x[0] = found[0], x[1] = found[1];
        }
        const bool fault = __any_sync(0xffffffffu, x[0]);
        const int in_place = !__any_sync(0xffffffffu, x[1] & 1) ? kElsewhere : __any_sync(0xffffffffu, x[1] & 2) ? kMixed : kInPlace;
        if (lane > 0) return;
        bad = fault;
        if (tells && fault) raise_flag(a.err, KL_FLAG_BAD_PAGE);
        if (first) units[unit] = EvictUnit{fault ? -1 : rows, in_place, 0, rows};
    };
    uint32_t key = 0;
    int shift = 31;
    if (want == 0) {
        meet();
        if (warp == 0) look_around();
        __syncthreads();
    }
    for (int round = 0; round < 3 && want > 0; ++round) {
        const int bits = round == 0 ? kBits0 : kBits, known = shift;     // bits known .. 30 are found
        shift -= bits;
        int *const h = hists[round & 1], *const rough = coarse[round & 1];
        for (int i = tid; i < kBins; i += kThreads) h[i] = 0;
        __syncthreads();
        // four consecutive weights per thread; the ends of the middle one by one
        const uint32_t mask = (1u << bits) - 1, so_far = key >> known;
        const int begin = max(mid0 - t0, 0), end = min(t1, mid1) - t0;   // of the middle in this piece
        for (int at = 4 * tid; at < end; at += 4 * kThreads) {
            const float4 x = *reinterpret_cast<const float4 *>(held + at);
            const uint32_t k[4] = {weight_key(x.x), weight_key(x.y), weight_key(x.z), weight_key(x.w)};
            bool hit[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) hit[e] = k[e] >> known == so_far;
            if (!(hit[0] || hit[1] || hit[2] || hit[3])) continue;
            const bool inside = at >= begin && at + 4 <= end;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (hit[e] && (inside || (at + e >= begin && at + e < end))) atomicAdd(h + ((k[e] >> shift) & mask), 1);
        }
        __syncthreads();
        for (int i = warp; i < kBins / 32; i += kSelWarps) {
            const int n = __reduce_add_sync(0xffffffffu, h[32 * i + lane]);
            if (lane == 0) rough[i] = n;
        }
        meet();
        // the bin of the want-th largest, from the top: which 32 of them (a lane looks at two), then which of these
        if (warp == 0) {
            if (round == 0) look_around();
            int n[2], f[1];
            add_cluster(rough + kBins / 32 - 2 - 2 * lane, cluster, n);
            const int sum = n[0] + n[1], upto = upto_lane(sum, lane);
            const int l = __ffs(__ballot_sync(0xffffffffu, want <= upto)) - 1;
            int above = __shfl_sync(0xffffffffu, upto - sum, l);
            const int upper = __shfl_sync(0xffffffffu, n[1], l);
            int group = kBins / 32 - 1 - 2 * l;
            if (want > above + upper) {
                above += upper;
                --group;
            }
            add_cluster(h + 32 * group + 31 - lane, cluster, f);
            const int here = above + upto_lane(f[0], lane);
            if (lane == __ffs(__ballot_sync(0xffffffffu, want <= here)) - 1) {
                border = key | (uint32_t)(32 * group + 31 - lane) << shift;
                wanted = want - (here - f[0]);
            }
        }
        __syncthreads();
        key = border;
        want = wanted;
        if (bad) break;
    }
    if (bad) {                                           // (every CTA of the cluster, once all have read)
        if (cluster > 1) cluster_sync();
        return;
    }
    // `want` of those on the border `key` stay, the first ones; with none wanted nothing between stays
    const bool none = !all && a.budget == a.sinks + a.recent;
    // 32 consecutive tokens per step: those above the border (or first, or last), those on it
    const int per = ((t1 - t0 + kSelWarps - 1) / kSelWarps + 31) & ~31;
    const int s0 = min(t0 + warp * per, t1), s1 = min(s0 + per, t1);
    int na = 0, no = 0;
#pragma unroll 2
    for (int t = s0; t < s1; t += 32) {
        const uint32_t k = weight_key(held[t + lane - t0]);
        const bool outer = all || t + lane < mid0 || t + lane >= mid1, here = t + lane < t1;
        const unsigned above = __ballot_sync(0xffffffffu, here && (outer || (!none && k > key)));
        const unsigned on = __ballot_sync(0xffffffffu, here && !outer && !none && k == key);
        if (lane == 0) sel[(t - t0) / 32] = make_uint2(above, on);
        na += __popc(above);
        no += __popc(on);
    }
    if (lane == 0) {
        warp_above[warp] = na;
        warp_on[warp] = no;
    }
    __syncthreads();
    int before = lane < warp ? warp_above[lane] : 0, on_before = lane < warp ? warp_on[lane] : 0;
    if (cluster > 1) {
        if (warp == 0) {
            const int x = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? warp_above[lane] : 0);
            const int y = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? warp_on[lane] : 0);
            if (lane < cluster) st_cluster(counts[rank], lane, x, y);
        }
        cluster_sync();                                  // (and every CTA holds its weights; the last meeting)
        if (lane < rank) {
            before += counts[lane][0];
            on_before += counts[lane][1];
        }
    }
    // above the border and on it before this warp's stretch; those that stay
    on_before = __reduce_add_sync(0xffffffffu, on_before);
    before = __reduce_add_sync(0xffffffffu, before) + min(on_before, want);
    grid_dep_launch();
    const int chunk = geo.D == 128 ? 5 : 6;              // rows of a chunk, as a power of two
    static_assert(kMovePieces == 512, "");
    int32_t *kept = a.kept + (size_t)unit * a.budget;
    float *nw = a.new_weights + (size_t)unit * a.stride;
    __syncwarp();                                        // (sel is this warp's own)
    const unsigned below = (1u << lane) - 1;
    int32_t *ends = need + (size_t)unit * marks * 16 - 1;
#pragma unroll 2
    for (int t = s0; t < s1; t += 32) {
        const uint2 x = sel[(t - t0) / 32];
        unsigned stay = x.x;
        if (x.y && on_before < want) {                   // of those on the border the first ones
            const int left = want - on_before;
            stay |= __ballot_sync(0xffffffffu, (x.y >> lane & 1) && __popc(x.y & below) < left);
            on_before += __popc(x.y);
        }
        // (all rows before this one stay: here is the first that goes)
        if (before == t && lane == __ffs(~stay) - 1) units[unit].gap = t + lane;
        if (stay >> lane & 1) {
            const int at = before + __popc(stay & below);
            kept[at] = t + lane;
            nw[at] = held[t + lane - t0];
        }
        before += __popc(stay);
        // the rows that have to be read before the chunk that ends here is written
        if (lane == 0 && (t + 32 & (1 << chunk) - 1) == 0 && t + 32 <= min(rows, t1)) ends[(t + 32) >> chunk] = before;
    }
    // (the whole cluster writes the rest; nothing there is read again)
    for (int t = rows + rank * kThreads + tid; t < L; t += cluster * kThreads) nw[t] = 0.f;
    for (uint32_t t = rows + rank * kThreads + tid; t < (uint32_t)a.budget; t += cluster * kThreads) kept[t] = -1;
}

constexpr int kMoveThreads = 128, kMoveCtas = 8;         // per SM
constexpr int64_t kEarlyBytes = 256 << 20;               // of rows: up to here the move starts early
constexpr int kShareUnits = 48;                          // fewer units: share_kernel
constexpr int kMoveDepth = kMovePieces / kMoveThreads;                            // 16-byte pieces per thread and turn

__device__ __forceinline__ uint64_t global_timer() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Whether the lowest n (or all 32) bits at `p` are set.
__device__ __forceinline__ bool all_read(const uint32_t *p, int n) {
    uint32_t v;
    asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return n >= 32 ? v == ~0u : (~v & ((1u << n) - 1)) == 0;
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
    int low;                 // the first row that is written
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
        each(j, [&](int k, int at) {
            if (at >= low) *piece(to[pg.page(at)], at) = x[k];
        });
    }
};
// A stretch of 2^cshift pieces, number `slice`, of the rows of a unit.
__device__ __forceinline__ Mover mover(const EvictArgs &a, int unit, const EvictUnit &u, int slice, int cshift, const Paging &pg) {
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
    m.rows = u.rows;
    m.low = u.first();
    m.pg = pg;
    return m;
}

// CTA ((unit * slices + slice) * groups + group) * team + rank: a cluster of `team` CTAs takes its chunks in turns, chunk
// rank of each; `groups` of them share a unit that moves to other pages, in place the first does it alone. Three turns
// ahead of the write a CTA reads which rows, two ahead their pages, one ahead the rows. Rows ahead of the first that
// goes are not written.
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
    if ((u.in_place && group > 0) || u.first() >= u.rows) return;
    const Mover m = mover(a, unit, u, slice, cshift, pg);
    const int chunk = kMovePieces >> cshift, step = chunk * team * (u.in_place ? 1 : groups);
    const int j0 = u.first() & ~(chunk - 1);             // (a power of two)
    uint4 x[kMoveDepth], y[kMoveDepth];
    int id[kMoveDepth], page[kMoveDepth], next[kMoveDepth];
    int j = j0 + (u.in_place ? rank : group * team + rank) * chunk;
    m.ids(j, id);
    m.ids(j + step, next);
    m.pages(j, id, page);
    m.load(j, id, page, x);
    m.pages(j + step, next, page);
#pragma unroll
    for (int k = 0; k < kMoveDepth; ++k) id[k] = next[k];
    m.ids(j + 2 * step, next);
    const int turns = (u.rows - j0 + step - 1) / step;   // (as many in all CTAs: they meet)
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

// CTA unit * team + t, whole rows: the CTAs of a unit take its chunks in order, from a counter. read[unit]: a bit per chunk
// from the first that is written on, set once its rows have been read; need[unit][chunk]: the first rows that have to be
// read before it is written. The last warp keeps the books: it takes tickets, announces chunks and looks at the other CTAs'
// while the movers' loads are on their way. A ticket is taken when there is room to read its chunk at once, so that no chunk waits
// for another's write before it is read: the chunks below one that waits are with CTAs that read them.
// The marks are bits of words that are read as words, with a fence between a chunk's reads and its mark, and one between
// the marks that a CTA has seen and its writes: what it overwrites has been read. (3 sequences of 90000 rows to 40821, 2
// heads: the fences cost 4 of 35 us, since they wait for the writes of all warps. Without them, 29 us: 86 with a wait for
// all chunks ahead instead of those that are needed, 36 with chunks in turns of the whole team instead of tickets.)
constexpr int kShareThreads = kMoveThreads + 32, kShareCtas = 6;
constexpr uint32_t kBarTake = 1, kBarRead = 2, kBarWrite = 3;    // a ticket is here; a chunk is; its place may be written
__device__ __forceinline__ void bar(uint32_t id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kShareThreads) : "memory"); }
__device__ __forceinline__ void gpu_fence() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }

__global__ void __launch_bounds__(kShareThreads, kShareCtas) share_kernel(const EvictArgs a, EvictUnit *units, uint32_t *read,
                                                                          const int32_t *need, int marks, int team, int cshift,
                                                                          const Paging pg) {
    __shared__ volatile int ticket, gone;
    grid_dep_wait();
    grid_dep_launch();
    const int unit = blockIdx.x / team, tid = threadIdx.x, lane = tid & 31;
    const EvictUnit u = units[unit];                     // (but for `taken`)
    const int rows = u.rows, in_place = u.in_place;
    if (rows < 0) return;
    if (unit % a.geo.Hkv == 0 && blockIdx.x % team == 0 && tid == 0) a.new_lens[unit / a.geo.Hkv] = rows;
    const int chunk = kMovePieces >> cshift, base = u.first() / chunk;    // the first chunk that is written
    if (u.first() >= rows) return;
    if (tid >= kMoveThreads) {
        uint32_t *const mine = read + (size_t)unit * marks;
        const int32_t *const first_rows = need + (size_t)unit * marks * 16;
        auto take = [&]() -> int {
            int c = 0;
            if (lane == 0) ticket = c = base + atomicAdd(&units[unit].taken, 1);
            return __shfl_sync(0xffffffffu, c, 0);
        };
        // chunk c may be written once those from base to below base + this have been read
        auto limit = [&](int c) -> int {
            if (!in_place || c * chunk >= rows) return 0;
            return ((c + 1) * chunk > rows ? c : min(c, (__ldcg(first_rows + c) + chunk - 1) / chunk)) - base;
        };
        if (lane == 0) gone = 0;
        int known = 0, c0 = take(), stop = limit(c0);    // known: so many chunks from base on have been read
        bar(kBarTake);
        while (c0 * chunk < rows) {
            bar(kBarRead);
            if (in_place && lane == 0) {
                gpu_fence();
                asm volatile("red.relaxed.gpu.global.or.b32 [%0], %1;"
                             ::"l"(mine + ((c0 - base) >> 5)), "r"(1u << ((c0 - base) & 31))
                             : "memory");
            }
            const int c1 = take();
            bar(kBarTake);
            const int next = limit(c1);
            const uint64_t t0 = global_timer();
            const bool looks = known < stop;
            while (known < stop) {
                // a word of marks per lane from the last whole one on; as many as follow each other from there
                const int first = known & ~31, n = min(32, stop - first - 32 * lane);
                const bool ok = n <= 0 || all_read(mine + (first >> 5) + lane, n);
                const unsigned not_yet = ~__ballot_sync(0xffffffffu, ok);
                known = not_yet ? max(known, first + 32 * (__ffs(not_yet) - 1)) : min(stop, first + 1024);
                // (one lane's clock decides for the warp)
                if (known < stop && __shfl_sync(0xffffffffu, global_timer() - t0 > a.wait_ns, 0)) {
                    if (lane == 0) gone = 1;
                    break;
                }
            }
            if (looks) gpu_fence();
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
    const Mover m = mover(a, unit, u, 0, cshift, pg);
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
        // (a word of every load goes into a branch, so that the rows are here and not only on their way: the 16 bytes of
        // a load come together)
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
    const int marks = kl_evict_marks(a.budget);
    uint32_t *read = static_cast<uint32_t *>(a.workspace);
    int32_t *need = reinterpret_cast<int32_t *>(read + (size_t)units * marks);
    EvictUnit *info = reinterpret_cast<EvictUnit *>(need + (size_t)units * marks * 16);
    const bool few = units * cluster <= sms;
    const auto kernel = few ? select_kernel<1024> : select_kernel<512>;
    static PerDeviceOnce once[2];
    const cudaError_t e = once[few].run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    KL_EVICT_MAX_TOKENS / kMostCluster / 4 * 17);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * cluster));
    cfg.blockDim = dim3(few ? 1024 : 512);
    cfg.dynamicSmemBytes = piece / 4 * 17;
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
