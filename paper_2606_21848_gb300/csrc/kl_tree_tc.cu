// Attention of a tree of drafted tokens over the paged Value-Only Cache (the verification step of
// speculative decoding), for sm_103a; head_dim 128.
//
// Sequence b holds L cached rows, the last n of them drafted tokens that form a forest: draft i's parent
// is an earlier draft or the last committed token. Draft i sees the committed tokens t < L - n, itself
// and its ancestors. With q_r = q W^R (Section 2.2) and the decode formula of Section 3,
//   s_t = scale <q_r, v_t>,  out = sum_t softmax(s)_t v_t   over the tokens that the draft sees.
// n = 1 is the decode step, a chain of drafts the causal chunk.
//
// The G heads of a value head's group times the n drafts read the same cache rows: a unit is a block of up
// to 128 of these (draft, head) rows with the sequence's cache tiles. One CTA per SM; all units' tiles
// are laid end to end and cut into equal runs, one per CTA, so that batches of any lengths fill the GPU
// evenly. A unit that lies in several runs leaves a state (m, l, O) per part, which a second kernel
// merges. For each segment (a unit's tiles within a run):
//
//   routing  Q_r = Q . W^R                             M = 128 rows, N = 128, K = 128
//   scores   S   = sum_i Q_i . V_t^T                   M = 128 rows, N = 64 tokens, K = 128 per term
//   output   O  += sum_i P_i . V_t                     M = 128 rows, N = 128 dims, K = 64 per term
//
// Each cached tile V_t [128 tokens x 128 dims] arrives once by TMA (one box per page and 64 dims) and
// feeds both products from the same shared-memory copy, as the K-major B operand of the scores and the
// MN-major one of the output. Q and P are A operands in tensor memory.
//
// Precision. bf16 outputs (Half): the tile is converted to fp16 in place (exact for bf16 values of magnitude
// 2^-14 to 65280, within 2^-25 below), the routed query is a sum of two fp16 operands (22 bits), the weights
// are one (11 bits: an output is off by 2^-12 of a weight's share, against its own rounding of 2^-8). With one
// operand for the query a score s was off by |s| 2^-12, which moves the weights of tokens with scores of
// hundreds by a tenth; a tile then took 1.0 us, with two 1.2 (64 sequences of 8192 tokens, 64 / 8 heads, 16 drafts
// 268 and 322 us, 512 to 32768 tokens, up to 24 drafts 501 and 598, one of 131072, 32 drafts 72 and 86). Values or
// queries past fp16's range make the outputs that take part in them NaN (KL_FLAG_RANGE).
// fp32 outputs (Full): query and weights are sums of three bf16 terms (24 bits), and since the tensor
// core's adds truncate, O moves every 128 tokens to a sum in shared memory.
//
// What bounds it. Half, on long caches: nothing alone; a tile's three products take 1.0 us at the peak rate, HBM
// delivers a tile to every SM in 0.73. (The sizes above take 323, 40 and 163 us at HBM's rate.) Short caches
// are bound by latency: starting a segment takes 5 us, of them the routing and the first scores 3.5, and units
// of several parts 3 to 5 us for the merge.
// Full: three score and three output products per tile (2.0 us at the peak rate); a tile takes 2.7 us. 12
// sequences of 3001 to 6007 tokens, 12 / 2 heads, 61 to 64 drafts, W^R per query head: 74 us.
//
// The softmax works on half tiles of 64 tokens, thread = row = TMEM lane. A row's reference maximum moves
// only when a half tile's maximum passes it by more than 2^14.
//
// Roles: two groups of four softmax warps (and epilogue), then one warp each for the producer (TMA), the routing
// and score MMAs (owner of the tensor memory) and the output MMAs, and four helpers, which for Half convert
// tiles to fp16 ahead of their score MMAs and for Full move O to the sum (by the softmax warps, between a half
// tile's maximum and its weights, a tile took 5 us). Every wait is bounded (kl_set_wait_timeout_ns); a
// wait that runs out raises KL_FLAG_TIMEOUT and every role leaves, drains its copies and MMAs and
// frees the tensor memory.
#include <cudaTypedefs.h>
#include <math.h>

#include "kl_internal.cuh"
#include "kl_tc_rows.cuh"
#include "kl_tree_plan.cuh"

namespace kl {
namespace {

constexpr int kD = 128;
constexpr int kBM = kTreeRows;                    // rows per block
constexpr int kBN = kTreeTile;                    // cache rows per tile
constexpr int kBS = 64;                           // cache rows per half tile
constexpr uint32_t kTileBytes = kBN * kD * 2;     // 32 KiB
constexpr uint32_t kHalfBytes = kTileBytes / 2;   // one 64-dim half: 128 rows x 128 B
constexpr uint32_t kTmemCols = 512;
// A reference moves when a weight would pass 2^14 (fp16 ends at 2^16; a stale reference costs no precision that
// bf16 outputs show, and three bf16 terms have fp32's range).
constexpr float kRescaleLog2 = 14.f;
constexpr uint64_t kTimeoutNs = kRowsTimeoutNs;
constexpr uint32_t kBarCompute = 1;   // named barrier of the compute warps (0 is __syncthreads)

// Operand forms and the layout that they leave room for. Two groups of four softmax warps (thread = row =
// TMEM lane) take alternate half tiles. Tensor memory: kSub buffers of kBuf columns (64 of scores, then the
// weights, 32 per term), then
//   Half: an O of 128 columns for each group, which so keeps its own reference and never waits for the other,
//     and the query's first term (64 columns). The second is in shared memory in the query block's place (with
//     both here and two buffers of scores 64 sequences of 8192 tokens took 350 us, this way 322). Four warps
//     convert tiles to fp16 ahead of the score MMAs.
//   Full: one O, the query's terms (64 columns each).
// The routed queries first land in columns 0 .. 255, before anything else is there.
struct Half {
    static constexpr bool kFp16 = true;
    static constexpr int kQTerms = 1, kPTerms = 1, kSub = kTreeSub, kStages = 5;
    static constexpr uint32_t kBuf = 64, kColO = 192, kColQ = 448;
};
struct Full {
    static constexpr bool kFp16 = false;
    static constexpr int kQTerms = 3, kPTerms = 3, kSub = kTreeSubFp32, kStages = 3;
    static constexpr uint32_t kBuf = 96, kColO = 192, kColQ = 320;
};
constexpr int kGroups = kTreeGroups;
// Registers: of the 128 per thread at launch, the other warps give up 32 and the softmax warps take them
// (a half tile of scores and weights, 64 registers, spilled at 128. 168 / 88: 1 to 3 % slower).
constexpr uint32_t kSoftmaxRegs = 160, kOtherRegs = 96;
static_assert(8 * kSoftmaxRegs + 8 * kOtherRegs <= 16 * 128, "");
template <typename C>
struct Warps {
    static constexpr int kCompute = 4 * kGroups;
    static constexpr int kProducer = kCompute, kMma = kCompute + 1, kPv = kCompute + 2, kHelp = kCompute + 4;
    static constexpr int kThreads = 32 * (kHelp + 4);
};
constexpr int kFoldSub = kTreeFold;   // Full: half tiles between two moves of O to the fp32 sum

template <typename C>
struct __align__(1024) TreeSmem {
    uint8_t q[kBM * kD * 2];               // query block, K-major SW128: [64-dim half][128 rows][128 B]; Half: then
                                           // the routed query's second term
    // Ring: the W^R matrices, then the cache tiles ([64-dim half][128 rows][128 B], SW128).
    uint8_t tiles[C::kStages][kTileBytes];
    float sum[C::kFp16 ? 4 : kBM * kD];    // Full: O of the half tiles folded so far, [row][128], its
                                           // 16-byte chunks c at c ^ (row % 32)
    // Barriers (set up anew for every segment): one completion per ring position r of its slot r % kStages on
    // empty, and on w_full where it holds a W^R; per tile t on full[t % kStages] (the copy) and v_full[t %
    // kStages] (Half: its rows are fp16) -- by the tile's number and not by its slot, so that a warp which
    // waits for tiles alone never meets W^R's phases; per half tile u on s_full[u % 4] (its scores),
    // p_full[u % 4] (its weights) and s_free[u % 4] (its output MMAs are done; of its buffer u % kSub: but
    // barriers by u % 4, so that a group meets every phase of those it waits for), and per lane quarter on
    // turn[.][u % kTreeTurns] (Full: the references after it).
    struct Bars {
        uint64_t w_full[C::kStages], full[C::kStages], empty[C::kStages];
        uint64_t s_full[4], s_free[4];
        uint64_t p_full[4], o_free, sum_full, v_full[C::kStages];
        uint64_t turn[4][kTreeTurns];
        uint64_t first[4];                 // per lane quarter: the maxima of half tile 1 are in lsum[1]
        uint64_t r_full[2], r_free[2];     // routing results, alternating halves of columns 0 .. 255
        uint64_t qr_ready, par_ready, drain, drain2;
    } bar;
    float mref[4][kBM];        // the rows' references: Full after half tile u at u % 4, Half each group's last
    float lsum[kGroups][kBM];  // the groups' shares of the row sums, for the epilogue; Full: before it,
                               // lsum[1] holds half tile 1's maxima for the first reference
    float fref[kBM];           // Full: the references of `sum`
    int32_t parent[KL_TREE_MAX_DRAFTS];
    unsigned int over[KL_TREE_MAX_DRAFTS / 32];   // drafts that are not finite (Half: as fp16)
    TreeSegment seg[2];        // this segment and the next
    int64_t warp_tiles[Warps<C>::kThreads / 32];
    int warp_units[Warps<C>::kThreads / 32];
    int64_t x0, x1;            // this CTA's run, moved down to cuts
    uint32_t tmem_base;
    int abort;
};
static_assert(sizeof(TreeSmem<Half>) + 1024 <= 227 * 1024 && sizeof(TreeSmem<Full>) + 1024 <= 227 * 1024, "");

// Arrivals that complete a phase of barrier i (in the order of Bars) when `quarters` of the four lane quarters
// hold rows (the softmax warps of the others rest).
template <typename C>
__device__ __forceinline__ uint32_t bar_count(int i, int quarters) {
    using B = typename TreeSmem<C>::Bars;
    if (i >= (int)(offsetof(B, p_full) / 8) && i < (int)(offsetof(B, v_full) / 8)) return quarters;
    if (i >= (int)(offsetof(B, v_full) / 8) && i < (int)(offsetof(B, turn) / 8)) return 4;
    if (i >= (int)(offsetof(B, r_free) / 8) && i <= (int)(offsetof(B, qr_ready) / 8)) return kGroups * quarters;
    return 1;
}

// The 64 bits off .. off + 63 of the 128-bit set (lo, hi), off in -63 .. 127; bits below 0 are ones.
__device__ __forceinline__ uint64_t window64(uint64_t lo, uint64_t hi, int off) {
    if (off < 0) return (lo << -off) | ((1ull << -off) - 1);
    if (off == 0) return lo;
    return off < 64 ? (lo >> off) | (hi << (64 - off)) : hi >> (off - 64);
}

// ---------------------------------------------------------------------- runs and segments ----
//
// All units lie end to end on one line, each as a.start (what starting a segment takes, in tiles) and its
// tiles; the runs are equal shares of it. A run's start moves down to a cut: the unit's start, or a multiple
// of the unit's step among its tiles.

// Sequence b as the units see it: its drafts, length, tiles per unit and units (0 where it has none).
struct TreeSeq {
    int q0, n, L, tiles, units;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs &a, int b, bool report) {
    TreeSeq s;
    s.q0 = a.cu_q[b];
    const int q1 = a.cu_q[b + 1];
    s.L = a.seq_lens[b];
    s.n = q1 - s.q0;
    s.tiles = s.units = 0;
    if (s.q0 < 0 || s.n < 0 || q1 > a.total_q || s.n > a.max_q || s.L < s.n ||
        s.L > a.geo.max_pages * a.geo.P) {
        if (report) raise_flag(a.err, KL_FLAG_BAD_LENGTH);
    } else if (s.n > 0) {
        s.tiles = (s.L + kBN - 1) / kBN;
        s.units = a.geo.Hkv * ((a.geo.G + a.hp - 1) / a.hp) * ((s.n + a.rpb - 1) / a.rpb);
    }
    return s;
}

// Cuts inside a unit of `tiles` tiles fall on multiples of this.
__device__ __forceinline__ int cut_step(const TreeArgs &a, int tiles) {
    return a.num_splits > 0 ? (tiles + a.num_splits - 1) / a.num_splits : tiles <= a.whole ? tiles : kTreeCut;
}

// Quotients of what mostly fits 32 bits (the 64-bit division is a long sequence of instructions).
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
    return (x | y) <= INT32_MAX ? (int)x / (int)y : x / y;
}

// The start of run c of the line that `s` shares out, and the run whose share holds x.
__device__ __forceinline__ int64_t run_start(const TreeShare &s, int c) {
    return s.each * c + min(c, s.extra);
}
__device__ __forceinline__ int run_of(const TreeShare &s, int64_t x) {
    const int64_t first = (s.each + 1) * s.extra;
    return x < first ? (int)quotient(x, s.each + 1) : s.extra + (int)quotient(x - first, s.each);
}

// The tile of a unit (`off` past its start on the line) that a run's start moves down to.
__device__ __forceinline__ int cut_tile(int start, int64_t off, int tiles, int step) {
    return off <= start ? 0 : off >= start + tiles ? tiles : ((int)off - start) / step * step;
}

// Finds this CTA's run: sm.x0, sm.x1 and the first segment; writes the CTA's entry for the merge. All
// threads; ends behind a barrier. False if there is nothing to do.
template <typename C>
__device__ bool find_run(TreeSmem<C> &sm, const TreeArgs &a) {
    constexpr int kThreads = Warps<C>::kThreads;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = blockIdx.x;
    const int B = a.geo.B, per = (B + kThreads - 1) / kThreads;
    const int b0 = tid * per, b1 = min(B, b0 + per);
    int64_t mine = 0;
    int units = 0;
    TreeSeq only = TreeSeq{0, 0, 0, 0, 0};           // (the sequence of a thread that has one)
    for (int b = b0; b < b1; ++b) {
        only = tree_seq(a, b, c == 0);
        mine += (int64_t)(only.tiles + a.start) * only.units;
        units += only.units;
    }
    int64_t upto = mine;                             // inclusive prefix
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    units = __reduce_add_sync(0xffffffffu, units);
    if (lane == 31) {
        sm.warp_tiles[warp] = upto;
        sm.warp_units[warp] = units;
    }
    if (tid == 0) a.merge[c].rows = 0;
    __syncthreads();
    int64_t total = 0;
    units = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) upto += sm.warp_tiles[w];
        total += sm.warp_tiles[w];
        units += sm.warp_units[w];
    }
    // as many runs as there are CTAs, while they have a.run tiles or a unit each
    const int64_t most = max((int64_t)units, total / (a.run + a.start));
    const int runs = (int)(most < (int64_t)gridDim.x ? most : (int64_t)gridDim.x);
    if (c >= runs) return false;
    const int64_t each = quotient(total, runs);
    const TreeShare share{each, (int)(total - each * runs), runs};
    // the threads whose sequences hold the run's two ends move them down to a cut
    for (int end = 0; end < 2; ++end) {
        const int64_t x = run_start(share, c + end);
        if (x == total) {
            if (tid == 0) sm.x1 = total;
            continue;
        }
        if (x < upto - mine || x >= upto) continue;
        int64_t start = upto - mine;
        for (int b = b0; b < b1; ++b) {
            const TreeSeq s = per == 1 ? only : tree_seq(a, b, false);
            const int len = s.tiles + a.start;
            const int64_t all = (int64_t)len * s.units;
            if (x < start + all) {
                const int unit = (int)quotient(x - start, len);
                const int64_t unit0 = start + (int64_t)unit * len;
                const int step = cut_step(a, s.tiles), tile0 = cut_tile(a.start, x - unit0, s.tiles, step);
                const int64_t at = tile0 ? unit0 + a.start + tile0 : unit0;
                if (end == 1) {
                    sm.x1 = at;
                } else {
                    sm.x0 = at;
                    sm.seg[0] = TreeSegment{unit0, b, unit, tile0, s.q0, s.n, s.L, s.tiles, s.units};
                    // the first run that starts inside the unit announces its parts
                    if (tile0 > 0 && cut_tile(a.start, run_start(share, c - 1) - unit0, s.tiles, step) == 0) {
                        const TreeBlock k = tree_block(a, sm.seg[0]);
                        a.merge[c] = TreeMerge{unit0, share, s.tiles, step,
                                               run_of(share, unit0 + a.start + s.tiles - 1), s.q0 + k.m0, k.rows,
                                               k.h, k.hn};
                    }
                }
                break;
            }
            start += all;
        }
    }
    __syncthreads();
    return sm.x1 > sm.x0;
}

// The segment after `s` in a run that goes on behind s's unit: the next unit.
__device__ __forceinline__ TreeSegment next_segment(const TreeArgs &a, const TreeSegment &s) {
    TreeSegment t = s;
    t.unit0 = s.unit0 + a.start + s.tiles;
    t.tile0 = 0;
    if (++t.unit == s.units) {
        t.unit = 0;
        TreeSeq q;
        do {
            ++t.b;
            q = tree_seq(a, t.b, false);
        } while (q.units == 0);                      // (the line goes on, so a sequence follows)
        t.q0 = q.q0;
        t.n = q.n;
        t.L = q.L;
        t.tiles = q.tiles;
        t.units = q.units;
    }
    return t;
}

// ------------------------------------------------------------------------------- kernel ----
// kExact: a limit of the waits below kExactWaitNs.
template <typename C, bool kExact>
__global__ void __launch_bounds__(Warps<C>::kThreads, 1)
    tree_tc_kernel(const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap wmap,
                   const __grid_constant__ CUtensorMap qmap, const TreeArgs a) {
    constexpr int kSub = C::kSub, kStages = C::kStages;
    constexpr int kComputeWarps = Warps<C>::kCompute, kProducerWarp = Warps<C>::kProducer;
    constexpr int kMmaWarp = Warps<C>::kMma, kPvWarp = Warps<C>::kPv, kHelpWarp = Warps<C>::kHelp;
    constexpr uint32_t kColO = C::kColO, kColQ = C::kColQ;
    using Smem = TreeSmem<C>;
    extern __shared__ uint8_t smem_raw[];
    Smem &sm = *reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const Geometry &geo = a.geo;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int hp = a.hp, rpb = a.rpb;

    // (set up while the kernel ahead ends: nothing here touches global memory)
    if (tid == 0) sm.abort = 0;
    if (warp == kMmaWarp) {
        ptx::tmem_alloc(&sm.tmem_base, kTmemCols);
        ptx::tmem_relinquish();
    }
    if (warp == kProducerWarp && lane == 0) {
        ptx::prefetch_tensormap(&vmap);
        if (a.w_r) {
            ptx::prefetch_tensormap(&wmap);
            ptx::prefetch_tensormap(&qmap);
        }
    }
    // rows of the query block that its box does not fill
    if (a.w_r) {
        for (int i = tid; i < (kBM - hp * rpb) * 16; i += Warps<C>::kThreads)
            *reinterpret_cast<uint4 *>(sm.q + (i & 8 ? kHalfBytes : 0) + (hp * rpb + (i >> 4)) * 128 +
                                       (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        ptx::fence_proxy_async_smem();
    }
    grid_dep_wait();
    ptx::tc_fence_before();
    const bool any = find_run(sm, a);
    ptx::tc_fence_after();
    if (!any) {
        if (warp == kMmaWarp) ptx::tmem_dealloc(sm.tmem_base, kTmemCols);
        return;
    }
    const int64_t x1 = sm.x1;
    const Waiter<kExact> wait{&sm.abort, a.err, a.wait_ns};

    // One segment's start for all threads: its block, the barriers, the drafts' parents
    struct Part {
        TreeSegment sg;
        TreeBlock blk;
        int n_tiles, n_sub;    // tiles, half tiles
        int ro;                // ring positions of W^R matrices
        bool has_drafts, whole, more;
    };
    auto begin = [&](int si) -> Part {
        const TreeSegment sg = sm.seg[si & 1];
        const bool more = x1 > sg.unit0 + a.start + sg.tiles;     // the run goes on behind the unit
        const int n_tiles = (int)min((int64_t)sg.tiles, x1 - sg.unit0 - a.start) - sg.tile0;
        // The block: drafts m0 .. m0 + rows - 1, heads h .. h + hn - 1 of the group; row r of the 128 is
        // draft m0 + r / hp with head h + r % hp.
        const TreeBlock blk = tree_block(a, sg);
        const int hn = blk.hn, n = sg.n, L = sg.L, tile0 = sg.tile0;
        const int base = L - n;                      // committed tokens
        const int n_sub = min(2 * n_tiles, (L + kBS - 1) / kBS - 2 * tile0);   // half tiles
        const bool has_drafts = (tile0 + n_tiles) * kBN > base;
        const bool whole = n_tiles == sg.tiles;
        // ring positions of W^R matrices: one, one per head of the block, or none (composed query)
        const int ro = a.w_r ? (geo.wr_per_qh ? hn : 1) : 0;

        uint64_t *const bars = reinterpret_cast<uint64_t *>(&sm.bar);
        if (tid < (int)(sizeof(sm.bar) / 8)) {
            if (si > 0) ptx::mbar_inval(bars + tid);
            ptx::mbar_init(bars + tid, bar_count<C>(tid, (blk.rows * hp + 31) >> 5));
            ptx::fence_mbar_init();
        }
        if (tid < KL_TREE_MAX_DRAFTS / 32) sm.over[tid] = 0;
        ptx::tc_fence_before();
        __syncthreads();
        ptx::tc_fence_after();
        if (si == 0) grid_dep_launch();
        return Part{sg, blk, n_tiles, n_sub, ro, has_drafts, whole, more};
    };
    // ... and its end; false after the run's last
    auto end = [&](const Part &k) {
        ptx::tc_fence_before();
        __syncthreads();
        ptx::tc_fence_after();
        return k.more && !sm.abort;
    };

    if (warp >= kComputeWarps) {
        ptx::regs_dec<kOtherRegs>();
        for (int si = 0;; ++si) {
            const Part k = begin(si);
            const uint32_t tmem = sm.tmem_base;
            const TreeSegment &sg = k.sg;
            const int m0 = k.blk.m0, h = k.blk.h, g = k.blk.g;
            const int q0 = sg.q0, L = sg.L, tile0 = sg.tile0, n_tiles = k.n_tiles;
            const int base = L - sg.n, n_sub = k.n_sub, ro = k.ro;
            if (warp == kProducerWarp) {
                // -------------------------------------------------------------- producer ----
                const int P = geo.P;
                const int ppt = kBN / P;                          // pages per tile (<= 8)
                const int seq_pages = (L + P - 1) / P;
                const uint32_t page_bytes = (uint32_t)P * 128u;   // one half of one page
                const int32_t *bt = a.block_table + (size_t)sg.b * geo.max_pages;
                int issued = 0;
                bool bad = false, ok = true;
                // the drafts' parents, on their way while the first copies are issued
                constexpr int kPer = KL_TREE_MAX_DRAFTS / 32;
                int32_t parent[kPer];
                if (k.has_drafts)
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        parent[i] = i * 32 + lane < sg.n ? a.parents[q0 + i * 32 + lane] : -1;
                // W^R matrices (B operand of the routing MMAs); the first brings the query block along
                for (int r = 0; r < ro; ++r) {
                    const int s = r % kStages;
                    if (r >= kStages && !(ok = wait(&sm.bar.empty[s], ((r / kStages) & 1) ^ 1))) break;
                    if (lane == 0) {
                        const int wrow = (geo.wr_per_qh ? h + r : g) * kD;
                        ptx::mbar_arrive_expect_tx(&sm.bar.w_full[s], kTileBytes + (r == 0 ? hp * rpb * kD * 2 : 0));
                        ptx::tma_load_2d(sm.tiles[s], &wmap, &sm.bar.w_full[s], 0, wrow);
                        ptx::tma_load_2d(sm.tiles[s] + kHalfBytes, &wmap, &sm.bar.w_full[s], 64, wrow);
                        if (r == 0) {
                            ptx::tma_load_3d(sm.q, &qmap, &sm.bar.w_full[s], 0, h, q0 + m0);
                            ptx::tma_load_3d(sm.q + kHalfBytes, &qmap, &sm.bar.w_full[s], 64, h, q0 + m0);
                        }
                    }
                    __syncwarp();
                    issued = r + 1;
                }
                if (k.has_drafts) {
                    // (one that is not an earlier draft or -1 counts as -1)
                    bool wrong = false;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        const int j = i * 32 + lane;
                        const bool fine = parent[i] >= -1 && parent[i] < j;
                        wrong |= !fine;
                        sm.parent[j] = fine ? parent[i] : -1;
                    }
                    if (wrong) raise_flag(a.err, KL_FLAG_BAD_TREE);
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sm.bar.par_ready);
                }
                for (int i = 0; ok && i < n_tiles; ++i) {
                    const int r = i + ro, s = r % kStages;
                    uint64_t *const full = &sm.bar.full[i % kStages];
                    const int pg = (tile0 + i) * ppt + lane;      // page index within the sequence
                    const bool exists = lane < ppt && pg < seq_pages;
                    const int page = exists ? bt[pg] : -1;
                    if (r >= kStages && !wait(&sm.bar.empty[s], ((r / kStages) & 1) ^ 1)) break;
                    const bool in_range = exists && page >= 0 && page < geo.num_pages;
                    if (exists && !in_range) bad = true;
                    const unsigned mask = __ballot_sync(0xffffffffu, in_range);
                    ptx::for_pages(
                        (page * geo.Hkv + g) * P, mask,
                        [&] { ptx::mbar_arrive_expect_tx(full, __popc(mask) * page_bytes * 2u); },
                        [&](int p, int row) {
                            uint8_t *dst = sm.tiles[s] + p * page_bytes;
                            ptx::tma_load_2d(dst, &vmap, full, 0, row);
                            ptx::tma_load_2d(dst + kHalfBytes, &vmap, full, 64, row);
                        });
                    issued = r + 1;
                }
                // the last commit of every slot lands before the barriers are set up anew
                for (int i = max(0, ro + n_tiles - kStages); ok && i < ro + n_tiles; ++i)
                    ok = wait(&sm.bar.empty[i % kStages], (i / kStages) & 1);
                if (__any_sync(0xffffffffu, bad) && lane == 0) raise_flag(a.err, KL_FLAG_BAD_PAGE);
                if (sm.abort) {
                    // copies still in flight land before the CTA's shared memory goes away
                    for (int i = max(0, issued - kStages); i < issued; ++i) {
                        const int t = i - ro;
                        uint64_t *const full = t < 0 ? &sm.bar.w_full[i % kStages] : &sm.bar.full[t % kStages];
                        const uint32_t parity = ((t < 0 ? i : t) / kStages) & 1;
                        const uint64_t t0 = ptx::globaltimer();
                        while (!ptx::mbar_try_wait(full, parity) && ptx::globaltimer() - t0 < kTimeoutNs) {
                        }
                    }
                }
            } else if (warp == kMmaWarp || warp == kPvWarp) {
                // ------------------------------------------------------------ MMA issuers ----
                // K-major SW128 operands step 32 B per 16 columns inside a 64-column half and jump a
                // half (kHalfBytes) every 4 steps; MN-major SW128 operands step 16 rows = 2 KiB; TMEM
                // A operands step 8 columns (16 packed 16-bit values).
                constexpr uint32_t idesc_qk =
                    C::kFp16 ? idesc_f16(128, kBS, false, false) : ptx::idesc_bf16(128, kBS, false, false);
                constexpr uint32_t idesc_route = ptx::idesc_bf16(128, 128, false, true);
                constexpr uint32_t idesc_pv = C::kFp16 ? idesc_f16(128, 128, false, true) : idesc_route;
                const uint64_t q_desc = ptx::smem_desc(ptx::smem_addr(sm.q), 16, 1024, ptx::kSwizzle128B);
                const uint64_t k_desc = ptx::smem_desc(ptx::smem_addr(sm.tiles[0]), 16, 1024, ptx::kSwizzle128B);
                const uint64_t mn_desc =
                    ptx::smem_desc(ptx::smem_addr(sm.tiles[0]), kHalfBytes, 1024, ptx::kSwizzle128B);
                auto kstep = [](int kk) -> uint32_t { return ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4; };
                if (warp == kMmaWarp) {
                    // Q_r = Q . W^R for all 128 rows, once per matrix, into alternating halves of columns
                    // 0 .. 255 (a row keeps the result of its head's matrix), then the scores
                    bool ok = true;
                    for (int r = 0; ok && r < ro; ++r) {
                        const int s = r % kStages;
                        ok = wait(&sm.bar.w_full[s], (r / kStages) & 1) &&
                             (r < 2 || wait(&sm.bar.r_free[r & 1], ((r >> 1) - 1) & 1));
                        if (!ok) break;
                        ptx::tc_fence_after();
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int kk = 0; kk < kD / 16; ++kk)
                                ptx::mma_bf16(tmem + (r & 1) * 128, q_desc + kstep(kk),
                                              mn_desc + ((s * kTileBytes + kk * 2048) >> 4), idesc_route, kk > 0);
                            ptx::mma_commit(&sm.bar.empty[s]);
                            ptx::mma_commit(&sm.bar.r_full[r & 1]);
                        }
                        __syncwarp();
                    }
                    ok = ok && wait(&sm.bar.qr_ready, 0);
                    // (the loop by one lane: warp-wide waits between two half tiles leave the tensor cores idle)
                    if (ok && ptx::elect_one()) {
                        ptx::tc_fence_after();
                        for (int u = 0; u < n_sub; ++u) {
                            const int t = u >> 1, s = (t + ro) % kStages, sb = u % kSub;
                            if (!wait.one(C::kFp16 ? &sm.bar.v_full[t % kStages] : &sm.bar.full[t % kStages],
                                          (t / kStages) & 1))
                                break;
                            // the output MMAs of half tile u - kSub have read this buffer's weights
                            if (u >= kSub && !wait.one(&sm.bar.s_free[(u - kSub) & 3], ((u - kSub) >> 2) & 1)) break;
                            ptx::tc_fence_after();
                            const uint64_t b0 = k_desc + ((s * kTileBytes + (u & 1) * kBS * 128) >> 4);
                            // (the small terms first: the tensor core's adds truncate the sum)
                            if constexpr (C::kFp16)
#pragma unroll
                                for (int kk = 0; kk < kD / 16; ++kk)
                                    ptx::mma_bf16(tmem + sb * C::kBuf, q_desc + kstep(kk), b0 + kstep(kk), idesc_qk,
                                                  kk > 0);
#pragma unroll
                            for (int i = C::kQTerms - 1; i >= 0; --i)
#pragma unroll
                                for (int kk = 0; kk < kD / 16; ++kk)
                                    ptx::mma_bf16_ts(tmem + sb * C::kBuf, tmem + kColQ + 64 * i + kk * 8,
                                                     b0 + kstep(kk), idesc_qk,
                                                     C::kFp16 || i < C::kQTerms - 1 || kk > 0);
                            ptx::mma_commit(&sm.bar.s_full[u & 3]);
                        }
                    }
                } else if (ptx::elect_one()) {
                    // O += P . V (Half: the group's); at a fold O starts over (its old value has been read by then)
                    for (int u = 0; u < n_sub; ++u) {
                        const int s = ((u >> 1) + ro) % kStages, sb = u % kSub;
                        if (!wait.one(&sm.bar.p_full[u & 3], (u >> 2) & 1)) break;
                        if (!C::kFp16 && u && u % kFoldSub == 0 && !wait.one(&sm.bar.o_free, (u / kFoldSub - 1) & 1))
                            break;
                        ptx::tc_fence_after();
                        const uint64_t b0 = mn_desc + ((s * kTileBytes + (u & 1) * kBS * 128) >> 4);
                        const bool more = C::kFp16 ? u >= kGroups : u % kFoldSub != 0;
                        const uint32_t o = tmem + kColO + (C::kFp16 ? (u & 1) * kD : 0);
#pragma unroll
                        for (int kk = 0; kk < C::kPTerms * kBS / 16; ++kk)
                            ptx::mma_bf16_ts(o, tmem + sb * C::kBuf + kk * 8,
                                             b0 + (((kk & 3) * 2048) >> 4), idesc_pv, (more || kk > 0) ? 1u : 0u);
                        ptx::mma_commit(&sm.bar.s_free[u & 3]);
                        if ((u & 1) || u == n_sub - 1) ptx::mma_commit(&sm.bar.empty[s]);
                    }
                }
                __syncwarp();
                // every MMA this warp issued completes before the segment ends
                uint64_t *drain = warp == kMmaWarp ? &sm.bar.drain : &sm.bar.drain2;
                if (ptx::elect_one()) ptx::mma_commit(drain);
                __syncwarp();
                const uint64_t t0 = ptx::globaltimer();
                while (!ptx::mbar_try_wait(drain, 0) && ptx::globaltimer() - t0 < kTimeoutNs) {
                }
            } else if (C::kFp16 && warp >= kHelpWarp) {
                // ----------------------------------------------------------- tiles to fp16 ----
                // Thread = (row, 64 dims) of both half tiles, in place, ahead of the score MMAs. The lanes start at
                // different 16-byte chunks so that a warp's accesses spread over all banks.
                const int r = (warp - kHelpWarp) * 32 + lane;
                for (int t = 0; t < n_tiles; ++t) {
                    const int st = (t + ro) % kStages;
                    if (!wait(&sm.bar.full[t % kStages], (t / kStages) & 1)) break;
                    const uint32_t v_s = ptx::smem_addr(sm.tiles[st]) + (r >> 6) * kHalfBytes + (r & 63) * 128;
                    const int t0 = (tile0 + t) * kBN;
                    uint32_t v[2][32];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            ld_shared_v4(v_s + j * kBS * 128 + ((c + lane) & 7) * 16, v[j] + 4 * c);
                    if (t0 + kBN > base) {
                        // Rows that not every draft sees must not reach the others through 0 * NaN: a row past the
                        // sequence's end, or a drafted one without a finite fp16 form, becomes zeros; a draft
                        // that sees such a row gets NaN by its bit in `over`.
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int vt = t0 + j * kBS + (r & 63);
                            bool over = false;
#pragma unroll
                            for (int e = 0; e < 32; ++e) over |= past_fp16(v[j][e]);
                            if (over && vt >= base && vt < L)
                                atomicOr(&sm.over[(vt - base) >> 5], 1u << ((vt - base) & 31));
                            if (vt >= L || (over && vt >= base))
#pragma unroll
                                for (int e = 0; e < 32; ++e) v[j][e] = 0u;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
#pragma unroll
                            for (int e = 4 * c; e < 4 * c + 4; ++e)
                                v[j][e] = pack_f16(__uint_as_float(v[j][e] << 16),
                                                   __uint_as_float(v[j][e] & 0xffff0000u));
                            st_shared_v4(v_s + j * kBS * 128 + ((c + lane) & 7) * 16, v[j][4 * c], v[j][4 * c + 1],
                                         v[j][4 * c + 2], v[j][4 * c + 3]);
                        }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sm.bar.v_full[t % kStages]);
                }
            } else if (!C::kFp16 && warp >= kHelpWarp) {
                // ------------------------------------------------------------- O to the sum ----
                // Every kFoldSub half tiles O, at its reference, joins the fp32 sum and the output MMAs start
                // over as soon as it has been read (thread = row = TMEM lane).
                const int qd = warp & 3, r = qd * 32 + lane;
                const uint32_t lane_base = (uint32_t)(qd * 32) << 16;
                float4 *const row = reinterpret_cast<float4 *>(sm.sum) + r * 32;
                float m_sum = -INFINITY;                     // the sum's reference
                bool okf = qd < (k.blk.rows * hp + 31) >> 5; // (a quarter without rows rests)
                for (int u = kFoldSub; okf && u < n_sub; u += kFoldSub) {
                    okf = wait(&sm.bar.s_free[(u - 1) & 3], ((u - 1) >> 2) & 1) &&
                          wait(&sm.bar.turn[qd][(u - 1) % kTreeTurns], ((u - 1) / kTreeTurns) & 1);
                    if (!okf) break;
                    ptx::tc_fence_after();
                    const float m = sm.mref[(u - 1) & 3][r];
                    const float f = m_sum == -INFINITY ? 0.f : ptx::ex2(m_sum - m);
                    const bool had = u > kFoldSub;
                    m_sum = m;
#pragma unroll
                    for (int c = 0; c < kD; c += 32) {
                        uint32_t o[32];
                        ptx::tmem_ld32(tmem + kColO + c + lane_base, o);
                        ptx::tmem_wait_ld();
                        ptx::reg_fence(o);
                        if (c == kD - 32) {
                            ptx::tc_fence_before();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(&sm.bar.o_free);
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            float4 &w = row[(c / 4 + e) ^ lane];
                            float4 y = had ? w : make_float4(0.f, 0.f, 0.f, 0.f);
                            y.x = fmaf(y.x, f, __uint_as_float(o[4 * e]));
                            y.y = fmaf(y.y, f, __uint_as_float(o[4 * e + 1]));
                            y.z = fmaf(y.z, f, __uint_as_float(o[4 * e + 2]));
                            y.w = fmaf(y.w, f, __uint_as_float(o[4 * e + 3]));
                            w = y;
                        }
                    }
                }
                if (okf && n_sub > kFoldSub) {
                    sm.fref[r] = m_sum;
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sm.bar.sum_full);
                }
            }
            if (!end(k)) break;
        }
    } else {
        ptx::regs_inc<kSoftmaxRegs>();
        for (int si = 0;; ++si) {
            const Part k = begin(si);
            const uint32_t tmem = sm.tmem_base;
            const bool has_drafts = k.has_drafts, whole = k.whole;
            const TreeSegment &sg = k.sg;
            const int m0 = k.blk.m0, rows = k.blk.rows, h = k.blk.h, hn = k.blk.hn;
            const int q0 = sg.q0, L = sg.L, tile0 = sg.tile0;
            const int base = L - sg.n, n_sub = k.n_sub, ro = k.ro;
            // ----------------------------------------------------- softmax, epilogue ----
            if (tid == 0 && k.more) sm.seg[(si + 1) & 1] = next_segment(a, sg);
            constexpr int kCols = kD / kGroups;             // columns of the query and of O per group
            const int qd = warp & 3, grp = warp >> 2;    // lane quarter, group
            const int quarters = (rows * hp + 31) >> 5;  // with rows of the block
            if (qd >= quarters) {
                (void)ptx::bar_and(kBarCompute, 32 * kComputeWarps, true);
                if (!end(k)) break;
                continue;
            }
            const int r = qd * 32 + lane;                // row = TMEM lane
            const int ri = r / hp, hh = r - ri * hp;     // draft and head within the block
            const bool live = ri < rows && hh < hn;
            const int c0 = grp * kCols;
            const uint32_t own_o = tmem + kColO + (C::kFp16 ? grp * kD : 0);
            const uint32_t lane_base = (uint32_t)(qd * 32) << 16;
            const float sl2 = geo.scale * kLog2e;
            auto row_id = [&] { return (size_t)(q0 + m0 + ri) * geo.Hq + h + hh; };   // of q and out
            bool ok = true;

            // Routed query row, this group's columns, times scale * log2 e, as operand terms
            uint32_t q[kCols];
            if (ro == 0) {
                // the composed query, as it is
                const uint4 *src = reinterpret_cast<const uint4 *>(a.q + row_id() * kD + c0);
#pragma unroll
                for (int c = 0; c < kCols / 8; ++c) {
                    const uint4 v = live ? src[c] : make_uint4(0u, 0u, 0u, 0u);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        q[8 * c + 2 * e] = w[e] << 16;
                        q[8 * c + 2 * e + 1] = w[e] & 0xffff0000u;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < kCols; ++e) q[e] = 0u;
                for (int i = 0; ok && i < ro; ++i) {
                    ok = wait(&sm.bar.r_full[i & 1], (i >> 1) & 1);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    const bool mine = ro == 1 || hh == i;
#pragma unroll
                    for (int c = 0; c < kCols; c += 32) {
                        uint32_t u[32];
                        ptx::tmem_ld32(tmem + (i & 1) * 128 + c0 + c + lane_base, u);
                        ptx::tmem_wait_ld();
                        ptx::reg_fence(u);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (mine) q[c + e] = u[e];
                    }
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sm.bar.r_free[i & 1]);
                }
            }
            if (ok) {
#pragma unroll
                for (int e = 0; e < kCols; ++e) q[e] = __float_as_uint(__uint_as_float(q[e]) * sl2);
#pragma unroll
                for (int t = 0; t < C::kQTerms; ++t)
#pragma unroll
                    for (int c = 0; c < kCols / 2; c += 16) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            uint32_t &x0 = q[2 * (c + e)], &x1 = q[2 * (c + e) + 1];
                            w[e] = C::kFp16 ? take_term_f16(x0, x1) : take_term(x0, x1);
                        }
                        ptx::tmem_st16(tmem + kColQ + 64 * t + c0 / 2 + c + lane_base, w);
                    }
                if constexpr (C::kFp16) {
                    // what is left, as a second fp16 term, takes the query block's place (which the routing has read)
                    const uint32_t row = ptx::smem_addr(sm.q) + grp * kHalfBytes + r * 128;
#pragma unroll
                    for (int c = 0; c < kCols / 8; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = pack_f16(__uint_as_float(q[8 * c + 2 * e]), __uint_as_float(q[8 * c + 2 * e + 1]));
                        st_shared_v4(row + ((c ^ (r & 7)) << 4), w[0], w[1], w[2], w[3]);
                    }
                    ptx::fence_proxy_async_smem();
                }
            }
            if (ok) {
                ptx::tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sm.bar.qr_ready);
            }

            // the drafts that this row's draft sees: itself and its ancestors (walked where they are needed,
            // in up to three half tiles of a unit)
            auto ancestors = [&](uint64_t &lo, uint64_t &hi) {
                lo = hi = 0;
                for (int j = m0 + min(ri, rows - 1); j >= 0; j = sm.parent[j]) {
                    if (j < 64) lo |= 1ull << j;
                    else hi |= 1ull << (j - 64);
                }
            };

            float m_used = -INFINITY;  // the reference of this thread's share of the row sum
            // The sum of this thread's half tiles' sums, and (Full) what its roundings lost: one number for all
            // weights loses the small ones (fp32 error of 64615 tokens with outliers in two parts 1e-5, 7e-7 so).
            float l_sum = 0.f, l_err = 0.f;
            bool okl = ok;
            for (int u = grp; okl && u < n_sub; u += kGroups) {
                const int t0 = tile0 * kBN + u * kBS, sb = u % kSub;
                const uint32_t sbuf = tmem + (uint32_t)sb * C::kBuf + lane_base;   // S, then P
                const bool drafts_here = t0 + kBS > base;
                okl = wait(&sm.bar.s_full[u & 3], (u >> 2) & 1);
                if (!okl) break;
                ptx::tc_fence_after();
                if constexpr (!C::kFp16) {
                    // Rows that not every draft sees must not reach the others through 0 * NaN: a row past the
                    // sequence's end, or a drafted one that is not finite, becomes zeros for the output MMAs; a
                    // draft that sees such a row gets NaN by its bit in `over` (its score may be -inf).
                    const int ring = (u >> 1) + ro;
                    if (drafts_here) {
                        okl = wait(&sm.bar.full[(u >> 1) % kStages], ((u >> 1) / kStages) & 1);
                        if (!okl) break;
                    }
                    // thread = (cache row, 64 dims)
#pragma unroll 1
                    for (int i = r; drafts_here && i < kBM; i += 32 * quarters) {
                        const int vt = t0 + (i & 63);
                        if (vt < base) continue;
                        const uint32_t v_s = ptx::smem_addr(sm.tiles[ring % kStages]) + (i >> 6) * kHalfBytes +
                                             ((u & 1) * kBS + (i & 63)) * 128;
                        bool bad = false;
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            uint32_t v[4];
                            ld_shared_v4(v_s + ((c + lane) & 7) * 16, v);
#pragma unroll
                            for (int e = 0; e < 4; ++e) bad |= not_finite(v[e]);
                        }
                        if (bad && vt < L) atomicOr(&sm.over[(vt - base) >> 5], 1u << ((vt - base) & 31));
                        if (bad || vt >= L)
#pragma unroll
                            for (int c = 0; c < 8; ++c) st_shared_v4(v_s + c * 16, 0u, 0u, 0u, 0u);
                    }
                }
                uint32_t s0[32], s1[32];
                ptx::tmem_ld32(sbuf, s0);
                ptx::tmem_ld32(sbuf + 32, s1);
                ptx::tmem_wait_ld();
                ptx::reg_fence(s0);
                ptx::reg_fence(s1);
                if (drafts_here) {
                    uint64_t lo, hi;
                    okl = wait(&sm.bar.par_ready, 0);
                    if (!okl) break;
                    ancestors(lo, hi);
                    const uint64_t see = window64(lo, hi, t0 - base);
                    const uint32_t v0 = (uint32_t)see, v1 = (uint32_t)(see >> 32);
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        if (!(v0 & (1u << e))) s0[e] = 0xff800000u;
                        if (!(v1 & (1u << e))) s1[e] = 0xff800000u;
                    }
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    mx[0] = max3(mx[0], __uint_as_float(s0[e]), __uint_as_float(s0[e + 1]));
                    mx[1] = max3(mx[1], __uint_as_float(s0[e + 2]), __uint_as_float(s0[e + 3]));
                    mx[2] = max3(mx[2], __uint_as_float(s1[e]), __uint_as_float(s1[e + 1]));
                    mx[3] = max3(mx[3], __uint_as_float(s1[e + 2]), __uint_as_float(s1[e + 3]));
                }
                float mt = max3(mx[0], mx[1], fmaxf(mx[2], mx[3]));
                float m_ref = -INFINITY;
                if constexpr (C::kFp16) {
                    m_ref = m_used;                      // the group's own
                } else if (u == 0) {
                    // the row's first reference is the maximum of its first two half tiles
                    if (n_sub > 1) {
                        okl = wait(&sm.bar.first[qd], 0);
                        if (!okl) break;
                        mt = fmaxf(mt, sm.lsum[1][r]);
                    }
                } else {
                    if (u == 1) {
                        sm.lsum[1][r] = mt;
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(&sm.bar.first[qd]);
                    }
                    okl = wait(&sm.bar.turn[qd][(u - 1) % kTreeTurns], ((u - 1) / kTreeTurns) & 1);
                    if (!okl) break;
                    m_ref = sm.mref[(u - 1) & 3][r];
                }
                const float m_new = fmaxf(m_ref, mt);
                const bool moves = __any_sync(0xffffffffu, m_new > m_ref + kRescaleLog2);
                // the last half tile that O holds (Full: O starts over at even half tiles)
                const int before = C::kFp16 ? u - kGroups : u % kFoldSub ? u - 1 : -1;
                // a new reference when the maximum grew by more than 2^14 (or is the first finite)
                if (moves) {
                    if (before >= 0) {
                        okl = wait(&sm.bar.s_free[before & 3], (before >> 2) & 1);
                        if (!okl) break;
                        ptx::tc_fence_after();
                        const float f =
                            (m_new == -INFINITY || m_ref == -INFINITY) ? 0.f : ptx::ex2(m_ref - m_new);
#pragma unroll
                        for (int c = 0; c < 128; c += 32) {
                            uint32_t o[32];
                            ptx::tmem_ld32(own_o + c + lane_base, o);
                            ptx::tmem_wait_ld();
                            ptx::reg_fence(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            ptx::tmem_st32(own_o + c + lane_base, o);
                        }
                        ptx::tmem_wait_st();
                    }
                    m_ref = m_new;
                }
                if constexpr (!C::kFp16) {
                    sm.mref[u & 3][r] = m_ref;
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sm.bar.turn[qd][u % kTreeTurns]);
                }
                // the group's sums move to this reference
                if (__any_sync(0xffffffffu, m_ref != m_used)) {
                    const float f = m_used == -INFINITY ? 0.f : ptx::ex2(m_used - m_ref);
                    l_sum *= f;
                    l_err *= f;
                    m_used = m_ref;
                }
                // the row's 64 weights -> 32 packed columns per term (the output MMAs of u - kSub, the
                // last reader of P there, finished before these scores were written)
                const float mr = m_ref == -INFINITY ? 0.f : m_ref;
                float2 la = make_float2(0.f, 0.f), lb = make_float2(0.f, 0.f);
                auto weights = [&](uint32_t(&s)[32]) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float2 d = sub2(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])),
                                              make_float2(mr, mr));
                        const float2 pe = make_float2(ptx::ex2(d.x), ptx::ex2(d.y));
                        if (e & 1) lb = add2(lb, pe); else la = add2(la, pe);
                        if constexpr (C::kFp16) {
                            s[e] = pack_f16(pe.x, pe.y);
                        } else {
                            s[2 * e] = __float_as_uint(pe.x);
                            s[2 * e + 1] = __float_as_uint(pe.y);
                        }
                    }
                };
                weights(s0);
                weights(s1);
                const float x = (la.x + la.y) + (lb.x + lb.y), t = l_sum + x, y = t - l_sum;
                if constexpr (!C::kFp16) l_err += (l_sum - (t - y)) + (x - y);
                l_sum = t;
                if constexpr (C::kFp16) {
                    ptx::tmem_st16(sbuf, s0);
                    ptx::tmem_st16(sbuf + 16, s1);
                } else {
#pragma unroll
                    for (int t = 0; t < C::kPTerms; ++t) {
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            w[e] = take_term(s0[2 * e], s0[2 * e + 1]);
                            w[16 + e] = take_term(s1[2 * e], s1[2 * e + 1]);
                        }
                        ptx::tmem_st32(sbuf + 32 * t, w);
                    }
                }
                ptx::tmem_wait_st();
                ptx::tc_fence_before();
                // rows zeroed here (generic-proxy stores) are read next by the output MMAs
                if (!C::kFp16 && drafts_here) ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sm.bar.p_full[u & 3]);
            }

            // Epilogue: out = O / l, or the part's state (m, l, O). Full: l is the groups' shares at the
            // reference of the last half tile; Half: the groups' states are joined as parts are. This
            // group's output dims.
            const int last = n_sub - 1, lg = last % kGroups;
            if (!C::kFp16 && okl && lg != grp) okl = wait(&sm.bar.turn[qd][last % kTreeTurns], (last / kTreeTurns) & 1);
            // (all of the last commits land before the barriers are set up anew)
            bool oke = okl;
            if (!C::kFp16 && oke && last >= kFoldSub) oke = wait(&sm.bar.sum_full, 0);
            for (int u = last; oke && u >= 0 && u > last - 3; --u) oke = wait(&sm.bar.s_free[u & 3], (u >> 2) & 1);
            float l = l_sum + l_err;
            float m_fin = 0.f;
            if constexpr (C::kFp16) {
                sm.mref[grp][r] = m_used;
            } else {
                m_fin = sm.mref[last & 3][r];
                if (oke && lg != grp) l = m_used == -INFINITY ? 0.f : l * ptx::ex2(m_used - m_fin);
            }
            sm.lsum[grp][r] = l;
            const bool okp = ptx::bar_and(kBarCompute, 32 * kComputeWarps, oke);
            if (okp) {
                ptx::tc_fence_after();
                float w0 = 1.f, w1 = 1.f;                    // of the groups' O
                if constexpr (C::kFp16) {
                    const float m0 = sm.mref[0][r], m1 = sm.mref[1][r];
                    m_fin = fmaxf(m0, m1);
                    // (a group that saw nothing has m = -inf, l = 0 and O = 0, or no O at all)
                    w0 = m0 == -INFINITY ? 0.f : ptx::ex2(m0 - m_fin);
                    w1 = m1 == -INFINITY ? 0.f : ptx::ex2(m1 - m_fin);
                }
                float lt = w0 * sm.lsum[0][r] + w1 * sm.lsum[1][r];
                if (has_drafts) {
                    const uint64_t o0 = sm.over[0] | (uint64_t)sm.over[1] << 32;
                    const uint64_t o1 = sm.over[2] | (uint64_t)sm.over[3] << 32;
                    if (o0 | o1) {
                        uint64_t lo, hi;
                        (void)wait(&sm.bar.par_ready, 0);
                        ancestors(lo, hi);
                        if ((lo & o0) | (hi & o1)) lt = NAN;
                    }
                }
                const float f = !whole ? 1.f : lt == 0.f ? 0.f : 1.f / lt;
                const bool folded = !C::kFp16 && last >= kFoldSub;
                float fs = 0.f;                              // of the sum
                if (folded) fs = sm.fref[r] == -INFINITY ? 0.f : ptx::ex2(sm.fref[r] - m_fin);
                // a part's state: [32 chunks of 4 dims][128 rows] float4, then [128 rows] {m, l}
                uint8_t *state = a.states + (size_t)(2 * blockIdx.x + (si > 0)) * kTreeStateBytes;
                float nf = live ? lt * 0.f : 0.f;            // x * 0 is NaN exactly when x is not finite
#pragma unroll 1
                for (int c4 = 0; c4 < kCols / 32; ++c4) {
                    uint32_t u[32];
                    ptx::tmem_ld32(tmem + kColO + c0 + c4 * 32 + lane_base, u);
                    ptx::tmem_wait_ld();
                    ptx::reg_fence(u);
                    if constexpr (C::kFp16) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) * w0);
                        if (n_sub > 1) {
                            uint32_t v[32];
                            ptx::tmem_ld32(tmem + kColO + kD + c0 + c4 * 32 + lane_base, v);
                            ptx::tmem_wait_ld();
                            ptx::reg_fence(v);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                u[e] = __float_as_uint(fmaf(__uint_as_float(v[e]), w1, __uint_as_float(u[e])));
                        }
                    }
                    if (folded) {
                        const float4 *row = reinterpret_cast<const float4 *>(sm.sum) + r * 32;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float4 y = row[(c0 / 4 + c4 * 8 + e) ^ lane];
                            u[4 * e] = __float_as_uint(fmaf(y.x, fs, __uint_as_float(u[4 * e])));
                            u[4 * e + 1] = __float_as_uint(fmaf(y.y, fs, __uint_as_float(u[4 * e + 1])));
                            u[4 * e + 2] = __float_as_uint(fmaf(y.z, fs, __uint_as_float(u[4 * e + 2])));
                            u[4 * e + 3] = __float_as_uint(fmaf(y.w, fs, __uint_as_float(u[4 * e + 3])));
                        }
                    }
                    if (live) {
                        if (C::kFp16)
#pragma unroll
                            for (int e = 0; e < 32; ++e) nf = fmaf(__uint_as_float(u[e]), 0.f, nf);
                        float4 *o = whole ? reinterpret_cast<float4 *>(static_cast<float *>(a.out) + row_id() * kD) +
                                                c0 / 4 + c4 * 8
                                          : reinterpret_cast<float4 *>(state) + (c0 / 4 + c4 * 8) * kBM + r;
                        if (!whole || a.out_dtype == KL_FP32) {
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                o[whole ? c : c * kBM] =
                                    make_float4(__uint_as_float(u[4 * c]) * f, __uint_as_float(u[4 * c + 1]) * f,
                                                __uint_as_float(u[4 * c + 2]) * f, __uint_as_float(u[4 * c + 3]) * f);
                        } else {
                            uint4 *ob = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) +
                                                                  row_id() * kD + c0 + c4 * 32);
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                uint32_t w[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    w[e] = pack2(__uint_as_float(u[8 * c + 2 * e]) * f,
                                                 __uint_as_float(u[8 * c + 2 * e + 1]) * f);
                                ob[c] = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                }
                if (!whole && grp == 0 && live)
                    reinterpret_cast<float2 *>(state + kBM * kD * 4)[r] = make_float2(m_fin, lt);
                if (C::kFp16 && __any_sync(0xffffffffu, nf != nf) && lane == 0) raise_flag(a.err, KL_FLAG_RANGE);
            }
            if (!end(k)) break;
        }
    }

    if (warp == kMmaWarp) ptx::tmem_dealloc(sm.tmem_base, kTmemCols);
}

// Merge of the parts of the units that lie in several runs: out = sum_s w_s O_s / sum_s w_s l_s with w_s =
// 2^(m_s - M) and M the largest m_s of a part with l_s > 0. CTA (c, y): the unit that run c enters first
// inside, dims 8 y .. + 7; thread = row and 4 dims, kMergeAhead parts in flight against a running M.
constexpr int kMergeThreads = 2 * kBM, kMergeAhead = 8;

__global__ void __launch_bounds__(kMergeThreads) tree_merge_kernel(const TreeArgs a) {
    __shared__ const uint8_t *part[kTreeMaxRuns];
    __shared__ int parts;
    grid_dep_wait();
    grid_dep_launch();
    const int c = blockIdx.x + 1, tid = threadIdx.x;
    const TreeMerge t = a.merge[c];
    if (t.rows == 0) return;
    if (tid < 32) {
        // The runs from c - 1 on that hold some of the unit; a run's first state where it starts inside it.
        auto cut = [&](int run) { return cut_tile(a.start, run_start(t.share, run) - t.unit0, t.tiles, t.step); };
        int n = 0;
        for (int r0 = c - 1; r0 <= t.last; r0 += 32) {
            const int run = r0 + tid;
            const bool some = run <= t.last && cut(run) < cut(run + 1);
            const unsigned all = __ballot_sync(0xffffffffu, some);
            if (some)
                part[n + __popc(all & ((1u << tid) - 1))] =
                    a.states + (size_t)(2 * run + (run_start(t.share, run) < t.unit0)) * kTreeStateBytes;
            n += __popc(all);
        }
        if (tid == 0) parts = n;
    }
    __syncthreads();
    const int r = tid % kBM, chunk = blockIdx.y * 2 + tid / kBM;
    const int ri = r / a.hp, hh = r - ri * a.hp;
    if (ri >= t.rows || hh >= t.hn) return;
    float M = -INFINITY, z = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < parts; i += kMergeAhead) {
        float2 ml[kMergeAhead];
        float4 o[kMergeAhead];
        float top = M;
#pragma unroll
        for (int e = 0; e < kMergeAhead; ++e) {
            ml[e] = make_float2(-INFINITY, 0.f);
            o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i + e < parts) {
                ml[e] = __ldcg(reinterpret_cast<const float2 *>(part[i + e] + kBM * kD * 4) + r);
                o[e] = __ldcg(reinterpret_cast<const float4 *>(part[i + e]) + chunk * kBM + r);
            }
        }
#pragma unroll
        for (int e = 0; e < kMergeAhead; ++e)
            if (ml[e].y != 0.f) top = fmaxf(top, ml[e].x);           // (l = 0: the row sees nothing there)
        const float f = M == -INFINITY ? 0.f : ptx::ex2(M - top);
        M = top;
        z *= f;
        acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
#pragma unroll
        for (int e = 0; e < kMergeAhead; ++e) {
            const float w = ml[e].y == 0.f ? 0.f : ptx::ex2(ml[e].x - M);
            z = fmaf(w, ml[e].y, z);
            acc.x = fmaf(w, o[e].x, acc.x);
            acc.y = fmaf(w, o[e].y, acc.y);
            acc.z = fmaf(w, o[e].z, acc.z);
            acc.w = fmaf(w, o[e].w, acc.w);
        }
    }
    const float inv = z == 0.f ? 0.f : 1.f / z;
    const size_t at = ((size_t)(t.row0 + ri) * a.geo.Hq + t.h + hh) * kD + 4 * chunk;
    if (a.out_dtype == KL_FP32)
        *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) =
            make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    else
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + at) =
            make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
}

// ------------------------------------------------------------------------ host side ------

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000,
                                             cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }
    return fn;
}

// bf16 tensor map of `rank` dimensions, innermost 128 elements, box 64 x ..., 128-byte swizzle.
bool encode(CUtensorMap *map, const void *base, int rank, const cuuint64_t *dims,
            const cuuint64_t *strides, const cuuint32_t *box) {
    auto fn = encode_fn();
    if (!fn) return false;
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(base), dims, strides,
              box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_tree_tc(const TreeArgs &a) {
    const Geometry &g = a.geo;
    CUtensorMap vmap, wmap, qmap;
    {
        // cache as [num_pages * Hkv * P rows][128], one box = one page of one head (64 dims)
        const cuuint64_t dims[2] = {kD, (cuuint64_t)g.num_pages * g.Hkv * g.P};
        const cuuint64_t strides[1] = {kD * 2};
        const cuuint32_t box[2] = {64, (cuuint32_t)g.P};
        if (!encode(&vmap, a.v_cache, 2, dims, strides, box)) return cudaErrorInvalidValue;
    }
    wmap = qmap = vmap;                 // (not read with a composed query)
    if (a.w_r) {
        // W^R as [Hw * 128 k rows][128 j], one box = a 64-column half of one matrix
        const cuuint64_t hw = g.wr_per_qh ? (cuuint64_t)g.Hq : (cuuint64_t)g.Hkv;
        const cuuint64_t dims[2] = {kD, hw * kD};
        const cuuint64_t strides[1] = {kD * 2};
        const cuuint32_t box[2] = {64, kD};
        if (!encode(&wmap, a.w_r, 2, dims, strides, box)) return cudaErrorInvalidValue;
        // q as [total_q][Hq][128], one box = rpb consecutive drafts of hp heads (64 dims); rows past
        // total_q and heads past Hq read as zeros
        const cuuint64_t qdims[3] = {kD, (cuuint64_t)g.Hq, (cuuint64_t)a.total_q};
        const cuuint64_t qstrides[2] = {kD * 2, (cuuint64_t)g.Hq * kD * 2};
        const cuuint32_t qbox[3] = {64, (cuuint32_t)a.hp, (cuuint32_t)a.rpb};
        if (!encode(&qmap, a.q, 3, qdims, qstrides, qbox)) return cudaErrorInvalidValue;
    }
    const bool full = a.out_dtype == KL_FP32;
    const bool exact = a.wait_ns < kExactWaitNs;
    const auto kernel = full ? exact ? tree_tc_kernel<Full, true> : tree_tc_kernel<Full, false>
                             : exact ? tree_tc_kernel<Half, true> : tree_tc_kernel<Half, false>;
    const size_t smem = (full ? sizeof(TreeSmem<Full>) : sizeof(TreeSmem<Half>)) + 1024;
    static PerDeviceOnce once[4];
    cudaError_t e = once[2 * full + exact].run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.ctas);
    cfg.blockDim = dim3(full ? Warps<Full>::kThreads : Warps<Half>::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = a.stream;
    const OverlapAttr overlap(cfg);
    e = cudaLaunchKernelEx(&cfg, kernel, vmap, wmap, qmap, a);
    // (units of up to a.whole tiles are not cut)
    const int64_t most_tiles = ((int64_t)g.max_pages * g.P + kBN - 1) / kBN;
    if (e != cudaSuccess || a.ctas == 1 || a.num_splits == 1 || (a.num_splits == 0 && most_tiles <= a.whole))
        return e;
    cfg.gridDim = dim3((unsigned)a.ctas - 1, kD / 8);
    cfg.blockDim = dim3(kMergeThreads);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, tree_merge_kernel, a);
}

}  // namespace kl
