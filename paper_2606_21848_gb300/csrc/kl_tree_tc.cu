// Attention of a tree of drafted tokens over the paged Value-Only Cache (the verification step of
// speculative decoding), for sm_103a; head_dim 128.
//
// Sequence b holds L cached rows, the last n of them drafted tokens that form a forest: draft i's parent
// is an earlier draft or the last committed token. Draft i sees the committed tokens t < L - n, itself
// and its ancestors. With q_r = q W^R (Section 2.2) and the decode formula of Section 3,
//   s_t = scale <q_r, v_t>,  out = sum_t softmax(s)_t v_t   over the tokens that the draft sees.
// n = 1 is the decode step, a chain of drafts the causal chunk.
//
// The G heads of a value head's group times the n drafts read the same cache rows. A block holds up to
// 128 of these (draft, head) rows; a block's cache tiles are cut over S CTAs, whose states are merged by
// the CTA that finishes last. One CTA per SM:
//
//   routing  Q_r = Q . W^R                             M = 128 rows, N = 128, K = 128
//   scores   S   = Q_hi . V_t^T + Q_lo . V_t^T         M = 128 rows, N = 64 tokens, K = 2 x 128
//   output   O  += P_hi . V_t + P_lo . V_t             M = 128 rows, N = 128 dims, K = 2 x 64
//
// Each cached tile V_t [128 tokens x 128 dims] arrives once by TMA (one box per page and 64 dims) and
// feeds both products from the same shared-memory copy, as the K-major B operand of the scores and the
// MN-major one of the output. Q and P are A operands in tensor memory (512 columns: 4 x 64 of scores,
// then weights; O 128; Q_hi | Q_lo 64 + 64). Both are pairs of bf16 operands, x = hi + lo (about 16
// significant bits), so that fp32 outputs are good to about 3e-6 of their size.
//
// The unit of the pipeline is a half tile of 64 tokens, four in flight, as in the prefill: thread = row
// = TMEM lane; two groups of four softmax warps take alternate half tiles and share each row's
// reference maximum, which moves only when a half tile's maximum passes it by more than 2^7.
//
// Roles (352 threads): warps 0-7 softmax and epilogue, warp 8 producer (TMA), warp 9 routing and score
// MMAs (owner of the tensor memory), warp 10 output MMAs. Every wait is bounded (about one second); a
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
constexpr int kBM = kTreeRows;                    // rows per CTA
constexpr int kBN = kTreeTile;                    // cache rows per tile
constexpr int kBS = 64;                           // cache rows per half tile
constexpr int kSub = 4;                           // half tiles in flight
constexpr int kStages = 5;
constexpr int kComputeWarps = 8;                  // two per TMEM lane quarter
constexpr int kProducerWarp = 8, kMmaWarp = 9, kPvWarp = 10;
constexpr int kThreads = 11 * 32;
constexpr uint32_t kTileBytes = kBN * kD * 2;     // 32 KiB
constexpr uint32_t kHalfBytes = kTileBytes / 2;   // one 64-dim half: 128 rows x 128 B
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0;                     // S of half tile u: 64 (u % 4) .. + 63, then its P
                                                  // (hi in the first 32, lo in the others); the
                                                  // routed queries first land in 0 .. 255
constexpr uint32_t kColO = 256;                   // O: columns 256 .. 383
constexpr uint32_t kColQ = 384;                   // Q_hi: 384 .. 447, Q_lo: 448 .. 511
constexpr uint32_t kLoCols = 64;                  // hi -> lo of the packed query
constexpr float kRescaleLog2 = 7.f;
constexpr uint64_t kTimeoutNs = kRowsTimeoutNs;
constexpr uint32_t kBarCompute = 1;   // named barrier of the compute warps (0 is __syncthreads)

struct __align__(1024) TreeSmem {
    uint8_t q[kBM * kD * 2];               // query block, K-major SW128: [64-dim half][128 rows][128 B]
    // Ring: the W^R matrices, then the cache tiles ([64-dim half][128 rows][128 B], SW128).
    uint8_t tiles[kStages][kTileBytes];
    uint64_t full[kStages], empty[kStages];
    uint64_t s_full[kSub], s_free[kSub], p_full[kSub];
    uint64_t turn[4][2];       // per lane quarter and parity: the references after a half tile
    uint64_t first[4];         // per lane quarter: the maxima of half tile 1 are in lsum[1]
    uint64_t r_full[2], r_free[2];   // routing results, alternating halves of the score columns
    uint64_t qr_ready, drain, drain2;
    float mref[2][kBM];        // the rows' references after the last half tile of each parity
    float lsum[2][kBM];        // the two groups' shares of the row sums, for the epilogue
    int32_t parent[KL_TREE_MAX_DRAFTS];
    uint32_t tmem_base;
    int is_last;
    int abort;
};
static_assert(sizeof(TreeSmem) + 1024 <= 227 * 1024, "one CTA per SM");

// The 64 bits off .. off + 63 of the 128-bit set (lo, hi), off in -63 .. 127; bits below 0 are ones.
__device__ __forceinline__ uint64_t window64(uint64_t lo, uint64_t hi, int off) {
    if (off < 0) return (lo << -off) | ((1ull << -off) - 1);
    if (off == 0) return lo;
    return off < 64 ? (lo >> off) | (hi << (64 - off)) : hi >> (off - 64);
}

__global__ void __launch_bounds__(kThreads, 1)
    tree_tc_kernel(const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap wmap,
                   const __grid_constant__ CUtensorMap qmap, const TreeArgs a) {
    extern __shared__ uint8_t smem_raw[];
    TreeSmem &sm = *reinterpret_cast<TreeSmem *>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const Geometry &geo = a.geo;
    const int blk = blockIdx.x % a.blocks, split = blockIdx.x / a.blocks;
    const int g = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    grid_dep_wait();
    const int q0 = a.cu_q[b], q1 = a.cu_q[b + 1];
    const int L = a.seq_lens[b];
    const int n = q1 - q0;
    if (q0 < 0 || n < 0 || q1 > a.total_q || n > a.max_q || L < n || L > geo.max_pages * geo.P) {
        if (tid == 0 && blockIdx.x == 0 && g == 0) raise_flag(a.err, KL_FLAG_BAD_LENGTH);
        return;
    }
    // The block: drafts m0 .. m0 + rows - 1, heads h .. h + hn - 1 of the group; row r of the 128 is
    // draft m0 + r / hp with head h + r % hp.
    const int hp = a.hp, rpb = a.rpb;
    const int nhg = (geo.G + hp - 1) / hp;       // blocks of heads
    const int m0 = (blk / nhg) * rpb;
    if (m0 >= n) return;
    const int rows = min(rpb, n - m0);
    const int h = g * geo.G + (blk % nhg) * hp;
    const int hn = min(hp, (g + 1) * geo.G - h);
    // This CTA's cache tiles: tile0 .. tile0 + n_tiles - 1, as half tiles 0 .. n_sub - 1 from there.
    const int base = L - n;                      // committed tokens
    const int seen = base + m0 + rows;           // no row sees a token from here on
    const int share = a.chunk / kBN;
    const int all_tiles = (seen + kBN - 1) / kBN;
    const int runs = (all_tiles + share - 1) / share;
    if (split >= runs) return;
    const int tile0 = split * share;
    const int n_tiles = min(share, all_tiles - tile0);
    const int n_sub = min(2 * n_tiles, (seen + kBS - 1) / kBS - 2 * tile0);
    const bool has_drafts = (tile0 + n_tiles) * kBN > base;
    // ring positions of W^R matrices: one, one per head of the block, or none (composed query)
    const int ro = a.w_r ? (geo.wr_per_qh ? hn : 1) : 0;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(&sm.full[s], 1);
            ptx::mbar_init(&sm.empty[s], 1);
        }
        // One completion per half tile u of its buffer u % kSub on s_full (its scores), p_full (its
        // weights) and s_free (its output MMAs are done), and per lane quarter on turn[.][u % 2].
        for (int i = 0; i < kSub; ++i) {
            ptx::mbar_init(&sm.s_full[i], 1);
            ptx::mbar_init(&sm.s_free[i], 1);
            ptx::mbar_init(&sm.p_full[i], kComputeWarps / 2);
        }
        for (int q = 0; q < 4; ++q) {
            for (int i = 0; i < 2; ++i) ptx::mbar_init(&sm.turn[q][i], 1);
            ptx::mbar_init(&sm.first[q], 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&sm.r_full[i], 1);
            ptx::mbar_init(&sm.r_free[i], kComputeWarps);
        }
        ptx::mbar_init(&sm.qr_ready, kComputeWarps);
        ptx::mbar_init(&sm.drain, 1);
        ptx::mbar_init(&sm.drain2, 1);
        sm.abort = 0;
        ptx::fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        ptx::tmem_alloc(&sm.tmem_base, kTmemCols);
        ptx::tmem_relinquish();
    }
    // (a parent that is not an earlier draft or -1 counts as -1)
    if (has_drafts && tid < n) {
        const int p = a.parents[q0 + tid];
        const bool fine = p >= -1 && p < tid;
        if (!fine) raise_flag(a.err, KL_FLAG_BAD_TREE);
        sm.parent[tid] = fine ? p : -1;
    }
    // rows of the query block that its box does not fill
    if (ro > 0) {
        for (int i = tid; i < (kBM - hp * rpb) * 16; i += kThreads)
            *reinterpret_cast<uint4 *>(sm.q + (i & 8 ? kHalfBytes : 0) + (hp * rpb + (i >> 4)) * 128 +
                                       (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        ptx::fence_proxy_async_smem();
    }
    if (warp == kProducerWarp && lane == 0) {
        ptx::prefetch_tensormap(&vmap);
        if (ro > 0) {
            ptx::prefetch_tensormap(&wmap);
            ptx::prefetch_tensormap(&qmap);
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    grid_dep_launch();

    const uint32_t tmem = sm.tmem_base;
    const Waiter wait{&sm.abort, a.err};

    if (warp == kProducerWarp) {
        // ------------------------------------------------------------------ producer ----
        const int P = geo.P;
        const int ppt = kBN / P;                          // pages per tile (<= 8)
        const int seq_pages = (L + P - 1) / P;
        const uint32_t page_bytes = (uint32_t)P * 128u;   // one half of one page
        const int32_t *bt = a.block_table + (size_t)b * geo.max_pages;
        int issued = 0;
        bool bad = false, ok = true;
        // W^R matrices (B operand of the routing MMAs); the first brings the query block along
        for (int r = 0; r < ro; ++r) {
            const int s = r % kStages;
            if (r >= kStages && !(ok = wait(&sm.empty[s], ((r / kStages) & 1) ^ 1))) break;
            if (lane == 0) {
                const int wrow = (geo.wr_per_qh ? h + r : g) * kD;
                ptx::mbar_arrive_expect_tx(&sm.full[s], kTileBytes + (r == 0 ? hp * rpb * kD * 2 : 0));
                ptx::tma_load_2d(sm.tiles[s], &wmap, &sm.full[s], 0, wrow);
                ptx::tma_load_2d(sm.tiles[s] + kHalfBytes, &wmap, &sm.full[s], 64, wrow);
                if (r == 0) {
                    ptx::tma_load_3d(sm.q, &qmap, &sm.full[s], 0, h, q0 + m0);
                    ptx::tma_load_3d(sm.q + kHalfBytes, &qmap, &sm.full[s], 64, h, q0 + m0);
                }
            }
            __syncwarp();
            issued = r + 1;
        }
        for (int i = 0; ok && i < n_tiles; ++i) {
            const int r = i + ro, s = r % kStages;
            const int pg = (tile0 + i) * ppt + lane;      // page index within the sequence
            const bool exists = lane < ppt && pg < seq_pages;
            const int page = exists ? bt[pg] : -1;
            if (r >= kStages && !wait(&sm.empty[s], ((r / kStages) & 1) ^ 1)) break;
            const bool in_range = exists && page >= 0 && page < geo.num_pages;
            if (exists && !in_range) bad = true;
            const unsigned mask = __ballot_sync(0xffffffffu, in_range);
            ptx::for_pages(
                (page * geo.Hkv + g) * P, mask,
                [&] { ptx::mbar_arrive_expect_tx(&sm.full[s], __popc(mask) * page_bytes * 2u); },
                [&](int p, int row) {
                    uint8_t *dst = sm.tiles[s] + p * page_bytes;
                    ptx::tma_load_2d(dst, &vmap, &sm.full[s], 0, row);
                    ptx::tma_load_2d(dst + kHalfBytes, &vmap, &sm.full[s], 64, row);
                });
            issued = r + 1;
        }
        if (__any_sync(0xffffffffu, bad) && lane == 0) raise_flag(a.err, KL_FLAG_BAD_PAGE);
        if (sm.abort) {
            // copies still in flight land before the CTA's shared memory goes away
            for (int i = max(0, issued - kStages); i < issued; ++i) {
                const uint64_t t0 = ptx::globaltimer();
                while (!ptx::mbar_try_wait(&sm.full[i % kStages], (i / kStages) & 1) &&
                       ptx::globaltimer() - t0 < kTimeoutNs) {
                }
            }
        }
    } else if (warp == kMmaWarp || warp == kPvWarp) {
        // ---------------------------------------------------------------- MMA issuers ----
        // K-major SW128 operands step 32 B per 16 columns inside a 64-column half and jump a
        // half (kHalfBytes) every 4 steps; MN-major SW128 operands step 16 rows = 2 KiB; TMEM
        // A operands step 8 columns (16 packed 16-bit values).
        constexpr uint32_t idesc_qk = ptx::idesc_bf16(128, kBS, false, false);
        constexpr uint32_t idesc_mn = ptx::idesc_bf16(128, 128, false, true);   // routing and output
        const uint64_t q_desc = ptx::smem_desc(ptx::smem_addr(sm.q), 16, 1024, ptx::kSwizzle128B);
        const uint64_t k_desc = ptx::smem_desc(ptx::smem_addr(sm.tiles[0]), 16, 1024, ptx::kSwizzle128B);
        const uint64_t mn_desc =
            ptx::smem_desc(ptx::smem_addr(sm.tiles[0]), kHalfBytes, 1024, ptx::kSwizzle128B);
        auto kstep = [](int kk) -> uint32_t { return ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4; };
        if (warp == kMmaWarp) {
            // Q_r = Q . W^R for all 128 rows, once per matrix, into alternating halves of the score
            // columns (a row keeps the result of its head's matrix), then the scores
            bool ok = true;
            for (int r = 0; ok && r < ro; ++r) {
                const int s = r % kStages;
                ok = wait(&sm.full[s], (r / kStages) & 1) &&
                     (r < 2 || wait(&sm.r_free[r & 1], ((r >> 1) - 1) & 1));
                if (!ok) break;
                ptx::tc_fence_after();
                if (ptx::elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < kD / 16; ++kk)
                        ptx::mma_bf16(tmem + kColS + (r & 1) * 128, q_desc + kstep(kk),
                                      mn_desc + ((s * kTileBytes + kk * 2048) >> 4), idesc_mn, kk > 0);
                    ptx::mma_commit(&sm.empty[s]);
                    ptx::mma_commit(&sm.r_full[r & 1]);
                }
                __syncwarp();
            }
            ok = ok && wait(&sm.qr_ready, 0);
            // (the loop by one lane: warp-wide waits between two half tiles leave the tensor cores idle)
            if (ok && ptx::elect_one()) {
                ptx::tc_fence_after();
                for (int u = 0; u < n_sub; ++u) {
                    const int r = (u >> 1) + ro, s = r % kStages, sb = u % kSub;
                    if (!wait.one(&sm.full[s], (r / kStages) & 1)) break;
                    if (u >= kSub && !wait.one(&sm.s_free[sb], (u / kSub - 1) & 1)) break;
                    ptx::tc_fence_after();
                    const uint64_t b0 = k_desc + ((s * kTileBytes + (u & 1) * kBS * 128) >> 4);
#pragma unroll
                    for (int kk = 0; kk < 2 * kD / 16; ++kk)
                        ptx::mma_bf16_ts(tmem + kColS + sb * kBS,
                                         tmem + kColQ + (kk >= 8 ? kLoCols : 0u) + (kk & 7) * 8,
                                         b0 + kstep(kk & 7), idesc_qk, kk > 0);
                    ptx::mma_commit(&sm.s_full[sb]);
                }
            }
        } else if (ptx::elect_one()) {
            for (int u = 0; u < n_sub; ++u) {
                const int s = ((u >> 1) + ro) % kStages, sb = u % kSub;
                if (!wait.one(&sm.p_full[sb], (u / kSub) & 1)) break;
                ptx::tc_fence_after();
                const uint64_t b0 = mn_desc + ((s * kTileBytes + (u & 1) * kBS * 128) >> 4);
                const uint32_t pa = tmem + kColS + sb * kBS;      // P_hi, then P_lo: 8 columns a step
#pragma unroll
                for (int kk = 0; kk < 2 * kBS / 16; ++kk)
                    ptx::mma_bf16_ts(tmem + kColO, pa + kk * 8, b0 + (((kk & 3) * 2048) >> 4), idesc_mn,
                                     (u > 0 || kk > 0) ? 1u : 0u);
                ptx::mma_commit(&sm.s_free[sb]);
                if ((u & 1) || u == n_sub - 1) ptx::mma_commit(&sm.empty[s]);
            }
        }
        __syncwarp();
        // every MMA this warp issued completes before TMEM is freed
        uint64_t *drain = warp == kMmaWarp ? &sm.drain : &sm.drain2;
        if (ptx::elect_one()) ptx::mma_commit(drain);
        __syncwarp();
        const uint64_t t0 = ptx::globaltimer();
        while (!ptx::mbar_try_wait(drain, 0) && ptx::globaltimer() - t0 < kTimeoutNs) {
        }
    } else {
        // --------------------------------------------------------- softmax, epilogue ----
        const int qd = warp & 3, hf = warp >> 2;     // lane quarter; group, and half of the columns
        const int r = qd * 32 + lane;                // row = TMEM lane
        const int ri = r / hp, hh = r - ri * hp;     // draft and head within the block
        const bool live = ri < rows && hh < hn;
        const int c0 = hf * 64;
        const uint32_t lane_base = (uint32_t)(qd * 32) << 16;
        const float sl2 = geo.scale * kLog2e;
        const size_t row_id = (size_t)(q0 + m0 + ri) * geo.Hq + h + hh;   // of q, out and the states
        bool ok = true;

        // Routed query row, this warp's 64 columns, times scale * log2 e, as hi + lo bf16 pairs
        {
            uint32_t x[64];
            if (ro == 0) {
                // the composed query, as it is
                const uint4 *src = reinterpret_cast<const uint4 *>(a.q + row_id * kD + c0);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint4 v = live ? src[c] : make_uint4(0u, 0u, 0u, 0u);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[8 * c + 2 * e] = w[e] << 16;
                        x[8 * c + 2 * e + 1] = w[e] & 0xffff0000u;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 64; ++e) x[e] = 0u;
                for (int i = 0; ok && i < ro; ++i) {
                    ok = wait(&sm.r_full[i & 1], (i >> 1) & 1);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    const bool mine = ro == 1 || hh == i;
                    const uint32_t rc = tmem + kColS + (i & 1) * 128 + c0 + lane_base;
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t u[32];
                        ptx::tmem_ld32(rc + c, u);
                        ptx::tmem_wait_ld();
                        ptx::reg_fence(u);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (mine) x[c + e] = u[e];
                    }
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sm.r_free[i & 1]);
                }
            }
            if (ok) {
                uint32_t hi[32], lo[32];
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    split2(__uint_as_float(x[2 * e]) * sl2, __uint_as_float(x[2 * e + 1]) * sl2, hi[e], lo[e]);
                ptx::tmem_st32(tmem + kColQ + c0 / 2 + lane_base, hi);
                ptx::tmem_st32(tmem + kColQ + kLoCols + c0 / 2 + lane_base, lo);
                ptx::tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sm.qr_ready);
            }
        }

        // the drafts that this row's draft sees: itself and its ancestors
        uint64_t anc_lo = 0, anc_hi = 0;
        if (has_drafts) {
            for (int j = m0 + min(ri, rows - 1); j >= 0; j = sm.parent[j]) {
                if (j < 64) anc_lo |= 1ull << j;
                else anc_hi |= 1ull << (j - 64);
            }
        }

        float m_used = -INFINITY;  // the reference of this thread's share of the row sum
        float2 la = make_float2(0.f, 0.f), lb = make_float2(0.f, 0.f);
        bool okl = ok;
        for (int u = hf; okl && u < n_sub; u += 2) {
            const int t0 = tile0 * kBN + u * kBS, sb = u % kSub;
            const uint32_t sbuf = tmem + kColS + (uint32_t)sb * kBS + lane_base;   // S, then P
            okl = wait(&sm.s_full[sb], (u / kSub) & 1);
            if (!okl) break;
            ptx::tc_fence_after();
            uint32_t s0[32], s1[32];
            ptx::tmem_ld32(sbuf, s0);
            ptx::tmem_ld32(sbuf + 32, s1);
            const bool drafts_here = t0 + kBS > base;
            if (drafts_here) {
                // Rows that not every draft sees must not reach the others through 0 * NaN: a row past
                // the sequence's end, or one that is not finite, is zeroed for the output MMAs (the
                // score MMAs have read it; a draft that sees such a row has a NaN score). Thread =
                // (cache row, 64-dim half).
                const int st = ((u >> 1) + ro) % kStages;
                okl = wait(&sm.full[st], (((u >> 1) + ro) / kStages) & 1);   // (the copy: completed)
                if (!okl) break;
                const int tr = r & 63;
                if (t0 + tr >= base) {
                    const uint32_t v_s = ptx::smem_addr(sm.tiles[st]) + (r >> 6) * kHalfBytes +
                                         (hf * kBS + tr) * 128;
                    bool zero = t0 + tr >= L;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint32_t v[4];
                        ld_shared_v4(v_s + ((c + lane) & 7) * 16, v);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            zero |= (v[e] & 0x7f80u) == 0x7f80u || (v[e] & 0x7f800000u) == 0x7f800000u;
                    }
                    if (zero)
#pragma unroll
                        for (int c = 0; c < 8; ++c) st_shared_v4(v_s + c * 16, 0u, 0u, 0u, 0u);
                }
            }
            ptx::tmem_wait_ld();
            ptx::reg_fence(s0);
            ptx::reg_fence(s1);
            if (drafts_here) {
                const uint64_t vis = window64(anc_lo, anc_hi, t0 - base);
                const uint32_t v0 = (uint32_t)vis, v1 = (uint32_t)(vis >> 32);
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    if (!(v0 & (1u << c))) s0[c] = 0xff800000u;
                    if (!(v1 & (1u << c))) s1[c] = 0xff800000u;
                }
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
                mx[0] = max3(mx[0], __uint_as_float(s0[c]), __uint_as_float(s0[c + 1]));
                mx[1] = max3(mx[1], __uint_as_float(s0[c + 2]), __uint_as_float(s0[c + 3]));
                mx[2] = max3(mx[2], __uint_as_float(s1[c]), __uint_as_float(s1[c + 1]));
                mx[3] = max3(mx[3], __uint_as_float(s1[c + 2]), __uint_as_float(s1[c + 3]));
            }
            float mt = max3(mx[0], mx[1], fmaxf(mx[2], mx[3]));
            float m_ref = -INFINITY;
            if (u == 0) {
                // the row's first reference is the maximum of its first two half tiles
                if (n_sub > 1) {
                    okl = wait(&sm.first[qd], 0);
                    if (!okl) break;
                    mt = fmaxf(mt, sm.lsum[1][r]);
                }
            } else {
                if (u == 1) {
                    sm.lsum[1][r] = mt;
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sm.first[qd]);
                }
                okl = wait(&sm.turn[qd][hf ^ 1], ((u - 1) >> 1) & 1);
                if (!okl) break;
                m_ref = sm.mref[hf ^ 1][r];
            }
            // a new reference when the maximum grew by more than 2^7 (or is the first finite)
            const float m_new = fmaxf(m_ref, mt);
            if (__any_sync(0xffffffffu, m_new > m_ref + kRescaleLog2)) {
                const float f = (m_new == -INFINITY || m_ref == -INFINITY) ? 0.f : ptx::ex2(m_ref - m_new);
                if (u > 0) {
                    // O holds half tiles 0 .. u - 1 once the output MMAs of u - 1 are done
                    okl = wait(&sm.s_free[(u - 1) % kSub], ((u - 1) / kSub) & 1);
                    if (!okl) break;
                    ptx::tc_fence_after();
#pragma unroll
                    for (int c = 0; c < 128; c += 32) {
                        uint32_t o[32];
                        ptx::tmem_ld32(tmem + kColO + c + lane_base, o);
                        ptx::tmem_wait_ld();
                        ptx::reg_fence(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        ptx::tmem_st32(tmem + kColO + c + lane_base, o);
                    }
                    ptx::tmem_wait_st();
                }
                m_ref = m_new;
            }
            sm.mref[hf][r] = m_ref;
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sm.turn[qd][hf]);
            // the group's sums move to this reference
            if (__any_sync(0xffffffffu, m_ref != m_used)) {
                const float f = m_used == -INFINITY ? 0.f : ptx::ex2(m_used - m_ref);
                la = mul2(la, f);
                lb = mul2(lb, f);
                m_used = m_ref;
            }
            // the row's 64 weights -> 32 packed columns of P_hi and 32 of P_lo
            const float mr = m_ref == -INFINITY ? 0.f : m_ref;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                uint32_t *s = e < 16 ? s0 + 2 * e : s1 + 2 * (e - 16);
                const float2 d = sub2(make_float2(__uint_as_float(s[0]), __uint_as_float(s[1])),
                                      make_float2(mr, mr));
                const float2 pe = make_float2(ptx::ex2(d.x), ptx::ex2(d.y));
                if (e & 1) lb = add2(lb, pe); else la = add2(la, pe);
                s[0] = __float_as_uint(pe.x);
                s[1] = __float_as_uint(pe.y);
            }
            uint32_t hi[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                uint32_t *s = e < 16 ? s0 + 2 * e : s1 + 2 * (e - 16);
                uint32_t lo;
                split2(__uint_as_float(s[0]), __uint_as_float(s[1]), hi[e], lo);
                s0[e] = lo;        // (s0[e] has been read: e <= 2 e)
            }
            // P over the buffer (the output MMAs of u - kSub, the last reader of P there, finished
            // before these scores were written)
            ptx::tmem_st32(sbuf, hi);
            ptx::tmem_st32(sbuf + 32, s0);
            ptx::tmem_wait_st();
            ptx::tc_fence_before();
            if (drafts_here) ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sm.p_full[sb]);
        }

        // Epilogue: out = O / l, or the run's state (m, l, O); l is the two groups' shares at the
        // reference of the last half tile. This warp's 64 output dims.
        const int last = n_sub - 1, lb2 = last & 1;
        if (okl && lb2 != hf) okl = wait(&sm.turn[qd][lb2], (last >> 1) & 1);
        const bool oke = okl && wait(&sm.s_free[last % kSub], (last / kSub) & 1);
        float l = (la.x + la.y) + (lb.x + lb.y);
        if (oke && lb2 != hf) {
            const float m_fin = sm.mref[lb2][r];
            l = m_used == -INFINITY ? 0.f : l * ptx::ex2(m_used - m_fin);
        }
        sm.lsum[hf][r] = l;
        const bool okp = ptx::bar_and(kBarCompute, 32 * kComputeWarps, oke);
        if (okp) {
            ptx::tc_fence_after();
            const float lt = l + sm.lsum[hf ^ 1][r];
            const bool whole = runs == 1;
            const float f = !whole ? 1.f : lt == 0.f ? 0.f : 1.f / lt;
            float *state = a.part_o + (row_id * a.S + split) * kD + c0;
#pragma unroll
            for (int c4 = 0; c4 < 2; ++c4) {
                uint32_t u[32];
                ptx::tmem_ld32(tmem + kColO + c0 + c4 * 32 + lane_base, u);
                ptx::tmem_wait_ld();
                ptx::reg_fence(u);
                if (live && (!whole || a.out_dtype == KL_FP32)) {
                    float4 *o = reinterpret_cast<float4 *>(
                        whole ? static_cast<float *>(a.out) + row_id * kD + c0 + c4 * 32 : state + c4 * 32);
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        o[c] = make_float4(__uint_as_float(u[4 * c]) * f, __uint_as_float(u[4 * c + 1]) * f,
                                           __uint_as_float(u[4 * c + 2]) * f, __uint_as_float(u[4 * c + 3]) * f);
                } else if (live) {
                    uint4 *o = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + row_id * kD + c0 +
                                                         c4 * 32);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = pack2(__uint_as_float(u[8 * c + 2 * e]) * f,
                                         __uint_as_float(u[8 * c + 2 * e + 1]) * f);
                        o[c] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (!whole) {
                if (hf == 0 && live)
                    reinterpret_cast<float2 *>(a.part_ml)[row_id * a.S + split] =
                        make_float2(sm.mref[lb2][r], lt);
                // The last CTA of the block to finish merges the states: out = sum_s w_s O_s / sum_s
                // w_s l_s with w_s = 2^(m_s - M); a warp per row, 4 dims per lane.
                ptx::bar_sync(kBarCompute, 32 * kComputeWarps);
                if (tid == 0)
                    sm.is_last = arrive_last(a.counters + ((size_t)b * geo.Hkv + g) * a.blocks + blk, runs);
                ptx::bar_sync(kBarCompute, 32 * kComputeWarps);
                if (sm.is_last) {
                    for (int i = warp; i < rows * hp; i += kComputeWarps) {
                        const int mi = i / hp, mh = i - mi * hp;
                        if (mh >= hn) continue;
                        const size_t id = (size_t)(q0 + m0 + mi) * geo.Hq + h + mh;
                        const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + id * a.S;
                        float M = -INFINITY;
                        for (int s = lane; s < runs; s += 32) {
                            const float2 v = __ldcg(ml + s);
                            if (v.y != 0.f) M = fmaxf(M, v.x);
                        }
#pragma unroll
                        for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
                        const float4 *po = reinterpret_cast<const float4 *>(a.part_o + id * a.S * kD) + lane;
                        float z = 0.f;
                        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                        for (int s = 0; s < runs; ++s) {
                            const float2 v = __ldcg(ml + s);
                            const float4 x = __ldcg(po + (size_t)s * (kD / 4));
                            // (a run in which the row sees nothing has l = 0 and m = -inf)
                            const float w = v.y == 0.f ? 0.f : ptx::ex2(v.x - M);
                            z = fmaf(w, v.y, z);
                            acc.x = fmaf(w, x.x, acc.x);
                            acc.y = fmaf(w, x.y, acc.y);
                            acc.z = fmaf(w, x.z, acc.z);
                            acc.w = fmaf(w, x.w, acc.w);
                        }
                        const float inv = z == 0.f ? 0.f : 1.f / z;
                        if (a.out_dtype == KL_FP32)
                            reinterpret_cast<float4 *>(static_cast<float *>(a.out) + id * kD)[lane] =
                                make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
                        else
                            reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + id * kD)[lane] =
                                make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
                    }
                }
            }
        }
    }

    ptx::tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, kTmemCols);
    }
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
    const size_t smem = sizeof(TreeSmem) + 1024;
    static PerDeviceOnce once;
    const cudaError_t e = once.run([&] {
        return cudaFuncSetAttribute(tree_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.blocks * a.S, g.Hkv, g.B);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = a.stream;
    const OverlapAttr overlap(cfg);
    return cudaLaunchKernelEx(&cfg, tree_tc_kernel, vmap, wmap, qmap, a);
}

}  // namespace kl
