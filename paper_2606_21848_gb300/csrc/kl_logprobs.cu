// Log probabilities of given tokens, the entropy and the largest logits of rows of logits, in one pass.
//
// With x = scale * logits, z = sum_j exp(x_j) and p = exp(x) / z:
//   logprob(t) = x_t - log z,   H = - sum_j p_j log p_j = log z - sum_j p_j x_j,
// and the `top` largest logits, ties to the lowest index. Bound by HBM: every logit is read once; 5 to 6
// instructions per bf16 logit leave the issue slots half busy at full bandwidth.
//
// The rows are cut into chunks of up to 32 KiB. Each CTA, three per SM, takes an equal run of consecutive
// chunks and streams them through a ring of bulk copies, so that loads stay in flight whatever the
// threads do. A thread keeps its own state over the chunks of a row, in fp32: its largest logit m, and
// with y = (x - m) scale log2 e (the difference first, so that rows of huge or lowest values neither
// overflow nor cancel) s1 = sum 2^y and s2 = sum y 2^y. States join as softmax states do: with d =
// (m - M) scale log2 e, s1' = 2^d s1, s2' = 2^d s2 + d s1'; at last log z = log(s1) above scale * M and
// H = log(s1) - s2 / s1 ln 2. (The rounding of scale log2 e to fp32 moves every y by the same part, which
// s2 takes out of s1 again; log probabilities are within a few units of 2^-24 of 1 and of their size.) A row
// that lies in several CTAs' runs is joined by the last of them.
//
// Selection: keys (value, lowest index first) above the smallest of the `top` best so far go to a list of
// candidates in shared memory, which is ranked by counting and cut to `top` after the row's first chunk,
// when it fills up and at the row's end. The first chunk's bound comes from the threads' maxima: with
// `top` of them known to be >= t, so are `top` logits; t is the larger of (the smallest, over the w warps
// with a vector for every thread, of the ceil(top / w)-th largest maximum) and (the largest over all warps of the
// top-th).
//
// Measured: 2048 rows of 151936 bf16 logits, no alternatives, 102 us (6100 GB/s, 0.90 of a copy's); 512 rows of
// 128256 with the 8 largest 40 us (3300 GB/s: 1.1 runs per row, whose selections' steps, some 4 us a row, do
// not overlap within a CTA); 96 rows of 50257 fp32 logits with the 20 largest 18 us, and one row of 32000 8.3 us
// (latency: first copy 1, first selection 2, further chunks 3, ranking 1.3, the join of a row's parts 4).
#include <float.h>
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "kl_internal.cuh"
#include "kl_tc_ptx.cuh"

namespace kl {
namespace {

constexpr int kLpThreads = 256, kLpWarps = 8;
constexpr int kLpVecs = 8;                               // 16-byte vectors per thread and chunk
constexpr int kLpChunk = kLpThreads * kLpVecs;           // vectors per chunk, at most
constexpr int kLpMinChunk = 512;                         // vectors per chunk where rows are few
constexpr int kLpStages = 2;
constexpr int kLpCtas = 3;                               // per SM
constexpr int kLpCap = 1024;                             // candidates in shared memory,
constexpr int kLpExtra = 16;                             // room among them for a row's head and tail
static_assert(KL_LOGPROBS_MAX_TOP <= 32, "a warp's sorted maxima bound the selection");

struct __align__(16) LogprobSmem {
    uint8_t ring[kLpStages][kLpChunk * 16];
    uint64_t full[kLpStages];
    uint64_t cand[kLpCap];
    uint64_t list[KL_LOGPROBS_MAX_TOP];                  // keys, largest first
    uint64_t wkey[kLpWarps];
    float wmax[kLpWarps], wnth[kLpWarps], wtop[kLpWarps];
    float s1[kLpWarps], e1[kLpWarps], s2[kLpWarps];
    int wcount[kLpWarps];
    int added[3];                                        // candidates of a chunk, by chunk number % 3
    int is_last;
    int lost;                                            // 1 + the number of a chunk that did not land in time
};
static_assert(sizeof(LogprobSmem) * kLpCtas <= (228 - kLpCtas) * 1024, "CTAs per SM");

// Keys order logits by value, then by lowest index; 0 is below every key. (-0 counts as +0.)
__device__ __forceinline__ uint64_t make_key(float x, int idx) {
    const int b = __float_as_int(x + 0.f);
    const uint32_t o = (uint32_t)(b >= 0 ? b : b ^ 0x7FFFFFFF) ^ 0x80000000u;
    return (uint64_t)o << 32 | (uint32_t)~idx;
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) {
    const int b = (int)((uint32_t)(k >> 32) ^ 0x80000000u);
    return __int_as_float(b >= 0 ? b : b ^ 0x7FFFFFFF);
}

// The 32-bit word w as logits: two bf16 (x the lower half) or one fp32 (x).
template <typename T>
__device__ __forceinline__ float2 lp_unpack(uint32_t w) {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w), -INFINITY);
    else return make_float2(bf16lo(w), bf16hi(w));
}

// Packed fp32 pairs (one instruction for two logits).
__device__ __forceinline__ float2 lp_add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 lp_mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "mul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 lp_fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "mov.b64 z, {%6, %7};\n\tfma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

// max of two packed bf16 pairs (a NaN loses).
__device__ __forceinline__ uint32_t lp_max_bf16(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

template <typename T>
__device__ __forceinline__ float lp_load(const void *row, int idx) {
    if constexpr (sizeof(T) == 4) return static_cast<const float *>(row)[idx];
    else return bf16lo((uint32_t)static_cast<const uint16_t *>(row)[idx]);
}

// s + x, with what the rounding lost added to e (exactly that while s and x are finite).
__device__ __forceinline__ float sum_of(float s, float x, float &e) {
    const float t = s + x, y = t - s;
    e += (s - (t - y)) + (x - y);
    return t;
}

// Sum over each warp of s1 and s2, to the warps' slots (block_sums() after the next barrier). Of s1, in which one
// logit often holds most, the roundings are kept: the other 12 adds would each take half a unit of it.
__device__ __forceinline__ void warp_sums(LogprobSmem &sm, float s1, float s2, int warp, int lane) {
    float e = 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        e += __shfl_xor_sync(0xffffffffu, e, o);
        s1 = sum_of(s1, __shfl_xor_sync(0xffffffffu, s1, o), e);
        s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    if (lane == 0) {
        sm.s1[warp] = s1;
        sm.e1[warp] = e;
        sm.s2[warp] = s2;
    }
}
__device__ __forceinline__ void block_sums(const LogprobSmem &sm, float &s1, float &s2) {
    float e = 0.f;
    s1 = s2 = 0.f;
#pragma unroll
    for (int w = 0; w < kLpWarps; ++w) {
        s1 = sum_of(s1, sm.s1[w], e);
        e += sm.e1[w];
        s2 += sm.s2[w];
    }
    s1 += e;
}

// The keys cand[0 .. n - 1] (all different), ranked: the largest `top` of them to list. n <= kLpCap.
__device__ __forceinline__ void rank_keys(LogprobSmem &sm, int n, int top, int tid) {
    for (int i = tid; i < n; i += kLpThreads) {
        const uint64_t k = sm.cand[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += sm.cand[j] > k;
        if (above < top) sm.list[above] = k;
    }
}

// The slow way, for any number of candidates: `top` rounds, each the largest key below the last one.
// best(prev) is the thread's own largest key below prev (0: none).
template <typename F>
__device__ __forceinline__ void take_keys(LogprobSmem &sm, int top, int tid, F &&best) {
    uint64_t prev = ~0ull;
    for (int i = 0; i < top; ++i) {
        uint64_t k = best(prev);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const uint64_t x = __shfl_xor_sync(0xffffffffu, k, o);
            if (x > k) k = x;
        }
        if ((tid & 31) == 0) sm.wkey[tid >> 5] = k;
        __syncthreads();
        prev = 0;
#pragma unroll
        for (int w = 0; w < kLpWarps; ++w)
            if (sm.wkey[w] > prev) prev = sm.wkey[w];
        if (tid == 0) sm.list[i] = prev;
        __syncthreads();
    }
}

// Largest of `n` values over the block by warps (each thread gets it after the barrier inside).
__device__ __forceinline__ float block_max(LogprobSmem &sm, float x, int warp, int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    if (lane == 0) sm.wmax[warp] = x;
    __syncthreads();
    x = sm.wmax[0];
#pragma unroll
    for (int w = 1; w < kLpWarps; ++w) x = fmaxf(x, sm.wmax[w]);
    return x;
}

// A state (m, s1, s2) moves to the reference M >= m. (One so low that its factor is 0 keeps only NaN.)
__device__ __forceinline__ void move_state(float m, float M, float c, float &s1, float &s2) {
    if (m == -INFINITY || m == M) return;                // (the sums are 0 or NaN; nothing moves)
    const float d = (m - M) * c, f = ptx::ex2(d);
    s1 *= f;
    s2 = f == 0.f ? s1 : fmaf(d, s1, f * s2);
}

// Where a row's chunks lie. The row starts with `head` logits ahead of a 16-byte boundary, then `vecs`
// vectors, then `tail` logits.
template <typename T>
struct LogprobRow {
    static constexpr int VEC = 16 / sizeof(T);
    const char *p;
    int head, vecs, tail;
    __device__ LogprobRow(const LogprobArgs &a, int row) {
        p = static_cast<const char *>(a.logits) + (size_t)row * a.stride * sizeof(T);
        head = min(a.vocab, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) % 16 / sizeof(T)));
        vecs = (a.vocab - head) / VEC;
        tail = a.vocab - head - vecs * VEC;
    }
};

// The copy of chunk k that has not landed at the first look, up to `limit` ns (short ones by the poll that does
// not suspend the thread); else sm.lost becomes k + 1.
__device__ __noinline__ void wait_slow(LogprobSmem &sm, int k, uint64_t limit) {
    uint64_t *bar = &sm.full[k % kLpStages];
    const uint32_t phase = (k / kLpStages) & 1;
    const uint64_t t0 = ptx::globaltimer();
    while (!(limit < kExactWaitNs ? ptx::mbar_test_wait(bar, phase) : ptx::mbar_try_wait(bar, phase)))
        if (ptx::globaltimer() - t0 > limit) {
            sm.lost = k + 1;
            return;
        }
}

// Runs of chunks: `each` per CTA, one more for the first `extra`. (The quotients mostly fit 32 bits, whose
// division is much shorter.)
struct LogprobRuns {
    int64_t each;
    int extra;
    __device__ LogprobRuns(int64_t total, int ctas) {
        each = quotient(total, ctas);
        extra = (int)(total - each * ctas);
    }
    static __device__ int64_t quotient(int64_t x, int64_t y) {
        return (x | y) <= INT32_MAX ? (int)x / (int)y : x / y;
    }
    __device__ int64_t start(int c) const { return each * c + min(c, extra); }
    // the CTA whose run holds chunk i
    __device__ int of(int64_t i) const {
        const int64_t first = (each + 1) * extra;
        return i < first ? (int)quotient(i, each + 1) : extra + (int)quotient(i - first, each);
    }
};

// Where the part of a row in CTA c's run lies, of a row that starts in CTA c0's: every run has at most one row
// that began in an earlier one (its first) and one that goes on in the next (its last).
__device__ __forceinline__ size_t part_slot(int c, int c0) { return 2 * (size_t)c + (c == c0); }

// The parts of a row that starts in CTA c0's run, joined by the CTA that arrived last: the sums to every
// thread, the keys to the list.
__device__ void join_parts(LogprobSmem &sm, const LogprobArgs &a, int c0, int parts, float c, float &m,
                           float &s1, float &s2) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, top = a.top;
    auto part = [&](int i) { return a.part + part_slot(c0 + i, c0); };
    auto keys = [&](int i) { return a.part_top + part_slot(c0 + i, c0) * top; };
    // every part's last key is a bound; the largest of them leaves few
    float M = -INFINITY;
    uint64_t least = 0;
    for (int i = tid; i < parts; i += kLpThreads) {
        M = fmaxf(M, __ldcg(part(i)).x);
        if (top > 0) {
            const uint64_t x = __ldcg(keys(i) + top - 1);
            if (x > least) least = x;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t x = __shfl_xor_sync(0xffffffffu, least, o);
        if (x > least) least = x;
    }
    if (lane == 0) sm.wkey[warp] = least;
    if (tid < KL_LOGPROBS_MAX_TOP) sm.list[tid] = 0;
    if (tid == 0) sm.wcount[0] = 0;
    M = block_max(sm, M, warp, lane);
    float a1 = 0.f, a2 = 0.f;
    for (int i = tid; i < parts; i += kLpThreads) {
        const float4 q = __ldcg(part(i));
        float p1 = q.y, p2 = q.z;
        move_state(q.x, M, c, p1, p2);
        a1 += p1;
        a2 += p2;
    }
    warp_sums(sm, a1, a2, warp, lane);
    if (top > 0) {
        least = 0;
#pragma unroll
        for (int w = 0; w < kLpWarps; ++w)
            if (sm.wkey[w] > least) least = sm.wkey[w];
        for (int i = tid; i < parts * top; i += kLpThreads) {
            const uint64_t x = __ldcg(keys(i / top) + i % top);
            if (x != 0 && x >= least) {
                const int at = atomicAdd(&sm.wcount[0], 1);
                if (at < kLpCap) sm.cand[at] = x;
            }
        }
    }
    __syncthreads();
    block_sums(sm, s1, s2);
    m = M;
    if (top > 0) {
        const int n = sm.wcount[0];
        if (n <= kLpCap) {
            rank_keys(sm, n, top, tid);
        } else {
            take_keys(sm, top, tid, [&](uint64_t prev) {
                uint64_t best = 0;
                for (int i = tid; i < parts * top; i += kLpThreads) {
                    const uint64_t x = __ldcg(keys(i / top) + i % top);
                    if (x < prev && x > best) best = x;
                }
                return best;
            });
        }
        __syncthreads();
    }
}

// The results of a row. One of -inf alone has no distribution: log probabilities of -inf, entropy 0. A NaN
// or +inf logit makes the sums, and with them everything but the ids, NaN.
template <typename T>
__device__ void finish_row(LogprobSmem &sm, const LogprobArgs &a, const char *rp, int row, float m, float s1,
                           float s2, int token, float given) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, top = a.top;
    const bool none = s1 == 0.f;
    const float lz = logf(fmaf(a.c_error * kLn2, s2, s1));       // (to first order: dz / dc = ln 2 s2 / c)
    auto logprob = [&](float x) { return none ? -INFINITY : fmaf(x - m, a.scale, -lz); };
    for (int i = tid; i < a.per_row; i += kLpThreads) {
        const bool here = i < kLpThreads;                // (the thread's first)
        const int id = here ? token : a.tokens[(size_t)row * a.per_row + i];
        float lp = 0.f;                                  // -1: no token
        if (id >= 0 && id < a.vocab) {
            lp = logprob(here ? given : lp_load<T>(rp, id));
        } else if (id != -1) {
            lp = NAN;
            raise_flag(a.err, KL_FLAG_BAD_TOKEN);
        }
        a.logprobs[(size_t)row * a.per_row + i] = lp;
    }
    if (tid == 0 && a.entropy) a.entropy[row] = none ? 0.f : fmaf(s2 / s1, -kLn2, lz);
    if (tid == 0 && s1 != s1) raise_flag(a.err, KL_FLAG_RANGE);
    if (top > 0 && sm.list[top - 1] == 0) {
        // fewer than `top` logits above -inf: the first of the others, in order
        int n = 0;
        while (sm.list[n] != 0) ++n;
        __syncthreads();
        for (int jb = 0; jb < a.vocab && n < top; jb += kLpThreads) {
            const int j = jb + tid;
            const bool mine = j < a.vocab && lp_load<T>(rp, j) == -INFINITY;
            const unsigned votes = __ballot_sync(0xffffffffu, mine);
            if (lane == 0) sm.wcount[warp] = __popc(votes);
            __syncthreads();
            int at = n + __popc(votes & ((1u << lane) - 1));
#pragma unroll
            for (int w = 0; w < kLpWarps; ++w) {
                if (w < warp) at += sm.wcount[w];
                n += sm.wcount[w];
            }
            if (mine && at < top) sm.list[at] = make_key(-INFINITY, j);
            __syncthreads();
        }
    }
    if (tid < top) {
        const uint64_t k = sm.list[tid];
        a.top_ids[(size_t)row * top + tid] = k ? key_index(k) : -1;
        a.top_logprobs[(size_t)row * top + tid] = k ? logprob(key_value(k)) : NAN;
    }
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads, kLpCtas) logprobs_kernel(const LogprobArgs a, const int per_chunk) {
    using Row = LogprobRow<T>;
    constexpr int VEC = Row::VEC;
    extern __shared__ __align__(16) uint8_t lp_smem[];
    LogprobSmem &sm = *reinterpret_cast<LogprobSmem *>(lp_smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int top = a.top;
    const float c = a.scale * kLog2e;
    const int64_t total = (int64_t)a.rows * a.chunks;
    const LogprobRuns runs(total, gridDim.x);
    const int64_t it0 = runs.start(blockIdx.x), it1 = runs.start(blockIdx.x + 1);
    const int steps = (int)(it1 - it0);
    if (tid == 0) {
        for (int s = 0; s < kLpStages; ++s) ptx::mbar_init(&sm.full[s], 1);
        ptx::fence_mbar_init();
    }
    if (tid < 3) sm.added[tid] = 0;
    if (tid == 3) sm.lost = INT_MAX;
    __syncthreads();
    grid_dep_wait();
    grid_dep_launch();

    // thread 0: the copy of the run's chunk k into its slot (called for k = 0, 1, 2, ...)
    int row = (int)LogprobRuns::quotient(it0, a.chunks), ch = (int)(it0 - (int64_t)row * a.chunks);
    int frow = row, fch = ch;
    auto fetch = [&](int k) {
        const Row r(a, frow);
        const int q0 = fch * per_chunk, nv = max(0, min(per_chunk, r.vecs - q0));
        if (++fch == a.chunks) {
            fch = 0;
            ++frow;
        }
        uint64_t *bar = &sm.full[k % kLpStages];
        if (nv == 0) {
            ptx::mbar_arrive(bar);
            return;
        }
        ptx::mbar_arrive_expect_tx(bar, (uint32_t)nv * 16u);
        ptx::bulk_load(sm.ring[k % kLpStages], r.p + (size_t)r.head * sizeof(T) + (size_t)q0 * 16, (uint32_t)nv * 16u, bar);
    };
    if (tid == 0)
        for (int k = 0; k < kLpStages && k < steps; ++k) fetch(k);

    float m = -INFINITY, s1 = 0.f, s2 = 0.f;             // this thread's state of the row
    float extra = -INFINITY;                             // its logit of the row's head or tail
    int extra_at = -1;
    int token = -1;                                      // its given token of the row and that one's logit,
    float given = 0.f;                                   // fetched while the chunks stream
    int kept = 0;                                        // candidates known to all threads
    float from = -FLT_MAX;                               // logits below do not matter
    uint64_t above = 0;                                  // nor do keys up to this one
    Row r(a, row);
    // The candidates that chunk k added become known: cut to the `top` largest when they are the row's
    // first (which gives the bound for the rest) or fill half of the list, or at the end. Where they
    // overflowed it (ties; rising rows), the chunk is read once more. All threads, after a barrier behind
    // the chunk's adds; ends behind a barrier if it cut.
    auto settle = [&](int k, bool all) {
        const int n = kept + sm.added[k % 3];
        if (tid == 0) sm.added[(k + 2) % 3] = 0;         // chunk k - 1's: read by all before that barrier
        if (n <= kLpCap - kLpExtra) {
            if (!all && (above != 0 || n < top) && n <= kLpCap / 2) {
                kept = n;
                return;
            }
            rank_keys(sm, n, top, tid);
            __syncthreads();
        } else {
            const int c = ch - (all ? 0 : 1);            // the chunk's number in the row
            const int j0 = r.head + c * per_chunk * VEC, j1 = r.head + min(r.vecs, (c + 1) * per_chunk) * VEC;
            take_keys(sm, top, tid, [&](uint64_t prev) {
                uint64_t best = 0;
                for (int i = tid; i < kept; i += kLpThreads)
                    if (sm.cand[i] < prev && sm.cand[i] > best) best = sm.cand[i];
                for (int j = j0 + tid; j < j1; j += kLpThreads) {
                    const float x = lp_load<T>(r.p, j);
                    const uint64_t y = x >= from ? make_key(x, j) : 0;
                    if (y < prev && y > best) best = y;
                }
                return best;
            });
        }
        kept = min(n, top);
        if (kept == top) {
            above = sm.list[top - 1];
            from = key_value(above);
        }
        if (tid < kept) sm.cand[tid] = sm.list[tid];
        if (tid == 0) sm.added[k % 3] = 0;
        __syncthreads();
    };

    for (int k = 0; k < steps; ++k, ++ch) {
        if (ch == a.chunks) {
            ch = 0;
            ++row;
        }
        const bool first = k == 0 || ch == 0, last = k == steps - 1 || ch == a.chunks - 1;
        if (first) {
            r = Row(a, row);
            m = -INFINITY;
            s1 = s2 = 0.f;
            kept = 0;
            from = -FLT_MAX;
            above = 0;
            // the logits outside the vectors: the first chunk's CTA takes the head, the last one's the tail
            const bool in_head = tid < r.head && ch == 0;
            const bool in_tail = tid >= 32 && tid - 32 < r.tail && it1 >= ((int64_t)row + 1) * a.chunks;
            extra_at = in_head ? tid : in_tail ? a.vocab - r.tail + tid - 32 : -1;
            extra = extra_at >= 0 ? lp_load<T>(r.p, extra_at) : -INFINITY;
            token = tid < a.per_row ? a.tokens[(size_t)row * a.per_row + tid] : -1;
        }
        // Everyone has read the last chunk's slot, and its candidates are complete.
        __syncthreads();
        // (the CTA leaves as a whole: a thread that is ahead may lose chunk k, but none before it)
        if (*(volatile int *)&sm.lost <= k) break;
        if (tid == 0 && k > 0 && k - 1 + kLpStages < steps) fetch(k - 1 + kLpStages);
        if (top > 0 && !first) settle(k - 1, false);
        // the chunk: vector i of the thread is i * 256 + tid
        const int slot = k % kLpStages;
        const int q0 = ch * per_chunk, nv = min(per_chunk, r.vecs - q0);
        if (a.wait_ns < kExactWaitNs || !ptx::mbar_try_wait(&sm.full[slot], (k / kLpStages) & 1))
            wait_slow(sm, k, a.wait_ns);
        // (read from shared memory once for the maximum and once for the sums: 64 logits held in between
        // spilled)
        const uint4 *const data = reinterpret_cast<const uint4 *>(sm.ring[slot]) + tid;
        const int mine = nv > tid ? (nv - tid + kLpThreads - 1) / kLpThreads : 0;   // vectors of this thread
        float tmax = -INFINITY;                          // (NaN does not take part)
        {
            uint32_t t = 0xff80ff80u;
            auto look = [&](const uint4 &x) {
                if constexpr (sizeof(T) == 4) {
                    tmax = fmaxf(fmaxf(fmaxf(__uint_as_float(x.x), __uint_as_float(x.y)), __uint_as_float(x.z)),
                                 fmaxf(tmax, __uint_as_float(x.w)));
                } else {
                    t = lp_max_bf16(lp_max_bf16(lp_max_bf16(x.x, x.y), lp_max_bf16(x.z, x.w)), t);
                }
            };
            if (mine == kLpVecs) {
#pragma unroll
                for (int i = 0; i < kLpVecs; ++i) look(data[i * kLpThreads]);
            } else {
                for (int i = 0; i < mine; ++i) look(data[i * kLpThreads]);
            }
            if constexpr (sizeof(T) == 2) tmax = fmaxf(bf16lo(t), bf16hi(t));
        }

        if (top > 0) {
            float bound = from;
            if (first) {
                const int full = min(kLpWarps, max(1, nv >> 5));     // warps without an idle thread
                // the bound: the threads' maxima sorted over the lanes (descending)
                float s = tmax;
#pragma unroll
                for (int g = 2; g <= 32; g <<= 1)
#pragma unroll
                    for (int j = g >> 1; j > 0; j >>= 1) {
                        const float o = __shfl_xor_sync(0xffffffffu, s, j);
                        const bool larger = ((lane & j) == 0) == ((lane & g) == 0);
                        s = larger ? fmaxf(s, o) : fminf(s, o);
                    }
                const int nth = (top + full - 1) / full;
                if (lane == nth - 1) sm.wnth[warp] = s;
                if (lane == top - 1) sm.wtop[warp] = s;
                __syncthreads();
                float lowest = sm.wnth[0], best = sm.wtop[0];
#pragma unroll
                for (int w = 1; w < kLpWarps; ++w) {
                    if (w < full) lowest = fminf(lowest, sm.wnth[w]);
                    best = fmaxf(best, sm.wtop[w]);
                }
                bound = fmaxf(-FLT_MAX, fmaxf(best, lowest));
            }
            // For each thread with a hit its warp looks at the thread's 32 words, one per lane.
            static_assert(kLpVecs * 4 == 32, "a word per lane");
            for (unsigned left = __ballot_sync(0xffffffffu, tmax >= bound); left; left &= left - 1) {
                const int at = (lane >> 2) * kLpThreads + warp * 32 + __ffs(left) - 1;   // vector
                if (at < nv) {
                    const float2 x = lp_unpack<T>(reinterpret_cast<const uint32_t *>(sm.ring[slot])[4 * at + (lane & 3)]);
                    const int j = r.head + (q0 + at) * VEC + (lane & 3) * (VEC / 4);
                    auto add = [&](float y, int index) {
                        const uint64_t key = make_key(y, index);
                        if (y >= bound && key > above) {
                            const int o = kept + atomicAdd(&sm.added[k % 3], 1);
                            if (o < kLpCap) sm.cand[o] = key;
                        }
                    };
                    add(x.x, j);
                    if (VEC == 8) add(x.y, j + 1);
                }
                __syncwarp();
            }
        }

        // the sums, at the thread's largest logit (a reference that stays behind leaves log2 s1 and the largest
        // x - m large, and their difference with those numbers' roundings)
        if (__any_sync(0xffffffffu, tmax > m)) {
            const float to = fmaxf(tmax, m);
            move_state(m, to, c, s1, s2);
            m = to;
        }
        {
            // (a weight of 0 at y = -inf has to add 0 to s2, not NaN: with the clamp, where it came up)
            const float mr = m == -INFINITY ? 0.f : m;
            const float2 neg_m = make_float2(-mr, -mr), cc = make_float2(c, c);
            const float b1 = s1, b2 = s2;
            auto sums = [&](auto clamp) {
                float2 a1 = make_float2(b1, 0.f), a2 = make_float2(b2, 0.f);
                auto pair = [&](float2 x) {
                    float2 y = lp_mul2(lp_add2(x, neg_m), cc);
                    const float2 p = make_float2(ptx::ex2(y.x), ptx::ex2(y.y));
                    if constexpr (decltype(clamp)::value) y = make_float2(fmaxf(y.x, -1e30f), fmaxf(y.y, -1e30f));
                    a2 = lp_fma2(p, y, a2);
                    return p;
                };
                // (a vector's own sum first: fewer roundings of the whole)
                auto vec = [&](const uint4 &x) {
                    if constexpr (VEC == 4) {
                        const float2 p = pair(make_float2(__uint_as_float(x.x), __uint_as_float(x.y)));
                        a1 = lp_add2(a1, lp_add2(p, pair(make_float2(__uint_as_float(x.z), __uint_as_float(x.w)))));
                    } else {
                        const float2 p = lp_add2(pair(lp_unpack<T>(x.x)), pair(lp_unpack<T>(x.y)));
                        const float2 q = lp_add2(pair(lp_unpack<T>(x.z)), pair(lp_unpack<T>(x.w)));
                        a1 = lp_add2(a1, lp_add2(p, q));
                    }
                };
                if (mine == kLpVecs && !decltype(clamp)::value) {
#pragma unroll
                    for (int i = 0; i < kLpVecs; ++i) vec(data[i * kLpThreads]);
                } else {
#pragma unroll 1
                    for (int i = 0; i < mine; ++i) vec(data[i * kLpThreads]);
                }
                s1 = a1.x + a1.y;
                s2 = a2.x + a2.y;
            };
            sums(std::false_type{});
            if (__any_sync(0xffffffffu, s2 != s2 && s1 == s1)) sums(std::true_type{});
        }
        if (first) given = token >= 0 && token < a.vocab ? lp_load<T>(r.p, token) : 0.f;
        if (!last) continue;

        // ------------------------------------------------------- the row, or its part in this run ----
        if (extra_at >= 0) {
            if (extra > m) {
                move_state(m, extra, c, s1, s2);
                m = extra;
            }
            const float y = (extra - (m == -INFINITY ? 0.f : m)) * c, p = ptx::ex2(y);
            s1 += p;
            s2 = fmaf(p, fmaxf(y, -1e30f), s2);
        }
        const float M = block_max(sm, m, warp, lane);    // (the barrier: the last candidates are there)
        move_state(m, M, c, s1, s2);
        m = M;
        warp_sums(sm, s1, s2, warp, lane);
        __syncthreads();
        block_sums(sm, s1, s2);
        if (top > 0) {
            settle(k, true);
            if (tid >= kept && tid < KL_LOGPROBS_MAX_TOP) sm.list[tid] = 0;
            if (r.head + r.tail > 0) {
                // the candidates outside the vectors
                if (extra_at >= 0 && extra >= from) {
                    const uint64_t key = make_key(extra, extra_at);
                    if (key > above) sm.cand[kept + atomicAdd(&sm.added[k % 3], 1)] = key;
                }
                __syncthreads();
                const int n = kept + sm.added[k % 3];
                if (n > kept) rank_keys(sm, n, top, tid);
            }
            __syncthreads();
            if (tid < 3) sm.added[tid] = 0;
        }
        const int64_t row0 = (int64_t)row * a.chunks;
        const int c0 = runs.of(row0);
        const int parts = runs.of(row0 + a.chunks - 1) - c0 + 1;
        if (parts > 1) {
            const size_t at = part_slot(blockIdx.x, c0);
            if (warp == 0) {
                if (lane == 0) a.part[at] = make_float4(m, s1, s2, 0.f);
                if (lane < top) a.part_top[at * top + lane] = sm.list[lane];
                __syncwarp();
                if (lane == 0) sm.is_last = arrive_last(a.counters + c0, parts);
            }
            __syncthreads();
            if (!sm.is_last) continue;
            join_parts(sm, a, c0, parts, c, m, s1, s2);
        }
        finish_row<T>(sm, a, r.p, row, m, s1, s2, token, given);
        __syncthreads();
    }
    // Copies still in flight land before the CTA's shared memory goes away: the lost chunk's and those behind it.
    __syncthreads();
    if (tid == 0 && sm.lost != INT_MAX) {
        raise_flag(a.err, KL_FLAG_TIMEOUT);
        const int k = sm.lost - 1;
        for (int i = k; i < steps && i < k + kLpStages; ++i) wait_slow(sm, i, kDefaultWaitNs);
    }
}

// Vectors per chunk when a row of `vecs` vectors is cut into `chunks`: a multiple of the threads, so that only
// a row's last chunk leaves some of them without a vector.
int chunk_vectors(int64_t vecs, int chunks) {
    const int64_t each = (vecs + chunks - 1) / chunks;
    return (int)((each + kLpThreads - 1) / kLpThreads * kLpThreads);
}

// Chunks of a row of `vecs` 16-byte vectors: of kLpChunk vectors, or smaller (kLpMinChunk) while every CTA still
// has one chunk at most (427 rows of 5428 bf16 logits, 8 alternatives: a chunk each 7.7 us, two 10.4).
int chunks_of(int64_t rows, int64_t vecs) {
    const int64_t ctas = logprob_ctas();
    int64_t n = (vecs + kLpChunk - 1) / kLpChunk;
    if (rows * n < ctas) {
        const int64_t want = ctas / rows, most = (vecs + kLpMinChunk - 1) / kLpMinChunk;
        n = max(n, min(want, most));
    }
    if (n < 1) return 1;
    const int64_t each = chunk_vectors(vecs, (int)n);
    return (int)max((vecs + each - 1) / each, (int64_t)1);
}

}  // namespace

int logprob_ctas() { return kLpCtas * device_sm_count(); }

int logprob_chunks(int rows, int vocab, kl_dtype dtype) {
    return chunks_of(rows, vocab / (dtype == KL_FP32 ? 4 : 8));
}

cudaError_t launch_logprobs(const LogprobArgs &a) {
    const int per_chunk = chunk_vectors(a.vocab / (a.dtype == KL_FP32 ? 4 : 8), a.chunks);
    const int64_t total = (int64_t)a.rows * a.chunks, ctas = logprob_ctas();
    const auto kernel = a.dtype == KL_FP32 ? logprobs_kernel<float> : logprobs_kernel<uint16_t>;
    static PerDeviceOnce once[2];
    const cudaError_t e = once[a.dtype == KL_FP32].run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(LogprobSmem));
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(total < ctas ? total : ctas));
    cfg.blockDim = dim3(kLpThreads);
    cfg.dynamicSmemBytes = sizeof(LogprobSmem);
    cfg.stream = a.stream;
    const OverlapAttr overlap(cfg);
    return cudaLaunchKernelEx(&cfg, kernel, a, per_chunk);
}

}  // namespace kl
