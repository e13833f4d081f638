// Log probabilities of given tokens, the entropy and the largest logits of rows of logits, in one pass.
//
// With x = scale * logits, z = sum_j exp(x_j) and p = exp(x) / z:
//   logprob(t) = x_t - log z,   H = - sum_j p_j log p_j = log z - sum_j p_j x_j,
// and the `top` largest logits, ties to the lowest index. A row is cut into chunks of up to 2048 16-byte
// vectors, one CTA each: the chunk stays in registers (8 vectors per thread, all loads in flight at
// once), so that the maximum, the sums against it, and the selection read HBM once. The CTA that
// finishes last joins the row's chunks. Bound by HBM: 6 to 7 instructions per logit leave the issue
// slots two thirds busy at full bandwidth.
//
// Sums are held in fp32 against the chunk's largest logit m: y = (x - m) scale log2 e (the difference
// first, so that rows of huge or lowest values neither overflow nor cancel), s1 = sum 2^y, s2 = sum y 2^y.
// Chunks join as softmax states do: with d = (m_c - M) scale log2 e, s1 += 2^d s1_c,
// s2 += 2^d (s2_c + d s1_c); then log z = log2(s1) ln 2 above scale * M and H = (log2 s1 - s2 / s1) ln 2.
//
// Selection: a logit among the row's largest is among its chunk's. Each thread has the maximum of its own
// logits; with `top` threads' maxima known to be >= t, so are `top` logits, and only logits above such a
// bound t go on: t is the larger of (the smallest, over the 8 warps, of the ceil(top / 8)-th largest
// maximum) and (the largest over the warps of the top-th). Those few are ranked by counting; if they are
// fewer than `top`, the rest are the lowest-indexed logits equal to t.
#include <math.h>

#include "kl_internal.cuh"

namespace kl {
namespace {

constexpr int kLpThreads = 256, kLpWarps = 8;
constexpr int kLpVecs = 8;                               // 16-byte vectors per thread
constexpr int kLpChunk = kLpThreads * kLpVecs;           // vectors per chunk, at most
constexpr int kLpCap = 1024;                             // candidates ranked in shared memory
static_assert(KL_LOGPROBS_MAX_TOP <= 32, "a warp's sorted maxima bound the selection");

struct LogprobSmem {
    uint64_t cand[kLpCap];
    uint64_t list[KL_LOGPROBS_MAX_TOP];                  // keys, largest first
    float wmax[kLpWarps], wnth[kLpWarps], wtop[kLpWarps];
    float s1[kLpWarps], s2[kLpWarps];
    uint64_t wkey[kLpWarps];
    int wcount[kLpWarps];
    int count;
    int is_last;
};

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

__device__ __forceinline__ float lp_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Element e of a 16-byte vector.
template <typename T>
__device__ __forceinline__ float lp_get(const uint4 &v, int e) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return (e & 1) ? bf16hi(w[e >> 1]) : bf16lo(w[e >> 1]);
}

template <typename T>
__device__ __forceinline__ float lp_load(const void *row, int idx) {
    if constexpr (sizeof(T) == 4) return static_cast<const float *>(row)[idx];
    else return bf16lo((uint32_t)static_cast<const uint16_t *>(row)[idx]);
}

// Sum over the block of one value per thread (every thread gets it).
__device__ __forceinline__ float block_sum(float v, float *red, int warp, int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) red[warp] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kLpWarps; ++w) t += red[w];
    return t;
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

template <typename T>
__global__ void __launch_bounds__(kLpThreads, 4) logprobs_kernel(const LogprobArgs a, const int per_chunk) {
    constexpr int VEC = 16 / sizeof(T);                  // logits per vector
    __shared__ LogprobSmem sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks;
    const char *rp = static_cast<const char *>(a.logits) + (size_t)row * a.stride * sizeof(T);
    // vectors from the 16-byte boundary at or before the row's start; logit i is element off + i
    const int off = (int)((reinterpret_cast<uintptr_t>(rp) & 15) / sizeof(T));
    const int64_t v0 = (int64_t)chunk * per_chunk;
    const float c = a.scale * kLog2e;
    const int top = a.top;
    if (tid < KL_LOGPROBS_MAX_TOP) sm.list[tid] = 0;
    if (tid == 0) sm.count = 0;
    grid_dep_wait();
    grid_dep_launch();

    uint4 v[kLpVecs];
    // logits outside the row (the edges' other elements, vectors past the end) count as -inf
    auto index_of = [&](int i, int e) -> int64_t { return (v0 + i * kLpThreads + tid) * VEC + e - off; };
#pragma unroll
    for (int i = 0; i < kLpVecs; ++i) {
        const int64_t j0 = index_of(i, 0);
        const bool inside = i * kLpThreads + tid < per_chunk;
        if (inside && j0 >= 0 && j0 + VEC <= a.vocab) {
            v[i] = __ldcs(reinterpret_cast<const uint4 *>(rp + j0 * (int64_t)sizeof(T)));
        } else {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
            if (inside && j0 < a.vocab)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int64_t j = j0 + e;
                    if (j < 0 || j >= a.vocab) continue;
                    if constexpr (sizeof(T) == 4) {
                        w[e] = reinterpret_cast<const uint32_t *>(rp)[j];
                    } else {
                        const uint32_t x = reinterpret_cast<const uint16_t *>(rp)[j];
                        w[e >> 1] = (e & 1) ? (w[e >> 1] & 0xffffu) | x << 16 : (w[e >> 1] & 0xffff0000u) | x;
                    }
                }
            v[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    float tmax = -INFINITY;                              // (NaN does not take part)
#pragma unroll
    for (int i = 0; i < kLpVecs; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) tmax = fmaxf(tmax, lp_get<T>(v[i], e));

    // the block's maximum, and the warps' bounds for the selection: the maxima sorted over the lanes
    float s = tmax;
    if (top > 0) {
#pragma unroll
        for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
            for (int j = k >> 1; j > 0; j >>= 1) {
                const float o = __shfl_xor_sync(0xffffffffu, s, j);
                const bool larger = ((lane & j) == 0) == ((lane & k) == 0);   // descending overall
                s = larger ? fmaxf(s, o) : fminf(s, o);
            }
        if (lane == (top + kLpWarps - 1) / kLpWarps - 1) sm.wnth[warp] = s;
        if (lane == top - 1) sm.wtop[warp] = s;
    } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, o));
    }
    if (lane == 0) sm.wmax[warp] = s;
    __syncthreads();
    float m = sm.wmax[0], bound = -INFINITY;
#pragma unroll
    for (int w = 1; w < kLpWarps; ++w) m = fmaxf(m, sm.wmax[w]);
    if (top > 0) {
        float lowest = sm.wnth[0];
        bound = sm.wtop[0];
#pragma unroll
        for (int w = 1; w < kLpWarps; ++w) {
            lowest = fminf(lowest, sm.wnth[w]);
            bound = fmaxf(bound, sm.wtop[w]);
        }
        bound = fmaxf(bound, lowest);
    }

    // the sums against the chunk's maximum (0 where nothing is above -inf)
    const float mr = m == -INFINITY ? 0.f : m;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < kLpVecs; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float y = (lp_get<T>(v[i], e) - mr) * c;
            const float p = lp_ex2(y);
            s1 += p;
            s2 = fmaf(p, fmaxf(y, -1e30f), s2);          // (a weight of 0 at y = -inf adds 0)
        }
    s1 = block_sum(s1, sm.s1, warp, lane);
    s2 = block_sum(s2, sm.s2, warp, lane);

    if (top > 0) {
        // logits above the bound
        if (tmax > bound) {
#pragma unroll
            for (int i = 0; i < kLpVecs; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float x = lp_get<T>(v[i], e);
                    if (x > bound) {
                        const int at = atomicAdd(&sm.count, 1);
                        if (at < kLpCap) sm.cand[at] = make_key(x, (int)index_of(i, e));
                    }
                }
        }
        __syncthreads();
        const int n = sm.count;
        if (n <= kLpCap) {
            rank_keys(sm, n, top, tid);
            // too few: the first logits equal to the bound, in order
            int have = n;
#pragma unroll
            for (int i = 0; i < kLpVecs; ++i) {
                if (have >= top) continue;               // (uniform: `have` is the block's)
                int mine = 0;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int64_t j = index_of(i, e);
                    mine += lp_get<T>(v[i], e) == bound && j >= 0 && j < a.vocab &&
                            i * kLpThreads + tid < per_chunk;
                }
                int before = mine;                       // inclusive prefix over the warp
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int x = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += x;
                }
                if (lane == 31) sm.wcount[warp] = before;
                __syncthreads();
                int at = have + before - mine, all = 0;
#pragma unroll
                for (int w = 0; w < kLpWarps; ++w) {
                    if (w < warp) at += sm.wcount[w];
                    all += sm.wcount[w];
                }
                if (mine > 0)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const int64_t j = index_of(i, e);
                        if (lp_get<T>(v[i], e) == bound && j >= 0 && j < a.vocab) {
                            if (at < top) sm.list[at] = make_key(bound, (int)j);
                            ++at;
                        }
                    }
                have += all;
                __syncthreads();
            }
        } else {
            take_keys(sm, top, tid, [&](uint64_t prev) {
                uint64_t k = 0;
#pragma unroll
                for (int i = 0; i < kLpVecs; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float x = lp_get<T>(v[i], e);
                        if (x > bound) {
                            const uint64_t y = make_key(x, (int)index_of(i, e));
                            if (y < prev && y > k) k = y;
                        }
                    }
                return k;
            });
        }
        __syncthreads();
    }

    if (a.chunks > 1) {
        const size_t slot = (size_t)row * a.chunks + chunk;
        if (tid == 0) a.part[slot] = make_float4(m, s1, s2, 0.f);
        if (tid < top) a.part_top[slot * top + tid] = sm.list[tid];
        __syncthreads();
        if (tid == 0) sm.is_last = arrive_last(a.counters + row, a.chunks);
        __syncthreads();
        if (!sm.is_last) return;
        // join the row's chunks
        const float4 *part = a.part + (size_t)row * a.chunks;
        float M = -INFINITY;
        for (int i = tid; i < a.chunks; i += kLpThreads) M = fmaxf(M, __ldcg(part + i).x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        if (lane == 0) sm.wmax[warp] = M;
        if (tid == 0) sm.count = 0;
        __syncthreads();
        m = sm.wmax[0];
#pragma unroll
        for (int w = 1; w < kLpWarps; ++w) m = fmaxf(m, sm.wmax[w]);
        s1 = s2 = 0.f;
        for (int i = tid; i < a.chunks; i += kLpThreads) {
            const float4 q = __ldcg(part + i);
            const float d = (q.x - m) * c, f = lp_ex2(d);
            // (a chunk of -inf has s1 = 0 and d = NaN or -inf; one so low that f is 0 adds nothing but NaN)
            if (q.y != 0.f && (f != 0.f || q.y != q.y)) {
                s1 = fmaf(f, q.y, s1);
                s2 = fmaf(f, fmaf(d, q.y, q.z), s2);
            }
        }
        s1 = block_sum(s1, sm.s1, warp, lane);
        s2 = block_sum(s2, sm.s2, warp, lane);
        if (top > 0) {
            // every chunk's last key is a bound; the largest of them leaves few
            const uint64_t *keys = a.part_top + (size_t)row * a.chunks * top;
            uint64_t k = 0;
            for (int i = tid; i < a.chunks; i += kLpThreads) {
                const uint64_t x = __ldcg(keys + (size_t)i * top + top - 1);
                if (x > k) k = x;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const uint64_t x = __shfl_xor_sync(0xffffffffu, k, o);
                if (x > k) k = x;
            }
            if (lane == 0) sm.wkey[warp] = k;
            if (tid < KL_LOGPROBS_MAX_TOP) sm.list[tid] = 0;
            __syncthreads();
            k = 0;
#pragma unroll
            for (int w = 0; w < kLpWarps; ++w)
                if (sm.wkey[w] > k) k = sm.wkey[w];
            const int64_t all = (int64_t)a.chunks * top;
            for (int64_t i = tid; i < all; i += kLpThreads) {
                const uint64_t x = __ldcg(keys + i);
                if (x != 0 && x >= k) {
                    const int at = atomicAdd(&sm.count, 1);
                    if (at < kLpCap) sm.cand[at] = x;
                }
            }
            __syncthreads();
            const int n = sm.count;
            if (n <= kLpCap) {
                rank_keys(sm, n, top, tid);
            } else {
                take_keys(sm, top, tid, [&](uint64_t prev) {
                    uint64_t best = 0;
                    for (int64_t i = tid; i < all; i += kLpThreads) {
                        const uint64_t x = __ldcg(keys + i);
                        if (x < prev && x > best) best = x;
                    }
                    return best;
                });
            }
            __syncthreads();
        }
    }

    // Results. A row of -inf alone has no distribution: log probabilities of -inf, entropy 0. A NaN or
    // +inf logit makes the sums, and with them everything but the ids, NaN.
    const bool none = s1 == 0.f;
    const float lz = log2f(s1);
    auto logprob = [&](float x) { return none ? -INFINITY : ((x - m) * c - lz) * kLn2; };
    if (tid == 0 && a.entropy) a.entropy[row] = none ? 0.f : (lz - s2 / s1) * kLn2;
    if (tid == 0 && s1 != s1) raise_flag(a.err, KL_FLAG_RANGE);
    for (int i = tid; i < a.per_row; i += kLpThreads) {
        const int id = a.tokens[(size_t)row * a.per_row + i];
        float lp = 0.f;                                  // -1: no token
        if (id >= 0 && id < a.vocab) {
            lp = logprob(lp_load<T>(rp, id));
        } else if (id != -1) {
            lp = NAN;
            raise_flag(a.err, KL_FLAG_BAD_TOKEN);
        }
        a.logprobs[(size_t)row * a.per_row + i] = lp;
    }
    if (tid < top) {
        const uint64_t k = sm.list[tid];
        a.top_ids[(size_t)row * top + tid] = k ? key_index(k) : -1;
        a.top_logprobs[(size_t)row * top + tid] = k ? logprob(key_value(k)) : NAN;
    }
}

// 16-byte vectors that a row of `vocab` logits can touch, whatever its alignment.
int64_t row_vectors(int vocab, int vec, bool aligned) {
    return ((int64_t)vocab + (aligned ? 0 : vec - 1) + vec - 1) / vec;
}

}  // namespace

int logprob_chunks(int vocab, kl_dtype dtype) {
    return (int)((row_vectors(vocab, dtype == KL_FP32 ? 4 : 8, false) + kLpChunk - 1) / kLpChunk);
}

cudaError_t launch_logprobs(const LogprobArgs &a) {
    LogprobArgs la = a;
    const int es = a.dtype == KL_FP32 ? 4 : 2;
    const bool aligned = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 &&
                         (a.rows == 1 || (a.stride * es) % 16 == 0);
    const int64_t vecs = row_vectors(a.vocab, 16 / es, aligned);
    la.chunks = (int)((vecs + kLpChunk - 1) / kLpChunk);
    const int per_chunk = (int)((vecs + la.chunks - 1) / la.chunks);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)a.rows * la.chunks));
    cfg.blockDim = dim3(kLpThreads);
    cfg.stream = a.stream;
    const OverlapAttr overlap(cfg);
    return a.dtype == KL_FP32 ? cudaLaunchKernelEx(&cfg, logprobs_kernel<float>, la, per_chunk)
                              : cudaLaunchKernelEx(&cfg, logprobs_kernel<uint16_t>, la, per_chunk);
}

}  // namespace kl
