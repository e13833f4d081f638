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
// logits; with `top` threads' maxima known to be >= t, so are `top` logits, and only logits from such a
// bound t on are candidates: t is the larger of (the smallest, over the 8 warps, of the ceil(top / 8)-th largest
// maximum) and (the largest over the warps of the top-th). Those few are ranked by counting. Masked and tied rows,
// where the bound leaves too few or too many, read their chunk a second time.
#include <float.h>
#include <math.h>

#include <type_traits>

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

// The registers of the chunk as the compiler may not know them from before: each phase unpacks them anew
// instead of keeping 64 unpacked logits (which spilled).
template <int N>
__device__ __forceinline__ void lp_forget(uint32_t (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(w[i]));
}

template <typename T>
__device__ __forceinline__ float lp_load(const void *row, int idx) {
    if constexpr (sizeof(T) == 4) return static_cast<const float *>(row)[idx];
    else return bf16lo((uint32_t)static_cast<const uint16_t *>(row)[idx]);
}

// Sum over each warp of s1 and s2, to the warps' slots (block_sums() after the next barrier).
__device__ __forceinline__ void warp_sums(LogprobSmem &sm, float s1, float s2, int warp, int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s1 += __shfl_xor_sync(0xffffffffu, s1, o);
        s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    if (lane == 0) {
        sm.s1[warp] = s1;
        sm.s2[warp] = s2;
    }
}
__device__ __forceinline__ void block_sums(const LogprobSmem &sm, float &s1, float &s2) {
    s1 = s2 = 0.f;
#pragma unroll
    for (int w = 0; w < kLpWarps; ++w) {
        s1 += sm.s1[w];
        s2 += sm.s2[w];
    }
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
    const int v0 = chunk * per_chunk;
    const float c = a.scale * kLog2e;
    const int top = a.top;
    if (tid < KL_LOGPROBS_MAX_TOP) sm.list[tid] = 0;
    if (tid == 0) sm.count = 0;
    grid_dep_wait();
    grid_dep_launch();

    // logit of word k of vector i (its lower half)
    auto index_of = [&](int i, int k) { return (v0 + i * kLpThreads + tid) * VEC + k * (VEC / 4) - off; };
    // Logits outside the row (the edges' other elements, vectors past the end) count as -inf.
    uint32_t v[4 * kLpVecs];
    bool edge = false;                                   // the thread holds some of those
#pragma unroll
    for (int i = 0; i < kLpVecs; ++i) {
        const int j0 = index_of(i, 0);
        const bool inside = i * kLpThreads + tid < per_chunk;
        if (inside && j0 >= 0 && j0 + VEC <= a.vocab) {
            const uint4 x = __ldcs(reinterpret_cast<const uint4 *>(rp + (int64_t)j0 * (int)sizeof(T)));
            v[4 * i] = x.x;
            v[4 * i + 1] = x.y;
            v[4 * i + 2] = x.z;
            v[4 * i + 3] = x.w;
        } else {
            edge = true;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[4 * i + k] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
            if (inside && j0 < a.vocab)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int j = j0 + e;
                    if (j < 0 || j >= a.vocab) continue;
                    if constexpr (sizeof(T) == 4) {
                        v[4 * i + e] = reinterpret_cast<const uint32_t *>(rp)[j];
                    } else {
                        uint32_t &w = v[4 * i + (e >> 1)];
                        const uint32_t x = reinterpret_cast<const uint16_t *>(rp)[j];
                        w = (e & 1) ? (w & 0xffffu) | x << 16 : (w & 0xffff0000u) | x;
                    }
                }
        }
    }
    float tmax;                                          // (NaN does not take part)
    if constexpr (sizeof(T) == 4) {
        tmax = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4 * kLpVecs; ++i) tmax = fmaxf(tmax, __uint_as_float(v[i]));
    } else {
        uint32_t t = 0xff80ff80u;
#pragma unroll
        for (int i = 0; i < 4 * kLpVecs; ++i) t = lp_max_bf16(t, v[i]);
        tmax = fmaxf(bf16lo(t), bf16hi(t));
    }

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

    // logits from the bound on (above it, where it is -inf)
    lp_forget(v);
    const float from = bound == -INFINITY ? -FLT_MAX : bound;
    if (top > 0 && tmax >= from) {
#pragma unroll
        for (int i = 0; i < 4 * kLpVecs; ++i) {
            const float2 x = lp_unpack<T>(v[i]);
            if (fmaxf(x.x, x.y) >= from) {
                const int j = index_of(i >> 2, i & 3);
                if (x.x >= from) {
                    const int at = atomicAdd(&sm.count, 1);
                    if (at < kLpCap) sm.cand[at] = make_key(x.x, j);
                }
                if (x.y >= from) {
                    const int at = atomicAdd(&sm.count, 1);
                    if (at < kLpCap) sm.cand[at] = make_key(x.y, j + 1);
                }
            }
        }
        lp_forget(v);
    }

    // The sums against the chunk's maximum (0 where nothing is above -inf). A weight of 0 at y = -inf has
    // to add 0 to s2, not NaN: the clamp for that is left out where the thread's logits do without.
    const float mr = m == -INFINITY ? 0.f : m;
    const float2 neg_m = make_float2(-mr, -mr), cc = make_float2(c, c);
    float s1, s2;
    auto sums = [&](auto clamp) {
        float2 a1 = make_float2(0.f, 0.f), a2 = a1;
#pragma unroll
        for (int i = 0; i < 4 * kLpVecs; i += VEC == 4 ? 2 : 1) {
            float2 x;
            if constexpr (VEC == 4) x = make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1]));
            else x = lp_unpack<T>(v[i]);
            float2 y = lp_mul2(lp_add2(x, neg_m), cc);
            const float2 p = make_float2(lp_ex2(y.x), lp_ex2(y.y));
            if constexpr (decltype(clamp)::value) y = make_float2(fmaxf(y.x, -1e30f), fmaxf(y.y, -1e30f));
            a1 = lp_add2(a1, p);
            a2 = lp_fma2(p, y, a2);
        }
        s1 = a1.x + a1.y;
        s2 = a2.x + a2.y;
    };
    if (!edge) sums(std::false_type{});
    if (edge || (s2 != s2 && s1 == s1)) {
        lp_forget(v);
        sums(std::true_type{});
    }
    warp_sums(sm, s1, s2, warp, lane);
    __syncthreads();
    block_sums(sm, s1, s2);

    if (top > 0) {
        int n = sm.count;
        if (n >= top && n <= kLpCap) {
            rank_keys(sm, n, top, tid);
        } else {
            // Too few (the bound is -inf) or too many (ties at the bound, or a chunk whose large logits lie
            // in a few threads): the chunk is read once more.
            const int j0 = max(0, v0 * VEC - off), j1 = min(a.vocab, (v0 + per_chunk) * VEC - off);
            __syncthreads();
            if (n > kLpCap) {
                if (tid == 0) sm.count = 0;
                __syncthreads();
                for (int j = j0 + tid; j < j1; j += kLpThreads) {
                    const float x = lp_load<T>(rp, j);
                    if (x > bound) {
                        const int at = atomicAdd(&sm.count, 1);
                        if (at < kLpCap) sm.cand[at] = make_key(x, j);
                    }
                }
                __syncthreads();
                n = sm.count;
            }
            if (n <= kLpCap) {
                rank_keys(sm, n, top, tid);
                // then the first logits equal to the bound, in order
                for (int jb = j0; jb < j1 && n < top; jb += kLpThreads) {
                    const int j = jb + tid;
                    const bool mine = j < j1 && lp_load<T>(rp, j) == bound;
                    const unsigned votes = __ballot_sync(0xffffffffu, mine);
                    if (lane == 0) sm.wcount[warp] = __popc(votes);
                    __syncthreads();
                    int at = n + __popc(votes & ((1u << lane) - 1));
#pragma unroll
                    for (int w = 0; w < kLpWarps; ++w) {
                        if (w < warp) at += sm.wcount[w];
                        n += sm.wcount[w];
                    }
                    if (mine && at < top) sm.list[at] = make_key(bound, j);
                    __syncthreads();
                }
            } else {
                take_keys(sm, top, tid, [&](uint64_t prev) {
                    uint64_t k = 0;
                    for (int j = j0 + tid; j < j1; j += kLpThreads) {
                        const float x = lp_load<T>(rp, j);
                        const uint64_t y = x > bound ? make_key(x, j) : 0;
                        if (y < prev && y > k) k = y;
                    }
                    return k;
                });
            }
        }
        __syncthreads();
    }

    if (a.chunks > 1) {
        const size_t slot = (size_t)row * a.chunks + chunk;
        if (warp == 0) {
            if (lane == 0) a.part[slot] = make_float4(m, s1, s2, 0.f);
            if (lane < top) a.part_top[slot * top + lane] = sm.list[lane];
            __syncwarp();
            if (lane == 0) sm.is_last = arrive_last(a.counters + row, a.chunks);
        }
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
        warp_sums(sm, s1, s2, warp, lane);
        __syncthreads();
        block_sums(sm, s1, s2);
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
