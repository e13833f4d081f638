// Internal declarations shared by the translation units of libkeyless.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "keyless.h"

namespace kl {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr uint64_t kDefaultWaitNs = 1000000000ull;   // about one second
// Wait limits below this are kept exactly: the decodes are then launched in a variant whose
// waits poll without suspending (a suspended try_wait can outlast such a limit).
constexpr uint64_t kExactWaitNs = 100000ull;

// The pipeline-wait limit in force (kl_set_wait_timeout_ns; the default unless set).
uint64_t current_wait_ns();

// Geometry of one decode call, resolved on the host.
struct Geometry {
    int B, Hq, Hkv, G, D, P, num_pages, max_pages, wr_per_qh;
    float scale;       // lambda / sqrt(d_k)
    int S;             // split count
    int chunk;         // tokens per split (a multiple of 128)
    int spc = 1;       // splits per CTA of the tensor-core decode (consecutive, same (b, g))
    // CTAs per (run of splits, b, g) and query rows of one CTA: as resolved, blocks of up to 8 query
    // heads (qbox: min(G, 8), or 2 G with two value heads), which the split plan and the workspace
    // count on; the wide decode's launcher sets its own blocks of 16 or 32 and spc for them.
    int nhb = 1;
    int qbox = 8;
    int vpc = 1;       // value heads per CTA of the tensor-core decode: 2 at head dim 64 (the
                       // two heads' rows side by side in one 128-wide tile), else 1
};

// Arguments of a decode launch (keyless or the standard K+V comparison).
struct DecodeArgs {
    Geometry geo;
    const uint16_t *q;        // [B][Hq][D] bf16
    const uint16_t *w_r;      // [Hw][D][D] bf16 (keyless only)
    // Pre-routed queries (tensor-core kernel only): when set, q and w_r are unused and the
    // kernel scores with q_routed[b][h][:] (fp32, [B][Hq][D]) as the routed query, e.g. the
    // absorbed query of a latent value-only cache.
    const float *q_routed;
    const uint16_t *k_cache;  // [num_pages][Hkv][P][D] bf16 (standard only)
    const uint16_t *v_cache;  // [num_pages][Hkv][P][D] bf16
    const int32_t *block_table;
    const int32_t *seq_lens;
    // Fused append (kl_decode_step): when v_new is set, the CTA whose split holds row
    // positions[b] writes v_new[b][g] there (into cache_rw, the value cache) before it reads it.
    const uint16_t *v_new;            // [B][Hkv][D] bf16 or nullptr
    const int32_t *positions;         // [B]
    uint16_t *cache_rw;
    // FP8 step (kl_decode_step_fp8): the row positions[b] of the code and scale caches receives
    // v_new[b][g] quantized, in the same way, from the CTA whose split holds it.
    uint8_t *codes_rw = nullptr;
    float *scales_rw = nullptr;
    float *part_o;            // [B][Hq][S][D]   split states (unless direct_out)
    float *part_ml;           // [B][Hq][S][2]
    void *out;                // [B][Hq][D]
    bool direct_out;          // true: S == 1 and the CTA writes `out` itself (no split states)
    bool merge_inside;        // true: the last split of each (b, g) merges the split states
                              // into `out` (tensor-core kernel), using the workspace counters
    unsigned int *counters;   // [B][Hkv][nhb] arrivals of the current call (zero between calls)
    kl_dtype out_dtype;
    int32_t *err;
    cudaStream_t stream;
    // Limit of each pipeline wait of the tensor-core decodes (ns); the drains of a CTA that gave
    // up keep the full default so that its copies and MMAs complete before it exits.
    uint64_t wait_ns = kDefaultWaitNs;
    // Latent path, behind the absorbed-query kernel (which signals once everything ahead of it in
    // the stream has completed): the CTAs set up and fill their ring of cache tiles at once,
    // every role then sleeps in grid_dep_wait until that kernel has finished (the compute warps
    // before reading q_routed; a CTA with an empty run before it ends).
    bool pdl = false;
    // The wide decode's tree form (kl_tree_attention): sequence b's drafts are rows cu_q[b] .. of q and out.
    struct {
        const int32_t *cu_q = nullptr, *parents = nullptr;
        int total_q = 0, max_q = 1;
    } tree;
    // Its forms for consecutive positions (kl_window_attention, kl_attention_weights; tree.cu_q, total_q and max_q
    // as above): a block is rpb positions of hp heads, a value head's nhg blocks of heads next to each other.
    // CTAs: the first `whole` units (b, g, block of rows) in one run each, the others in runs of geo.spc splits;
    // states and sums of the units behind those alone.
    struct {
        int hp = 1, rpb = 1, nhg = 1;
        int whole = 0, two_per_sm = 0;
        int window = 0, sinks = 0;
        // kl_attention_weights: the scores times log2 e, [B][Hkv][nhb][rows][pitch], each run's {maximum (of
        // these), sum}, [B][Hkv][nhb][16][S], and the longest sequence
        int rows = 1, stride = 0;
        int64_t pitch = 0;
        float *scores = nullptr;
        float2 *stats = nullptr;
        const float *weights = nullptr;   // [B][Hkv][stride]; not read where decay is 0
        float decay = 0.f;
        float *new_weights = nullptr;     // [B][Hkv][stride]
    } causal;
};

// Arguments of a kl_evict launch. The workspace holds kEvictUnitBytes for every sequence and value head, and a word and 16
// numbers for every 16 chunks of 32 rows or more.
constexpr int kEvictUnitBytes = 16, kEvictMarkBytes = 4 + 16 * 4;
inline int kl_evict_marks(int budget) { return budget / 512 + 1; }
struct EvictArgs {
    Geometry geo;             // S and chunk unused
    const float *weights;     // [B][Hkv][stride]
    int stride, budget, sinks, recent;
    const int32_t *block_table, *new_table;
    const int32_t *seq_lens;
    uint16_t *v_cache;
    float *new_weights;       // [B][Hkv][stride]
    int32_t *kept;            // [B][Hkv][budget]
    int32_t *new_lens;        // [B]
    void *workspace;
    int32_t *err;
    uint64_t wait_ns;         // bound of a wait for other CTAs' reads
    cudaStream_t stream;
};

// Arguments of a chunked-prefill launch (kl_prefill_attention). Sequence b's query rows are
// cu_q[b] .. cu_q[b + 1] - 1 of q / out ([total_q][Hq][D]); they are the last n_b rows of its
// seq_lens[b] cached rows, so query row i sits at position seq_lens[b] - n_b + i.
struct PrefillArgs {
    Geometry geo;             // S and chunk unused
    int total_q;              // rows of q and out
    int max_q;                // host bound on n_b (grid sizing)
    // Layout (set by the launcher, plan_prefill): a block of 128 rows holds hp heads of one value head's group,
    // rpb query rows each; a cluster of cs CTAs splits a block's cache tiles.
    int hp = 1, rpb = 128, cs = 1;
    int window = 0, sinks = 0;   // kl_window_attention (where w_r may be nullptr: q is the composed query)
    // kl_attention_weights: the scores times log2 e, [block][pitch / 4][128 rows] of four tokens each, and every CTA's
    // {maximum (of these), sum}, [block][128][8]
    int64_t pitch = 0;
    float4 *scores = nullptr;
    float2 *stats = nullptr;
    int stride = 0;
    const float *weights = nullptr;
    float decay = 0.f;
    float *new_weights = nullptr;
    const uint16_t *q;        // [total_q][Hq][D] bf16
    const uint16_t *w_r;      // [Hw][D][D] bf16
    const uint16_t *v_cache;  // [num_pages][Hkv][P][D] bf16
    const int32_t *block_table;
    const int32_t *seq_lens;
    const int32_t *cu_q;      // [B + 1]
    void *out;                // [total_q][Hq][D]
    kl_dtype out_dtype;
    int32_t *err;
    cudaStream_t stream;
};

// How the line of all units is shared out among the runs: `each` to a run, one more to the first `extra`.
struct TreeShare {
    int64_t each;
    int extra, runs;
};

// A unit that lies in several runs, for the merge of its parts (written by the first run that starts inside
// it; rows 0: none).
struct TreeMerge {
    int64_t unit0;            // its start on the line of all units
    TreeShare share;
    int tiles, step;          // its tiles, and what cuts fall on multiples of
    int last;                 // the last run that holds some of the unit
    int row0, rows, h, hn;    // its drafts (rows of q and out) and heads
};

// Arguments of a tree-attention launch (kl_tree_attention). Sequence b's drafts are rows cu_q[b] ..
// cu_q[b + 1] - 1 of q / out ([total_q][Hq][D]), its last n_b cached rows.
struct TreeArgs {
    Geometry geo;             // S and chunk unused
    int total_q;              // rows of q and out
    int max_q;                // host bound on n_b
    int hp, rpb, ctas;        // layout (plan_tree)
    int start, run, whole;    // ... in tiles
    int num_splits;           // most parts of a unit; 0: no such limit
    const uint16_t *q;        // [total_q][Hq][D] bf16
    const uint16_t *w_r;      // [Hw][D][D] bf16, or nullptr: q is the composed query
    const uint16_t *v_cache;  // [num_pages][Hkv][P][D] bf16
    const int32_t *block_table;
    const int32_t *seq_lens;
    const int32_t *cu_q;      // [B + 1]
    const int32_t *parents;   // [total_q]
    TreeMerge *merge;         // [ctas]
    uint8_t *states;          // [ctas][2] states of kTreeStateBytes
    void *out;                // [total_q][Hq][D]
    kl_dtype out_dtype;
    uint64_t wait_ns;         // bound of the pipeline's waits (kl_set_wait_timeout_ns)
    int32_t *err;
    cudaStream_t stream;
};

// A segment, the part of a unit (sequence b, its block `unit`) that lies in a run: from tile0 on.
struct TreeSegment {
    int64_t unit0;                // the unit's start on the line of all units
    int b, unit, tile0;
    int q0, n, L, tiles, units;   // of the sequence: drafts, length, tiles per unit, units
};

// A unit's block: value head g, drafts m0 .. m0 + rows - 1, query heads h .. h + hn - 1.
struct TreeBlock {
    int g, m0, rows, h, hn;
};
__device__ __forceinline__ TreeBlock tree_block(const TreeArgs &a, const TreeSegment &s) {
    const int nhg = (a.geo.G + a.hp - 1) / a.hp, nm = (s.n + a.rpb - 1) / a.rpb;
    const int hg = s.unit % nhg, rest = s.unit / nhg;
    TreeBlock k;
    k.g = rest / nm;
    k.m0 = rest % nm * a.rpb;
    k.rows = min(a.rpb, s.n - k.m0);
    k.h = k.g * a.geo.G + hg * a.hp;
    k.hn = min(a.hp, a.geo.G - hg * a.hp);
    return k;
}

// Arguments of a kl_token_logprobs launch.
struct LogprobArgs {
    int rows;                 // T
    int vocab;                // V
    int64_t stride;           // elements between two rows of logits
    const void *logits;       // [T][stride], the first V of each row
    kl_dtype dtype;
    float scale;
    float c_error;            // (scale log2 e - c) / c of c, its value in fp32
    const int32_t *tokens;    // [T][per_row]
    int per_row;
    int top;                  // largest logits wanted
    int chunks;               // pieces of a row (logprob_chunks)
    float *logprobs;          // [T][per_row]
    float *entropy;           // [T] or nullptr
    float *top_logprobs;      // [T][top]
    int32_t *top_ids;         // [T][top]
    // chunks > 1, for up to logprob_ctas() CTAs:
    unsigned int *counters;   // [CTA] arrivals of the row that starts there and goes on (zero between calls)
    float4 *part;             // [CTA][2] {maximum, sum, weighted sum, -}: of a row begun earlier, of that one
    uint64_t *part_top;       // [CTA][2][top] keys, largest first
    uint64_t wait_ns;         // bound of the waits for copies (kl_set_wait_timeout_ns)
    int32_t *err;
    cudaStream_t stream;
};

// bf16 bit helpers (a bf16 value is the upper half of a binary32 value).
__device__ __forceinline__ float bf16lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ void raise_flag(int32_t *err, int32_t bits) {
    if (err) atomicOr(err, bits);
}

// Arrival of one split of a (b, g) unit on its counter in the workspace: true for the last of
// the unit's n splits. The increment wraps the counter back to zero on that arrival, so the
// workspace is ready for the next call without any reset; one atomic per split, no retry.
// Acquire-release at GPU scope: it publishes the split state that this CTA's threads wrote
// before the CTA barrier that precedes it, and, for the last arrival, makes every other
// split's state visible to the threads that synchronize with this one afterwards.
__device__ __forceinline__ bool arrive_last(unsigned int *counter, int n) {
    unsigned int old;
    asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;"
                 : "=r"(old)
                 : "l"(counter), "r"((unsigned int)(n - 1))
                 : "memory");
    return old == (unsigned int)(n - 1);
}

// Programmatic dependent launch. A kernel launched with programmatic stream serialization may
// start before the kernel ahead of it in the stream has finished: grid_dep_wait() blocks the
// calling thread until that kernel has completed and its writes are visible (it returns at once
// for an ordinary launch), and grid_dep_launch() lets such a follower start once every CTA of
// the calling grid has signalled or exited.
__device__ __forceinline__ void grid_dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dep_launch() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Launch attribute of a programmatic dependent of the kernel ahead of it in the stream: of every
// kernel here but the CUDA-core decode, route_kernel and quantize_rows_kernel (ordinary launches).
// Where the kernel ahead signals early (all of these but the prefill and the latent expansion do,
// once all of their CTAs run), the launch latency and the set-up overlap its end; behind any other
// kernel it starts as an ordinary launch.
//
// Stream order holds because each kernel calls grid_dep_wait() in all threads before its first
// access to global memory (through pointers without __restrict__, whose loads the compiler may not
// move above the wait). The two kernels behind the latent path's absorbed-query kernel start
// earlier: the decode reads lengths, table and cache and appends, and the expansion reads W_post,
// before they wait. The absorbed-query kernel signals only after its own wait, so all that was
// ahead of the call has completed by then; every CTA of the decode, one with an empty run too,
// then waits for the absorbed-query kernel, and the expansion (one lane, before it reads the
// decode's output; no CTA ends without it) for the decode, so that what waits for the expansion
// waits for all three.
//
// A kernel signals only once it holds its tensor memory, so that no CTA that waits for it can take
// that. Calls one after another: 8 x 4096 tokens 20.0 -> 16.9 us, one sequence of 131072
// 49.4 -> 47.0 us, 32 x 8192 at head dim 64 86.2 -> 81.9 us, the 70B batch 604 -> 594 us.
struct OverlapAttr {
    cudaLaunchAttribute attr[1];
    explicit OverlapAttr(cudaLaunchConfig_t &cfg) {
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
};

// Launchers (each returns cudaGetLastError() of its launch).
cudaError_t launch_append(const Geometry &g, const uint16_t *v_new, const int32_t *block_table,
                          const int32_t *positions, uint16_t *v_cache, int32_t *err,
                          cudaStream_t stream);
cudaError_t launch_route(const Geometry &g, const uint16_t *q, const uint16_t *w_r, float *q_r,
                         cudaStream_t stream);
cudaError_t launch_combine(int B, int Hq, int D, int S, const float *part_o,
                           const float *part_ml, void *out, kl_dtype out_dtype,
                           cudaStream_t stream);
cudaError_t launch_decode_simt(const DecodeArgs &a, bool standard);
// Merges the split states of a finished decode into `out` unless it wrote `out` directly or
// the caller asked for the states.
cudaError_t finish_decode(const DecodeArgs &a, bool states_requested);

// Tensor-core path: whether it supports a geometry, and its launcher.
bool tc_supported(const Geometry &g, bool standard);
// Whether the tensor-core kernel can merge this geometry's split states itself.
bool tc_merge_inside(const Geometry &g, bool standard);
cudaError_t launch_decode_tc(const DecodeArgs &a, bool standard);

// Chunked prefill on the tensor cores (head_dim 128, compute capability 10.3) and the
// chunk append.
bool prefill_tc_supported(const Geometry &g);
cudaError_t launch_prefill_tc(const PrefillArgs &a);
cudaError_t launch_append_chunk(const Geometry &g, int total_q, int max_q, const uint16_t *v_new,
                                const int32_t *block_table, const int32_t *seq_lens,
                                const int32_t *cu_q, uint16_t *v_cache, int32_t *err,
                                cudaStream_t stream);

// Attention of a tree of drafted tokens (the geometry of the prefill), and the move of the accepted
// path's rows.
cudaError_t launch_tree_tc(const TreeArgs &a);
// The same by the wide decode's kernel (tree_wide_blocks): a.geo with its splits and blocks (nhb), a.tree.
cudaError_t launch_tree_wide(const DecodeArgs &a);
// Attention of consecutive positions with a sliding window, on the wide decode's kernel (a.causal) and on the
// prefill's; with all tokens before a position and each cached row's weight added up.
cudaError_t launch_window_wide(const DecodeArgs &a);
cudaError_t launch_window_tc(const PrefillArgs &a);
cudaError_t launch_attention_weights(const DecodeArgs &a);
cudaError_t launch_weights_fade(const DecodeArgs &a);   // a call without new tokens
cudaError_t launch_weights_tc(const PrefillArgs &a);
cudaError_t launch_evict(const EvictArgs &a);
cudaError_t launch_tree_commit(const Geometry &g, const int32_t *cu_q, const int32_t *path,
                               const int32_t *path_lens, int max_path, const int32_t *block_table,
                               const int32_t *seq_lens, int32_t *new_lens, uint16_t *v_cache,
                               int32_t *err, cudaStream_t stream);

// Log probabilities, entropy and largest logits of rows of logits; the pieces of a row; most CTAs of a launch.
int logprob_chunks(int rows, int vocab, kl_dtype dtype);
int logprob_ctas();
cudaError_t launch_logprobs(const LogprobArgs &a);

// FP8 value cache (E4M3 codes [num_pages][Hkv][P][D] with fp32 row scales [num_pages][Hkv][P]):
// the decode on the tensor cores (a.v_cache holds the codes; states or direct output, merged by
// the combine kernel) and the quantizing append.
cudaError_t launch_decode_fp8(const DecodeArgs &a, const float *v_scales);
cudaError_t launch_append_fp8(const Geometry &g, const uint16_t *v_new, const int32_t *block_table,
                              const int32_t *positions, uint8_t *codes, float *scales, int32_t *err,
                              cudaStream_t stream);
cudaError_t launch_quantize_fp8(size_t rows, const uint16_t *v, uint8_t *codes, float *scales,
                                cudaStream_t stream);

// Latent value-only cache (head_dim D of queries and outputs, latent width r):
// q_lat[b][h] = (q[b][h] W^R[w(h)]) W_post[h]^T and out[b][h] = o_lat[b][h] W_post[h].
// Tensor-core kernels (D 64 or 128, r 128); the expansion is launched as a programmatic
// dependent of the kernel ahead of it.
cudaError_t launch_latent_query(int B, int Hq, int G, int D, int r, int wr_per_qh,
                                const uint16_t *q, const uint16_t *w_r, const uint16_t *w_post,
                                float *q_lat, int32_t *err, cudaStream_t stream);
cudaError_t launch_latent_expand(int B, int Hq, int D, int r, const float *o_lat,
                                 const uint16_t *w_post, void *out, kl_dtype out_dtype,
                                 int32_t *err, cudaStream_t stream);

// Number of SMs of the current device (cached per device).
int device_sm_count();

// A launch site's one-time set-up of its kernel (a function attribute, which belongs to the
// function on the current device): run once per device (ordinals below 64; others every time).
struct PerDeviceOnce {
    std::atomic<uint64_t> done{0};
    template <typename F>
    cudaError_t run(F &&setup) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
        if (bit && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
        e = setup();
        if (e == cudaSuccess && bit) done.fetch_or(bit, std::memory_order_release);
        return e;
    }
};

}  // namespace kl
