// What consecutive query positions see under the causal mask with a sliding window and first tokens that
// stay visible: position p sees t <= p with t < sinks or t > p - window.
#pragma once

namespace kl {

// The cache tiles of 128 tokens that positions p0 .. p1 may see, laid end to end: those of the first tokens,
// then the window's. Token x of this line is token x of the sequence up to `first`, x + shift behind it.
struct WindowSpan {
    int first, shift, len;
};
__host__ __device__ inline WindowSpan window_span(int p0, int p1, int window, int sinks) {
    const int end = p1 + 1, head = ((sinks < end ? sinks : end) + 127) / 128;
    const int low = p0 - window + 1 > 0 ? (p0 - window + 1) / 128 : 0;
    WindowSpan s;
    s.first = head * 128;
    s.shift = low > head ? (low - head) * 128 : 0;
    s.len = end - s.shift;
    return s;
}

// Most tokens of that line for `rows` consecutive positions of a sequence of up to max_tokens tokens (window
// and sinks at most max_tokens): the window and the rows touch one tile more than they fill.
__host__ __device__ inline int64_t window_line(int64_t rows, int64_t window, int64_t sinks, int64_t max_tokens) {
    const int64_t n = ((sinks + 127) / 128 + (window + rows - 2) / 128 + 2) * 128;
    return n < max_tokens ? n : max_tokens;
}

// The rows of a block with `rows` rows per value head (positions x heads of a group): 16 or 32 on the wide
// decode's kernel, 0: 128 on the prefill's. fp32 outputs take operands of three bf16 terms, and a W^R per query head
// a place in tensor memory each, which leaves room for 16.
inline int window_rows(int64_t rows, bool fp32, bool per_qh) {
    if (rows <= 16 || fp32) return 16;
    if (rows <= 32) return per_qh ? 16 : 32;
    return 0;
}

}  // namespace kl
