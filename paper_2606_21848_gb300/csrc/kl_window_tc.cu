// Attention of consecutive positions with a sliding window and first tokens that stay visible, in blocks of 128 rows
// (kl_prefill_tc_kernel.cuh, kWindow): chunks, prompts, and the last tokens of large groups. The tensor cores bound long
// windows, a block's start and outputs (7 us, against 1.05 per tile) short ones. Measured: 8 chunks of 512 rows on 8192,
// 32 / 8 heads, window 1024: 129 us; a prompt of 32768, 12 / 2 heads, window 4096: 853 us (1.37 PFLOP/s issued, two thirds
// of them useful).
#include "kl_prefill_tc_kernel.cuh"

namespace kl {

cudaError_t launch_window_tc(const PrefillArgs &a) {
    const int64_t line = window_line(kPrefillRows, a.window, a.sinks, (int64_t)a.geo.max_pages * a.geo.P);
    return a.out_dtype == KL_FP32 ? launch_rows<kModeWindow, 3, 3>(a, line) : launch_rows<kModeWindow, 2, 1>(a, line);
}

}  // namespace kl
