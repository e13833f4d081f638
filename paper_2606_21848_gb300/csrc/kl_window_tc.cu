// Attention of consecutive positions with a sliding window and first tokens that stay visible, in blocks of 128 rows
// (kl_prefill_tc_kernel.cuh, kWindow): chunks, prompts, and the last tokens of large groups.
#include "kl_prefill_tc_kernel.cuh"

namespace kl {

cudaError_t launch_window_tc(const PrefillArgs &a) {
    const int64_t line = window_line(kPrefillRows, a.window, a.sinks, (int64_t)a.geo.max_pages * a.geo.P);
    return a.out_dtype == KL_FP32 ? launch_rows<kModeWindow, 3, 3>(a, line) : launch_rows<kModeWindow, 2, 1>(a, line);
}

}  // namespace kl
