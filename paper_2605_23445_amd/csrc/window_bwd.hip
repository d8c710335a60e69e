// Backward pass of attention over a window: its launches for sequences of one length.
#include "window_bwd.h"

namespace dfs {

int run_window_bwd(const WindowArgs& a, int d, int dtype, hipStream_t st) { return run_bwd<false>("dfs_window_attn_bwd", a, d, dtype, st); }

}  // namespace dfs
