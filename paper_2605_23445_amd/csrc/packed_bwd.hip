// Backward pass of attention over packed sequences: the launches of the windowed one's kernels for these.
#include "window_bwd.h"

namespace dfs {

int run_packed_bwd(const WindowArgs& a, int d, int dtype, hipStream_t st) { return run_bwd<true>("dfs_packed_attn_bwd", a, d, dtype, st); }

}  // namespace dfs
