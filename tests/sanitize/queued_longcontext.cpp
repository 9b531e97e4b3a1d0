// The queued device (queued_device.cpp) with the launches of rotated appends, page bounds and sparse preds: what their kernels would read of pinned memory.
#include "queued_device.cpp"
#include "sparse.hpp"

namespace symkv {
int enter_device(int) { return -1; }
void leave_device(int) {}
bool stream_captures(hipStream_t) { return false; }
hipError_t launch_rope_rows(RopeRowsArgs, const RopeTable&, int, hipStream_t) { return launch({}); }
hipError_t launch_append_rope(AppendRopeArgs a, const RopeTable&, int, hipStream_t) {
  Command c{{}, a.done};
  if (!a.by_args) add(c, a.runs, (int64_t)a.n_runs * RUN_WORDS * 4);
  add(c, a.host_words, a.copy_words * 4);
  return launch(c);
}
hipError_t launch_bounds(const BoundsArgs& a, int, hipStream_t) {
  Command c{{}, a.done};
  if (!a.by_args) add(c, a.pages, (int64_t)a.n_pages * 4);
  return launch(c);
}
hipError_t launch_sparse_first(const AppendRopeArgs&, const RopeTable&, const SparseArgs&, int, hipStream_t) { return launch({}); }
hipError_t launch_sparse_scores(const SparseArgs&, int, hipStream_t) { return launch({}); }
hipError_t launch_sparse_attend(const SparseArgs&, int, hipStream_t) { return launch({}); }
}  // namespace symkv
