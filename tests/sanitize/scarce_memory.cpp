// The queued device (queued_device.cpp) on a host whose memory runs out: from the n-th allocation of the library on, every one fails.  Those of the
// stand-ins for launches are not the library's.
#include <cstdint>
#include <cstdlib>
#include <new>

namespace {
int64_t left = -1;        // allocations until the first that fails; -1: none fails
struct Device {           // while a launch is taken
  int64_t kept = left;
  Device() { left = -1; }
  ~Device() { left = kept; }
};
}  // namespace
extern "C" void memory_left(int64_t n) { left = n; }
void* operator new(size_t n) {
  if (left == 0) throw std::bad_alloc();
  if (left > 0) --left;
  if (void* p = malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

#define launch_prologue queued_prologue
#include "queued_device.cpp"
#undef launch_prologue
#include "sparse.hpp"

namespace symkv {
hipError_t launch_prologue(PrologueArgs a, hipStream_t st) {
  const Device here;
  return queued_prologue(a, st);
}
int enter_device(int) { return -1; }
void leave_device(int) {}
bool stream_captures(hipStream_t) { return false; }
hipError_t launch_rope_rows(RopeRowsArgs, const RopeTable&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_append_rope(AppendRopeArgs a, const RopeTable&, int, hipStream_t) {
  const Device here;
  return launch({{}, a.done});
}
hipError_t launch_bounds(const BoundsArgs& a, int, hipStream_t) {
  const Device here;
  return launch({{}, a.done});
}
hipError_t launch_sparse_first(const AppendRopeArgs&, const RopeTable&, const SparseArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_sparse_scores(const SparseArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_sparse_attend(const SparseArgs&, int, hipStream_t) { return hipSuccess; }
}  // namespace symkv
