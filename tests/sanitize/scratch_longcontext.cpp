// The queued device (queued_device.cpp) with launches of sparse preds that look at the scratch they are given: every section inside the
// workspace and apart from the others, as long as the launch's rows need it.
#include "queued_device.cpp"
#include "sparse.hpp"

namespace {
uintptr_t ws_at;
int64_t ws_bytes, outside, attends, most_splits, least_splits;
int64_t G, D;

struct Span {
  uintptr_t at;
  int64_t bytes;
};
void look(std::vector<Span> spans) {
  for (size_t i = 0; i < spans.size(); ++i) {
    const Span& s = spans[i];
    if (s.bytes == 0) continue;
    if (s.at < ws_at || s.at + (uintptr_t)s.bytes > ws_at + (uintptr_t)ws_bytes) ++outside;
    for (size_t j = 0; j < i; ++j)
      if (spans[j].bytes > 0 && s.at < spans[j].at + (uintptr_t)spans[j].bytes && spans[j].at < s.at + (uintptr_t)s.bytes) ++outside;
  }
}
std::vector<Span> sections(const symkv::SparseArgs& a, bool scores) {
  const int64_t units = (int64_t)a.n_rows * a.Hkv;
  const bool parts = a.splits > 1;
  std::vector<Span> s = {{(uintptr_t)a.rows, (a.row0 + a.n_rows) * symkv::SPARSE_ROW_WORDS * 4ll},
                         {(uintptr_t)a.counters, parts ? units * 4 : 0},
                         {(uintptr_t)a.part_ml, parts ? units * a.splits * G * 2 * 4 : 0},
                         {(uintptr_t)a.part_acc, parts ? units * a.splits * G * D * 4 : 0}};
  if (scores) s.push_back({(uintptr_t)a.scores, units * a.score_stride * 4});
  const uintptr_t q = (uintptr_t)a.q;
  if (q >= ws_at && q < ws_at + (uintptr_t)ws_bytes) s.push_back({q, (a.row0 + a.n_rows) * (int64_t)a.Hq * 256});
  return s;
}
}  // namespace

extern "C" {
void scratch_of(uintptr_t at, int64_t bytes, int64_t group, int64_t dim) {
  ws_at = at;
  ws_bytes = bytes;
  G = group;
  D = dim;
  attends = most_splits = 0;
  least_splits = 1 << 30;
}
void scratch_seen(int64_t* out) {
  out[0] = outside;
  out[1] = attends;
  out[2] = least_splits;
  out[3] = most_splits;
}
}

namespace symkv {
int enter_device(int) { return -1; }
void leave_device(int) {}
bool stream_captures(hipStream_t) { return false; }
hipError_t launch_rope_rows(RopeRowsArgs, const RopeTable&, int, hipStream_t) { return launch({}); }
hipError_t launch_append_rope(AppendRopeArgs a, const RopeTable&, int, hipStream_t) {
  if (a.dev_words) look({{(uintptr_t)a.dev_words, (a.copy_words + 3) / 4 * 16}, {(uintptr_t)a.q_out, a.q ? (int64_t)a.n_runs * a.Hq * 256 : 0}});
  return launch({{}, a.done});
}
hipError_t launch_bounds(const BoundsArgs& a, int, hipStream_t) { return launch({{}, a.done}); }
hipError_t launch_sparse_first(const AppendRopeArgs&, const RopeTable&, const SparseArgs& a, int, hipStream_t) { return look(sections(a, true)), launch({}); }
hipError_t launch_sparse_scores(const SparseArgs& a, int, hipStream_t) { return look(sections(a, true)), launch({}); }
hipError_t launch_sparse_attend(const SparseArgs& a, int, hipStream_t) {
  look(sections(a, !a.own && a.n_scored > 0));
  ++attends;
  most_splits = std::max<int64_t>(most_splits, a.splits);
  least_splits = std::min<int64_t>(least_splits, a.splits);
  return launch({});
}
}  // namespace symkv
