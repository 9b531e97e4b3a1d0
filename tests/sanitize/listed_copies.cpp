// The queued device (queued_device.cpp) with the launches for beams, which keeps what lies in the lists of page copies at their launch; the
// queue sees whether it still does when the launch is carried out.
#include "queued_longcontext.cpp"
#include "beam.hpp"

namespace {
struct Copies {
  std::vector<int32_t> words;
  bool by_args;
};
std::vector<Copies> listed;
}  // namespace

extern "C" int64_t listed_launches() { return (int64_t)listed.size(); }
extern "C" int32_t listed_copies(int64_t launch) { return (int32_t)listed[(size_t)launch].words.size() / 3; }
extern "C" int listed_by_args(int64_t launch) { return listed[(size_t)launch].by_args; }
extern "C" void listed_words(int64_t launch, int32_t* out) {
  const Copies& c = listed[(size_t)launch];
  std::copy(c.words.begin(), c.words.end(), out);
}
extern "C" void listed_forget() { listed.clear(); }

namespace symkv {
hipError_t launch_select_rows(const SelectArgs&, int, hipStream_t) { return launch({}); }
hipError_t launch_select_best(const SelectArgs&, const GroupRows&, int32_t, int32_t, int, hipStream_t) { return launch({}); }
hipError_t launch_states(const StatesArgs&, const GroupRows&, int32_t, hipStream_t) { return launch({}); }
hipError_t launch_copies(const CopyArgs& a, hipStream_t) {
  Command c{{}, a.done};
  if (!a.by_args) add(c, a.list, (int64_t)a.n_copies * 12);
  if (!a.by_args && c.reads.empty()) return hipErrorInvalidValue;      // a list that is not pinned
  listed.push_back({std::vector<int32_t>(a.list, a.list + 3 * a.n_copies), a.by_args != 0});
  return launch(c);
}
}  // namespace symkv
