// The rounds in which the least chosen score of a row is found (ScoreRange of sparse.hpp), walked on the host as the kernel walks them.
#include <algorithm>
#include <cstdint>
#include <vector>

#include "sparse.hpp"

using symkv::ScoreRange;

extern "C" {

// The places chosen of `m` scores, behind which `fill` zeros lie (what a thread holds past the end).  Returns how many were chosen, written to
// `out` (room for m + fill) in order; -1: the rounds did not end, -2: a step beyond the 256 was counted.
int64_t choice_pick(const uint32_t* scores, int64_t m, int64_t fill, int64_t want, int32_t* out) {
  std::vector<uint32_t> key(scores, scores + m);
  key.resize((size_t)(m + fill), 0u);
  ScoreRange r{*std::min_element(scores, scores + m), *std::max_element(scores, scores + m)};
  uint32_t need = (uint32_t)want, t = 0;
  bool ended = false;
  for (int round = 0; round < symkv::kChoiceRounds && !ended; ++round) {
    const int shift = r.shift();
    uint32_t hist[256] = {};
    for (uint32_t k : key)
      if (r.holds(k)) {
        if (r.step(k, shift) > 255) return -2;
        ++hist[r.step(k, shift)];
      }
    int step = 255;
    uint32_t above = 0;
    while (step > 0 && above + hist[step] < need) above += hist[step--];
    need -= above;
    r.narrow((uint32_t)step, shift);
    if (need == hist[step]) {
      t = r.lo - 1;
      need = 0;
      ended = true;
    } else if (shift == 0) {
      t = r.lo;
      ended = true;
    }
  }
  if (!ended) return -1;
  int64_t n = 0;
  uint32_t equal = 0;
  for (size_t i = 0; i < key.size(); ++i) {
    if (key[i] < t || key[i] == 0) continue;
    if (key[i] > t || equal < need) out[n++] = (int32_t)i;
    equal += key[i] == t;
  }
  return n;
}

// 0 if every step of [lo, hi] is a range inside it, not wider than it says, that does not hold 0, and all steps together are [lo, hi].
int choice_range(uint32_t lo, uint32_t hi) {
  const ScoreRange whole{lo, hi};
  const int shift = whole.shift();
  const uint32_t last = whole.step(hi, shift);
  if (last > 255) return 1;
  uint64_t next = lo;
  for (uint32_t s = 0; s <= last; ++s) {
    ScoreRange r = whole;
    r.narrow(s, shift);
    if (r.lo != next || r.hi < r.lo || r.hi > hi || r.holds(0u) || r.hi - r.lo >= (1u << shift)) return 2;
    if (whole.step(r.lo, shift) != s || whole.step(r.hi, shift) != s) return 3;
    next = (uint64_t)r.hi + 1;
  }
  return next == (uint64_t)hi + 1 ? 0 : 4;
}
}
