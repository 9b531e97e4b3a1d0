// Argument blocks and launch functions of the kernels for beams: choices, state rows (beam.hip) and page copies (pages.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace symkv {

constexpr int kBeamsMost = 64;         // rows of a group
constexpr int kBestMost = 128;         // choices of a group
constexpr int kGroupsAtOnce = 256;     // groups of a launch: their first rows travel with its arguments (1 KB)
struct GroupRows {
  int32_t base;                        // row of the launch's first group
  int32_t each;                        // rows of every group, where they are equal: any number of groups in a launch
  int32_t first[kGroupsAtOnce + 1];    // rows before each group, from there on
  __host__ __device__ int32_t row(int32_t g) const { return base + (each ? g * each : first[g]); }
  __host__ __device__ int32_t rows(int32_t g) const { return each ? each : first[g + 1] - first[g]; }
};

constexpr int kOctet = 8;              // what a row is cut by, in logits
constexpr int kMostParts = 256;        // parts of a group that its choice starts from
struct SelectArgs {
  const void* logits;
  int64_t stride;                      // elements from row to row
  const float* scores;
  const uint8_t* allowed;              // or null
  int64_t allowed_stride;              // bytes from row to row
  float* best_scores;
  int32_t* best_beams;
  int32_t* best_tokens;
  // scratch, [rows][parts]: the logit that exponents are counted from, their sum; [rows][parts][64]: the largest logit of each lane, and the
  // group of 16 bytes that holds it first
  double* sums;
  float* refs;
  float* most;
  int32_t* most_at;
  int32_t rows, vocab, n_best;
  int32_t parts, parts_bits, part_octets;      // wavefronts of a row (a power of two), octets of logits of each
};

// How a row is cut: a power of two of parts, octets of a part.
struct SelectCut {
  int32_t bits, part_octets;
};
constexpr int kSelectWaves = 2048;
inline SelectCut select_cut(int64_t rows, int32_t most_beams, int32_t vocab, int32_t n_best) {
  const int64_t octets = (vocab + kOctet - 1) / kOctet, want = (kSelectWaves + rows - 1) / rows, most = std::min<int64_t>(kMostParts / most_beams, 64);
  int32_t bits = 0;
  // enough lists that the best of one row's are a choice's; then wavefronts, of no more than 8192 logits and no less than 2048
  while ((2ll << bits) <= most && ((32ll << bits) < n_best || ((octets >> bits) > 256 && ((1ll << bits) < want || (octets >> bits) > 1280)))) ++bits;
  return SelectCut{bits, (int32_t)((((octets + (1ll << bits) - 1) >> bits) + 63) / 64 * 64)};
}

constexpr int kStatesAtOnce = 8;       // arrays of a launch
struct StateArray {
  uint8_t* dst;
  const uint8_t* src;
  int64_t outer_stride, row_stride, row_bytes;
  uint32_t chunks;                     // workgroups of a group's rows
  uint32_t end;                        // workgroups of this array and those before it
};
struct StatesArgs {
  StateArray array[kStatesAtOnce];
  const int32_t* parents;
  int32_t n_arrays, n_groups;
};
constexpr int kStateUnit = 16;         // bytes of each row that a thread moves
constexpr int kStateThreads = 256;
// Columns of a thread, by the rows of the largest group.
constexpr int state_columns(int beams) { return beams <= 4 ? 4 : beams <= 8 ? 2 : 1; }

constexpr int kArgCopies = 256;        // copies that travel with the arguments (3 KB of the 4 KB that a launch may have)
struct CopyArgs {
  uint8_t* pool;
  int64_t page_bytes, layer_bytes;
  uint8_t* bounds;                     // or null
  int64_t layer_bounds;
  const int32_t* list;                 // (source, destination, slots | 1 << 8: bounds too): host (by_args), or pinned
  int32_t n_copies, n_layers, Hkv;
  int32_t by_args;
  hipEvent_t done;
};

// Weak: see sparse.hpp.
#define SYMKV_LAUNCH __attribute__((weak))
SYMKV_LAUNCH hipError_t launch_select_rows(const SelectArgs& a, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_select_best(const SelectArgs& a, const GroupRows& g, int32_t group0, int32_t n_groups, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_states(const StatesArgs& a, const GroupRows& g, int32_t most_beams, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_copies(const CopyArgs& a, hipStream_t st);
#undef SYMKV_LAUNCH

}  // namespace symkv
