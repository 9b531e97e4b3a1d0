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
// Parts, first, until the lists of one row can hold a choice.  Then, while a part has more than 2048 logits (a wavefront's loads under way), until there
// are 2048 wavefronts, but no more parts of a group than 512 threads hold in the second launch (rows of 131072 bf16 logits, calls of 4, 16, 64 requests
// of 4 beams: 12, 14, 23 us; with up to 256 parts of a group 14, 18, 23; wavefronts 1024 or 4096: 13.9 and 19.8 us for 16 requests), or until a
// part has no more than 40960 logits of 16 bits (2048 rows of 131072: 97 us; 20480 101, 10240 105, 81920 100), 10240 of fp32 (1024 rows of 65537, 32
// choices of 16 beams: 58 us; 62 with half as many or four times as many: what is looked at again is a list, a 64th of a part).
// The bound of 64 parts is the one that 4 beams want.  Few wide requests of 16-bit logits lose by it: 1 and 4 requests of 16 beams of 131072 take 17.4 and
// 18.9 us, with 256 parts 12.4 and 14.3, of 32 beams 20 and 22 against 15 and 18, of 64 beams of 40960 22 and 23 against 17 and 20; with 16 requests
// of 16 beams and more, and with fp32 logits of so many, the two are alike within 2 us.
constexpr int kSelectWaves = 2048, kSelectParts = 64;
inline SelectCut select_cut(int64_t rows, int32_t most_beams, int32_t vocab, int32_t n_best, int32_t logit_bytes) {
  const int64_t octets = (vocab + kOctet - 1) / kOctet, most = std::min<int64_t>(kMostParts / most_beams, 64);
  const int64_t longest = logit_bytes == 4 ? 1280 : 5120;
  int32_t bits = 0;
  const auto more = [&] {
    if ((32ll << bits) < n_best) return true;
    if ((octets >> bits) <= 256) return false;
    return (octets >> bits) > longest || ((rows << bits) < kSelectWaves && ((int64_t)most_beams << (bits + 1)) <= kSelectParts);
  };
  while ((2ll << bits) <= most && more()) ++bits;
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
