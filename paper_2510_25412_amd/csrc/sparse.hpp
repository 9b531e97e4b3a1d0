// Argument blocks and launch functions of the kernels for rotary positions, page bounds and sparse preds (see sparse.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace symkv {

// How rows turn: pair i of a head by turns[i] whole turns per position, times mag.
enum { ROPE_NONE = 0, ROPE_HALVES, ROPE_HALVES_ANY, ROPE_INTERLEAVED };      // HALVES: half the turned elements are whole 16-byte chunks
struct RopeTable {
  double turns[64];
  double mag;
  int32_t path;             // ROPE_*
  int32_t dims;             // elements of a head that turn
};

constexpr int kMostRopeRows = 1 << 22;      // tokens of a launch
struct RopeRowsArgs {
  const void* q;            // [n][Hq][row], or null
  void* q_out;              // may be q
  const void* k;            // [n][Hkv][row], or null
  void* k_out;
  const int32_t* pos;       // device [n]
  int32_t n, Hq, Hkv;
  int32_t tokens;           // per workgroup (filled by the launch function)
};

constexpr int RUN_WORDS = 4;      // first token, its slot (page * P + slot), tokens | page completed << 8, position of the first token
// Runs of an append that travel with the kernel's arguments (2 KB of the 4 KB that a launch may have); more are read from memory.
constexpr int kArgRuns = 128;
struct AppendRopeArgs {
  uint8_t* pool;
  int64_t page_bytes, layer_bytes;
  uint8_t* bounds;          // [layers][pages][Hkv][512], or null
  int64_t layer_bounds;     // bytes of a layer of the bounds
  const void* k;            // [layers][T][Hkv][row]
  const void* v;
  int64_t layer_rows;       // bytes of a layer's rows in k and in v
  const void* q;            // [T][Hq][row] to be turned into q_out, or null
  void* q_out;
  const int32_t* pos;       // device [T], or null: the position that the run says
  const int32_t* runs;      // host (at most kArgRuns), or pinned / device
  int32_t n_runs, Hq, Hkv, n_layers;
  int32_t run_tokens;       // tokens of the longest run
  int32_t by_args;          // the runs are host memory and travel with the arguments
  const int32_t* host_words;   // lists to be copied along the way: pinned host memory, where to, how many words
  int32_t* dev_words;
  int64_t copy_words;
  hipEvent_t done;
};

constexpr int kArgPages = 256;    // pages whose ids travel with the arguments
struct BoundsArgs {
  const uint8_t* pool;
  int64_t page_bytes, layer_bytes;
  uint8_t* bounds;
  int64_t layer_bounds;
  const int32_t* pages;     // host (at most kArgPages), or pinned / device
  int32_t n_pages, Hkv, n_layers;
  int32_t by_args;
  hipEvent_t done;
};

constexpr int SPARSE_ROW_WORDS = 2;    // page table (offset into the tables), tokens seen
// Consecutive tokens of one file, scored together: first row, rows, page table (offset into the tables), end of the pages to score.
constexpr int SPARSE_GROUP_WORDS = 4;
constexpr int kGroupRows = 4;
constexpr int kPartPages = 2048;       // most pages of a part of a row's list (one workgroup's)
struct SparseArgs {
  const uint8_t* pool;
  int64_t page_bytes;
  const uint8_t* bounds;    // of this layer
  const void* q;            // [rows][Hq][row]
  float* out;               // [rows][Hq][D]
  int32_t* picked;          // [rows][Hkv][budget] or null: index of the pages read, -1 past the last
  const int32_t* rows;      // [rows][SPARSE_ROW_WORDS]
  const int32_t* groups;    // [n_groups][SPARSE_GROUP_WORDS]
  const int32_t* tables;
  uint32_t* scores;         // [rows of the launch][Hkv][score_stride]: in the order of the scores, from page `first` on
  float* part_acc;          // [rows of the launch][Hkv][splits][G][D]
  float* part_ml;           // [rows of the launch][Hkv][splits][G][2]
  int32_t* counters;        // [rows of the launch][Hkv]: parts that are done (several parts); 0 between launches
  int32_t row0, n_rows;     // rows of this launch
  int32_t group0, n_groups, group_rows;   // groups of this launch, which need scores, and the most rows of one
  int32_t most_scored;      // pages of the group with most to score
  int32_t Hq, Hkv, budget, first, last;
  int32_t score_stride;
  int32_t splits;
  int32_t stream;           // no two rows read the same pages, as far as the host looks
  float scale_log2e;
};

// Whether a workgroup of the attention scores its row's pages itself.
constexpr int kOwnScores = 512;
inline bool scores_itself(int64_t most_scored) { return most_scored <= kOwnScores; }
inline int attend_waves(int64_t most_scored) { return scores_itself(most_scored) ? 4 : 8; }

// Whether the append of a batch and its scores are one launch, for a batch of single tokens with no bounds missing: turned query rows
// in pairs that a lane holds, and few wavefronts to score.
constexpr int kFirstPages = 16;            // of a wavefront that scores there
constexpr int64_t kFirstWaves = 2048;
inline bool scores_with_append(const RopeTable& r, bool turns, int Hkv, int64_t n_groups, int64_t most_scored) {
  return turns && (r.path == ROPE_HALVES || r.path == ROPE_INTERLEAVED) && n_groups > 0 && !scores_itself(most_scored) &&
         (most_scored + kFirstPages - 1) / kFirstPages * Hkv * n_groups <= kFirstWaves;
}

// Weak: the host code is also built without kernels (by tests of the host side, against stand-ins for the launches it made before these).
#define SYMKV_LAUNCH __attribute__((weak))
SYMKV_LAUNCH hipError_t launch_rope_rows(RopeRowsArgs a, const RopeTable& r, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_append_rope(const AppendRopeArgs& a, const RopeTable& r, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_bounds(const BoundsArgs& a, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_sparse_first(const AppendRopeArgs& a, const RopeTable& r, const SparseArgs& s, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_sparse_scores(const SparseArgs& a, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_sparse_attend(const SparseArgs& a, int dtype, hipStream_t st);
// Makes the device current and returns the one that was (-1: nothing to undo); the other way round.
SYMKV_LAUNCH int enter_device(int device);
SYMKV_LAUNCH void leave_device(int before);
// Whether work on the stream is being recorded instead of run.
SYMKV_LAUNCH bool stream_captures(hipStream_t st);
#undef SYMKV_LAUNCH

}  // namespace symkv
