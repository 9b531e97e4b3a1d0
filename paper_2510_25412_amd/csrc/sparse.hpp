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
// Runs of an append that travel with the kernel's arguments (2 KB of the 4 KB that a launch may have); more are read from memory: a sparse
// pred of one file 19.1 us a call (20.1 from pinned memory), an append to 64 files 10.1 (10.3).
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
  int32_t apart;            // keys and values in workgroups of their own (set by the launch function)
  const int32_t* host_words;   // lists to be copied along the way: pinned host memory, where to, how many words
  int32_t* dev_words;
  int64_t copy_words;
  hipEvent_t done;
};

constexpr int kArgPages = 256;    // pages whose ids travel with the arguments: one fp32 file of 300..700 tokens 4.9 us a call (5.3 from pinned memory, staging included)
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
// A row with pages to score: row, page table (offset into the tables), end of the pages to score.
constexpr int SPARSE_SCORED_WORDS = 3;
constexpr int kPartPages = 2048;       // most pages of a part of a row's list (one workgroup's)
struct SparseArgs {
  const uint8_t* pool;
  int64_t page_bytes;
  const uint8_t* bounds;    // of this layer
  const void* q;            // [rows][Hq][row]
  float* out;               // [rows][Hq][D]
  int32_t* picked;          // [rows][Hkv][budget] or null: index of the pages read, -1 past the last
  const int32_t* rows;      // [rows][SPARSE_ROW_WORDS]
  const int32_t* scored;    // [n_scored][SPARSE_SCORED_WORDS]
  const int32_t* tables;
  uint32_t* scores;         // [rows of the launch][Hkv][score_stride]: in the order of the scores, from page `first` on (own: none)
  float* part_acc;          // [rows of the launch][Hkv][splits][G][D]
  float* part_ml;           // [rows of the launch][Hkv][splits][G][2]
  int32_t* counters;        // [rows of the launch][Hkv]: parts that are done (several parts); 0 between launches
  int32_t row0, n_rows;     // rows of this launch
  int32_t scored0, n_scored;              // scored rows of this launch
  int32_t most_scored;      // pages of the one with most of them
  int32_t Hq, Hkv, budget, first, last;
  int32_t score_stride;
  int32_t splits, waves;    // parts of a row's list; wavefronts of a workgroup that attends
  int32_t own;              // the workgroups that attend score their row's pages themselves
  int32_t stream;           // no two rows read the same pages, as far as the host looks
  float scale_log2e;
};

// Whether the workgroups that attend score their row's pages themselves, for `units` rows and heads with pages to score, `most` of
// them in the longest.  That saves a launch and the scores' way through memory.  Beyond a workgroup for every compute unit nothing is lost by it: 64
// files of 256, 512, 1024 and 2000 pages, 8 heads: 65, 81, 106 and 152 us a call, 78, 96, 125 and 175 with a launch of its own.  With
// fewer rows a wavefront has more to score (and every part of a row's list does it again): one file of 128, 256, 512 pages 17.7, 19.9,
// 25.1 us, and 20.8, 21.5, 21.8 with the launch; 4 files of 256 pages 23.2 and 24.8, 8 files 31.1 and 28.1; 16 and 32 files of 128 pages
// 32.6 and 43.5, and 32.8 and 42.8.
constexpr int kOwnScores = 2048;
inline bool scores_itself(int64_t units, int64_t most) { return most <= (units > 256 ? kOwnScores : units <= 32 ? 256 : 128); }
// Wavefronts of a workgroup that attends.  Eight share the choice of a long row, where there are no more rows than compute units: 8 files
// of 32k..131k tokens 84 us a call (89 with four), 32 files of 36000 tokens 102 (107), 8 layers of one file 186 (192).  Otherwise four, of
// which more fit: 64 files of 512..4096 tokens 61 us (70 with eight), 64 files of 36000 tokens 184 (192).
inline int attend_waves(bool own, int64_t units) { return !own && units <= 256 ? 8 : 4; }

// Whether the append of a batch and its scores are one launch, for a batch of single tokens with no bounds missing: turned query rows
// in pairs that a lane holds, and no more wavefronts to score than run at once: each turns query rows again.  8 layers of 1, 2, 4 and 8
// files of 30000 tokens: 173, 202, 242 and 354 us a step, and 203, 237, 267 and 357 with two launches a layer; 4 layers of 1, 2 and 4
// files of 60000 tokens with 64 query heads: 118, 146 and 201, and 129, 150 and 179.
constexpr int kFirstPages = 16;            // of a wavefront that scores there
constexpr int64_t kFirstWaves = 4096;
inline bool scores_with_append(const RopeTable& r, int Hkv, int64_t n_scored, int64_t most_scored) {
  return (r.path == ROPE_HALVES || r.path == ROPE_INTERLEAVED) && n_scored > 0 && (most_scored + kFirstPages - 1) / kFirstPages * Hkv * n_scored <= kFirstWaves;
}

// The scores that the least chosen one can still be, lo <= it <= hi, in rounds: 256 equal steps (a power of two each), of which the one with
// the wanted score becomes the range.  Scores are whole numbers from 1 on (0: none) up to 2^32 - 1, and a range may end at
// the last of them: its end is found by subtracting, since lo + a step's width may not fit 32 bits.
constexpr int kChoiceRounds = 4;           // a range of less than 2^32, 2^24, 2^16, 2^8: the last one's steps are single values
struct ScoreRange {
  uint32_t lo, hi;
  __host__ __device__ int shift() const { return hi - lo < 256 ? 0 : 24 - __builtin_clz(hi - lo); }
  __host__ __device__ bool holds(uint32_t k) const { return k - lo <= hi - lo; }
  __host__ __device__ uint32_t step(uint32_t k, int by) const { return (k - lo) >> by; }
  // to its step s, steps of 1 << by
  __host__ __device__ void narrow(uint32_t s, int by) {
    lo += s << by;
    const uint32_t most = (1u << by) - 1;
    hi = hi - lo < most ? hi : lo + most;
  }
};

// Weak: the host code is also built without kernels (by tests of the host side, against stand-ins for the launches it made before these).
#define SYMKV_LAUNCH __attribute__((weak))
SYMKV_LAUNCH hipError_t launch_rope_rows(RopeRowsArgs a, const RopeTable& r, int dtype, hipStream_t st);
SYMKV_LAUNCH hipError_t launch_append_rope(AppendRopeArgs a, const RopeTable& r, int dtype, hipStream_t st);
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
