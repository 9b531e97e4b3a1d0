// Beam search beside the cache: the best continuations of a request's beams, and state rows that follow their beams.
#include <cfloat>

#include "../../include/symphony_kv.h"
#include "beam.hpp"
#include "device.hpp"

namespace symkv {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kLastLevelBytes = 256ll << 20;

// ---- steps across the lanes of a wavefront ---------------------------------------------------

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return as_f32(__builtin_amdgcn_update_dpp(as_u32(x), as_u32(x), CTRL, 0xf, 0xf, false));
}
// The largest of three: an instruction, where fmaxf makes quiet values of its operands first.  NaN only where all are.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}
// x of every lane combined over aligned subsets of 2^BITS lanes, in every lane
template <int BITS, typename F>
__device__ __forceinline__ float across(float x, F f) {
  if constexpr (BITS > 0) x = f(x, dpp<0xB1>(x));      // quad_perm [1,0,3,2]
  if constexpr (BITS > 1) x = f(x, dpp<0x4E>(x));      // quad_perm [2,3,0,1]
  if constexpr (BITS > 2) x = f(x, dpp<0x141>(x));     // row_half_mirror
  if constexpr (BITS > 3) x = f(x, dpp<0x140>(x));     // row_mirror
  if constexpr (BITS > 4) {
    const auto s = __builtin_amdgcn_permlane16_swap(as_u32(x), as_u32(x), false, false);
    x = f(as_f32(s[0]), as_f32(s[1]));
  }
  if constexpr (BITS > 5) {
    const auto s = __builtin_amdgcn_permlane32_swap(as_u32(x), as_u32(x), false, false);
    x = f(as_f32(s[0]), as_f32(s[1]));
  }
  return x;
}
struct Larger {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Smaller {
  __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
};
// The sum over the wavefront, in every lane: the same steps on both halves of a double.
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp((uint32_t)u, (uint32_t)u, CTRL, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp((uint32_t)(u >> 32), (uint32_t)(u >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  x += dpp<0x141>(x);
  x += dpp<0x140>(x);
  uint64_t u = __builtin_bit_cast(uint64_t, x);
  const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false), b = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  x = __builtin_bit_cast(double, (uint64_t)b[0] << 32 | a[0]) + __builtin_bit_cast(double, (uint64_t)b[1] << 32 | a[1]);
  u = __builtin_bit_cast(uint64_t, x);
  const auto c = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false), d = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)d[0] << 32 | c[0]) + __builtin_bit_cast(double, (uint64_t)d[1] << 32 | c[1]);
}
// The same over aligned subsets of 1 << bits lanes, bits the same in every lane.
__device__ __forceinline__ float most_of_parts(float x, int bits) {
  if (bits > 0) x = fmaxf(x, dpp<0xB1>(x));
  if (bits > 1) x = fmaxf(x, dpp<0x4E>(x));
  if (bits > 2) x = fmaxf(x, dpp<0x141>(x));
  if (bits > 3) x = fmaxf(x, dpp<0x140>(x));
  if (bits > 4) x = pair16_max(x);
  if (bits > 5) x = pair32_max(x);
  return x;
}
__device__ __forceinline__ double sum_of_parts(double x, int bits) {
  if (bits > 0) x += dpp<0xB1>(x);
  if (bits > 1) x += dpp<0x4E>(x);
  if (bits > 2) x += dpp<0x141>(x);
  if (bits > 3) x += dpp<0x140>(x);
  if (bits > 4) x += __shfl_xor(x, 16);
  if (bits > 5) x += __shfl_xor(x, 32);
  return x;
}
__device__ __forceinline__ int lanes_of(uint64_t b) { return __builtin_popcountll(b); }

// Floats as whole numbers of the same order, and back.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = as_u32(x);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return as_f32(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// A value that at least K of a wavefront's 256 values (four to a lane) reach, not many more than `limit` of them where they differ.  Of at
// least K disjoint subsets each has one that reaches the smallest of the subsets' largest; from there by halves.  Fewer than
// K above -inf: a value that all of those reach.
__device__ __forceinline__ float reached_by(const float (&x)[4], int K, int limit) {
  const float a = fmaxf(x[0], x[1]), b = fmaxf(x[2], x[3]), most = fmaxf(a, b);
  const float top = across<6>(most, Larger());
  float low = top;
  if (K > 64) low = across<6>(fminf(a, b), Smaller());
  else if (K > 32) low = across<6>(most, Smaller());
  else if (K > 16) low = across<6>(across<1>(most, Larger()), Smaller());
  else if (K > 8) low = across<6>(across<2>(most, Larger()), Smaller());
  else if (K > 4) low = across<6>(across<3>(most, Larger()), Smaller());
  else if (K > 1) low = across<6>(across<4>(most, Larger()), Smaller());
  const auto count = [&](float t) __attribute__((always_inline)) {
    return lanes_of(__ballot(x[0] >= t)) + lanes_of(__ballot(x[1] >= t)) + lanes_of(__ballot(x[2] >= t)) + lanes_of(__ballot(x[3] >= t));
  };
  if (!(low >= -FLT_MAX)) {
    low = -FLT_MAX;
    if (count(low) < K) return low;
  }
  uint32_t lo = __builtin_amdgcn_readfirstlane(key_of(low)), hi = __builtin_amdgcn_readfirstlane(key_of(top));
  while (hi > lo + 1 && count(of_key(lo)) > limit) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (count(of_key(mid)) >= K) lo = mid;
    else hi = mid;
  }
  return of_key(lo);
}

// ---- the rows' part: largest logits and normaliser of a stretch of a row --------------------------

typedef u32x4_t __attribute__((aligned(2))) u32x4_a2;
typedef u32x4_t __attribute__((aligned(4))) u32x4_a4;
template <bool FAR, typename T>
__device__ __forceinline__ u32x4_t load16(const uint8_t* p) {
  if constexpr (FAR) return __builtin_nontemporal_load((const T*)p);
  else return *(const T*)p;
}
// n < 8 logits of 16 bits
template <typename R>
__device__ __forceinline__ R few16(const uint8_t* p, int n) {
  R r = {};
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (j < n) r.w[j >> 1] |= (uint32_t)((const uint16_t*)p)[j] << (16 * (j & 1));
  return r;
}
struct LogitBF16 {
  static constexpr int kBytes = 2, kGroup = 8;
  struct Raw {
    u32x4_t w;
  };
  template <bool FAR>
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return Raw{load16<FAR, u32x4_a2>(p)}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = as_f32(r.w[i] << 16);
      x[2 * i + 1] = as_f32(r.w[i] & 0xffff0000u);
    }
  }
  // from the upper half of the first word on, to the lower half of the word behind
  static __device__ __forceinline__ void unpack_late(const Raw& r, uint32_t behind, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t next = i < 3 ? r.w[i + 1] : behind;
      x[2 * i] = as_f32(r.w[i] & 0xffff0000u);
      x[2 * i + 1] = as_f32(next << 16);
    }
  }
  static __device__ __forceinline__ Raw few(const uint8_t* p, int n) { return few16<Raw>(p, n); }
};
struct LogitF16 {
  static constexpr int kBytes = 2, kGroup = 8;
  struct Raw {
    u32x4_t w;
  };
  template <bool FAR>
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return Raw{load16<FAR, u32x4_a2>(p)}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)r.w[i]);
      x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i] >> 16));
    }
  }
  // from the upper half of the first word on, to the lower half of the word behind
  static __device__ __forceinline__ void unpack_late(const Raw& r, uint32_t behind, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t next = i < 3 ? r.w[i + 1] : behind;
      x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i] >> 16));
      x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)next);
    }
  }
  static __device__ __forceinline__ Raw few(const uint8_t* p, int n) { return few16<Raw>(p, n); }
};
struct LogitF32 {
  static constexpr int kBytes = 4, kGroup = 4;
  struct Raw {
    u32x4_t w;
  };
  template <bool FAR>
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return Raw{load16<FAR, u32x4_a4>(p)}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = as_f32(r.w[i]);
  }
  static __device__ __forceinline__ Raw few(const uint8_t* p, int n) {
    Raw r = {};
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < n) r.w[j] = ((const uint32_t*)p)[j];
    return r;
  }
};

// One wavefront: a part of a row, a group of logits (16 bytes) to a lane at a time, so that neighbouring lanes read neighbouring
// addresses.  What is read is counted from the row's start, whatever the address, so equal rows give equal results.  TINY: rows of less
// than a group, read one by one.
template <typename E, bool MASKED, bool TINY>
struct Part {
  static constexpr int N = E::kGroup;
  const uint8_t* row;
  const uint8_t* bits;
  int vocab, first, end;               // groups of this part
  uint32_t last;                       // where the last of them is read, in bytes

  // Group o.  The last one of a row that does not end with it: the row's last N logits.  What is not wanted comes from where others read.
  template <bool FAR = false>
  __device__ __forceinline__ typename E::Raw raw(int o, bool want) const {
    if constexpr (TINY) return E::few(row, vocab);
    const uint32_t at = min((uint32_t)o * 16, last);
    return E::template load<FAR>(row + (MASKED && !want ? last : at));
  }
  __device__ __forceinline__ uint32_t allowed(int o) const {
    constexpr uint32_t all = (1u << N) - 1;
    const bool in = o < end;
    uint32_t m = all;
    if constexpr (MASKED) {
      const int at = (in ? o : first) * N;
      m = (uint32_t)bits[at >> 3] >> (at & 7) & all;
    }
    return in ? m : 0;
  }
  // -inf in the place of what does not count.  m: the group's allowed bits
  __device__ __forceinline__ void mask(float (&x)[N], int o, uint32_t m) const {
    const int over = (o + 1) * N - vocab;                  // more than a row's last group holds
    if constexpr (TINY) m = over > 0 ? m & (((1u << N) - 1) >> over) : m;
    else m = over > 0 ? m << over : m;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t keep = (uint32_t)((int32_t)(m << (31 - j)) >> 31);
      x[j] = as_f32((as_u32(x[j]) & keep) | (0xff800000u & ~keep));
    }
  }
  __device__ __forceinline__ int token(int o, int j) const { return (TINY ? 0 : min(o * N, vocab - N)) + j; }
  // Group o's logits, masked
  __device__ __forceinline__ void read(int o, float (&x)[N]) const {
    const uint32_t m = allowed(o);
    E::unpack(raw(o, m != 0), x);
    mask(x, o, m);
  }
};

// Groups of a part.
template <typename E>
__device__ __forceinline__ int part_groups(const SelectArgs& a) { return a.part_octets * (kOctet / E::kGroup); }
// The part of row `row` that begins at group `first`.
template <typename E, bool MASKED, bool TINY>
__device__ __forceinline__ Part<E, MASKED, TINY> part_of(const SelectArgs& a, int row, int first) {
  Part<E, MASKED, TINY> p;
  p.row = (const uint8_t*)a.logits + (int64_t)row * a.stride * E::kBytes;
  p.bits = MASKED ? a.allowed + (int64_t)row * a.allowed_stride : nullptr;
  p.vocab = a.vocab;
  p.first = first;
  p.end = min(first + part_groups<E>(a), (a.vocab + E::kGroup - 1) / E::kGroup);
  p.last = TINY ? 0 : (uint32_t)min((p.end - 1) * E::kGroup, a.vocab - E::kGroup) * E::kBytes;
  return p;
}

// One pass over the logits.  Of every part: its normaliser's share, and for each lane (a list: groups 64 apart) the largest logit and the
// group where it is found first; the choice needs no more to know where it has to look again.  Bound: HBM where the rows are many (1024 rows of 65537
// fp32 logits, 268 MB: 46 us, 5.9 TB/s), what is under way where they are few (256 rows of 131072 bf16 logits, 67 MB: 14 us, 4.7 TB/s).
// FAR: more logits than the last-level cache holds are read past it (268 MB 62.7 -> 58.8 us a call, 537 MB 123.6 -> 115.3), fewer may lie there from their
// making, or from this kernel when the choice looks at some again (52 MB 24.4 us, past the cache 27.3; 67 MB 23.8, 24.3).
template <typename E, bool MASKED, bool TINY, bool FAR, bool HALVES = false>
__global__ __launch_bounds__(64) void select_rows_kernel(SelectArgs a) {
  const int lane = threadIdx.x & 63;
  const int row = (int)(blockIdx.x / (uint32_t)a.parts), part = (int)(blockIdx.x % (uint32_t)a.parts);
  const int64_t at = blockIdx.x;
  const float score = as_f32((uint32_t)sload((const int32_t*)a.scores + row));
  const auto p = part_of<E, MASKED, TINY>(a, row, part * part_groups<E>(a));
  if (p.first >= p.end || !(fabsf(score) < INFINITY)) {    // behind the row's end, or no beam lives here
    a.most[at * 64 + lane] = -INFINITY;
    if (lane == 0) {
      a.sums[at] = 0.0;
      a.refs[at] = -FLT_MAX;
    }
    return;
  }
  constexpr int N = E::kGroup, kAhead = 32 / N;            // groups of a lane that are added at a time
  const int whole = min(p.end, a.vocab / N);               // groups that need no look at the row's end

  // Sums of exp(x - c), eight to a lane (four of fp32).  c is a lane's largest logit so far, so that no exponent is positive: a rounding of (x - c)
  // log2 e then weighs at most 2^-24 of the sum, where with c some way below the largest it would weigh that many times as much.  The first
  // c is the wavefront's: rows short enough for one group to a lane then sum the same numbers whatever their order, and in 64 bits, so
  // that rows of the same logits in another order have equal scores.
  float c = -FLT_MAX, s[N] = {}, most = -INFINITY;
  int most_at = p.first + lane;
  const int batches = (p.end - p.first + 64 * kAhead - 1) / (64 * kAhead);
  const auto group = [&](int i, int d) __attribute__((always_inline)) { return p.first + (i * kAhead + d) * 64 + lane; };
  // HALVES: rows of 16-bit logits some of which begin in the middle of a word (every other one of an odd vocabulary).  16 bytes from there cost the
  // memory more than from a word's beginning, so batches that are not at an end of such a row read a half word early, and each lane
  // takes its last logit from the next one (2048 rows of 131071 bf16 logits 144 -> 119 us a call; where no row begins so the
  // registers that this takes cost 67 MB 1.8 us of 23.3).
  const bool late = HALVES && ((uintptr_t)p.row & 2);
  const auto early = [&](int i) __attribute__((always_inline)) {
    const int from = p.first + i * kAhead * 64, to = from + kAhead * 64;
    return late && from > 0 && to <= p.end && to * N < p.vocab;
  };
  struct Batch {
    typename E::Raw raw[kAhead];
    uint32_t m[kAhead], behind;                            // the word behind the last lane's
  };
  uint32_t m_next[kAhead];                                 // allowed bits are known a batch before the logits that they ask for
  const auto load = [&](Batch& b, int i) __attribute__((always_inline)) {
    if (HALVES && early(i)) {
      const uint8_t* row = p.row - 2;
#pragma unroll
      for (int d = 0; d < kAhead; ++d) b.raw[d] = E::template load<FAR>(row + (uint32_t)group(i, d) * 16);
      if (lane == 63) b.behind = *(const uint32_t*)(row + (uint32_t)(group(i, kAhead - 1) + 1) * 16);
    } else {
#pragma unroll
      for (int d = 0; d < kAhead; ++d) {
        b.m[d] = m_next[d];
        b.raw[d] = p.template raw<FAR>(group(i, d), b.m[d] != 0);
      }
    }
#pragma unroll
    for (int d = 0; d < kAhead; ++d) m_next[d] = p.allowed(group(i + 1, d));
  };
  const auto add = [&](const Batch& b, int i) __attribute__((always_inline)) {
    float x[kAhead][N];
    if constexpr (HALVES) {
      if (early(i)) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
          const uint32_t first = b.raw[d].w[0], last = d + 1 < kAhead ? __builtin_amdgcn_readfirstlane(b.raw[d + 1 < kAhead ? d + 1 : d].w[0]) : b.behind;
          const uint32_t next = __builtin_amdgcn_update_dpp(first, first, 0x130, 0xf, 0xf, false);      // wave_shl:1
          E::unpack_late(b.raw[d], lane == 63 ? last : next, x[d]);
        }
      } else {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) E::unpack(b.raw[d], x[d]);
      }
    } else {
#pragma unroll
      for (int d = 0; d < kAhead; ++d) E::unpack(b.raw[d], x[d]);
    }
    if (MASKED || TINY || p.first + (i + 1) * kAhead * 64 > whole) {
#pragma unroll
      for (int d = 0; d < kAhead; ++d) p.mask(x[d], group(i, d), b.m[d]);
    }
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
      float top = max3(x[d][0], x[d][1], x[d][2]);
      if constexpr (N == 8) top = max3(max3(top, x[d][3], x[d][4]), max3(x[d][5], x[d][6], x[d][7]), -INFINITY);
      else top = max3(top, x[d][3], x[d][3]);
      most_at = top > most ? group(i, d) : most_at;
      most = max3(most, top, top);
    }
    float to = max3(c, most, most);
    if (i == 0) to = across<6>(to, Larger());
    const float by = __builtin_amdgcn_exp2f((c - to) * kLog2e);
    c = to;
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] *= by;
#pragma unroll
    for (int d = 0; d < kAhead; ++d)
#pragma unroll
      for (int j = 0; j < N; ++j) s[j] += __builtin_amdgcn_exp2f((x[d][j] - c) * kLog2e);
  };
  Batch even, odd;                                         // the next one is under way while one is added; behind the last nothing counts
#pragma unroll
  for (int d = 0; d < kAhead; ++d) m_next[d] = p.allowed(group(0, d));
  load(even, 0);
  for (int i = 0; i < batches; i += 2) {
    load(odd, i + 1);
    add(even, i);
    load(even, i + 2);
    add(odd, i + 1);
  }
  a.most[at * 64 + lane] = most;
  a.most_at[at * 64 + lane] = most_at;
  const float ref = across<6>(c, Larger());
  double of_lane = 0.0;
#pragma unroll
  for (int j = 0; j < N; ++j) of_lane += (double)s[j];
  const double sum = wave_sum(of_lane * (double)__builtin_amdgcn_exp2f((c - ref) * kLog2e));
  if (lane == 0) {
    a.sums[at] = sum;
    a.refs[at] = ref;
  }
}

// ---- a group's choice --------------------------------------------------------------------------

// A logit, or a list by its largest, in the order of choices: by score, then row, logit (scores of one row are in the order of its logits even
// where 64 bits cannot tell them apart), token or group.  rest: row, logit from the largest down, token (24 bits).
struct Choice {
  double score;
  uint64_t rest;
};
__device__ __forceinline__ uint64_t rest_of(int row, float value, int token) { return (uint64_t)row << 56 | (uint64_t)~key_of(value + 0.0f) << 24 | (uint32_t)token; }
__device__ __forceinline__ bool before(const Choice& a, const Choice& b) { return a.score > b.score || (a.score == b.score && a.rest < b.rest); }
constexpr uint64_t kNone = ~0ull;

constexpr int kFewLists = 4096, kFewThreads = 512, kRanked = 256;
static_assert(kRanked >= kBestMost, "more than the K best");
struct RowScore {
  double base, from;
};

__device__ __forceinline__ double of_order(uint64_t k) { return __builtin_bit_cast(double, k >> 63 ? k ^ 1ull << 63 : ~k); }
// In how many threads x holds, in every thread.  One barrier: the wavefronts' counts lie in one half of `counts` (32) and the next call's in the other.
template <int THREADS>
__device__ __forceinline__ int threads_with(bool x, int* counts, int* half) {
  static_assert(THREADS <= 1024, "16 counts to a half");
  const int lane = threadIdx.x & 63;
  const int of_wave = lanes_of(__ballot(x));
  if (lane == 0) counts[*half + (threadIdx.x >> 6)] = of_wave;
  __syncthreads();
  int n = (lane & 15) < THREADS / 64 ? counts[*half + (lane & 15)] : 0;
  *half ^= 16;
  n += __builtin_amdgcn_update_dpp(0, n, 0xB1, 0xf, 0xf, false);
  n += __builtin_amdgcn_update_dpp(0, n, 0x4E, 0xf, 0xf, false);
  n += __builtin_amdgcn_update_dpp(0, n, 0x141, 0xf, 0xf, false);
  n += __builtin_amdgcn_update_dpp(0, n, 0x140, 0xf, 0xf, false);
  return __builtin_amdgcn_readfirstlane(n);
}

// The K-th of the threads' choices (those of the first n, n >= K), from the highest bit down, of the scores first.  Bits that all have alike are
// passed over: of equal logits only the tokens' differ (64 requests of 4 beams of 131072 equal logits, 128 choices: 0.53 -> 0.26 ms).
template <int THREADS>
__device__ __forceinline__ Choice kth_best(const Choice& mine, const Choice& one, bool is, int K) {
  __shared__ uint32_t unlike[4];
  __shared__ int counts[32];
  int half = 0;
  const auto in = [&](bool x) __attribute__((always_inline)) { return threads_with<THREADS>(x, counts, &half); };
  const auto key_of_score = [](double x) __attribute__((always_inline)) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
    return u ^ ((uint64_t)((int64_t)u >> 63) | 1ull << 63);
  };
  const uint64_t key = key_of_score(mine.score), of_one = key_of_score(one.score);
  if (threadIdx.x < 4) unlike[threadIdx.x] = 0;
  __syncthreads();
  if (is) {
    const uint64_t d = key ^ of_one, e = mine.rest ^ one.rest;
    atomicOr(&unlike[0], (uint32_t)d);
    atomicOr(&unlike[1], (uint32_t)(d >> 32));
    atomicOr(&unlike[2], (uint32_t)e);
    atomicOr(&unlike[3], (uint32_t)(e >> 32));
  }
  __syncthreads();
  const uint64_t scores = (uint64_t)unlike[1] << 32 | unlike[0], rests = (uint64_t)unlike[3] << 32 | unlike[2];
  const auto highest = [](uint64_t x) __attribute__((always_inline)) { return 1ull << (63 - __builtin_clzll(x)); };
  uint64_t score = of_one & ~scores, rest = one.rest | rests;
  for (uint64_t m = scores; m; m &= ~highest(m))
    if (in(is && key >= (score | highest(m))) >= K) score |= highest(m);
  const int left = K - in(is && key > score);
  if (in(is && key == score) == left) return Choice{of_order(score), kNone - 1};      // (all of them)
  for (uint64_t m = rests; m; m &= ~highest(m))
    if (in(is && key == score && mine.rest <= (rest ^ highest(m))) >= left) rest ^= highest(m);
  return Choice{of_order(score), rest};
}

// Of the n > K choices in `found` the K best stay, in any order; the K-th of them, or what none of the others reaches.
template <int THREADS>
__device__ __forceinline__ Choice keep_k(Choice* found, int* n_found, int n, int K) {
  const int tid = threadIdx.x;
  const Choice mine = found[min(tid, n - 1)], cut = kth_best<THREADS>(mine, found[0], tid < n, K);
  if (tid == 0) *n_found = 0;
  __syncthreads();
  if (tid < n && !before(cut, mine)) found[atomicAdd(n_found, 1)] = mine;
  __syncthreads();
  return cut;
}

// The K best of many, in `found` in any order, or all where they are fewer; returns how many.  What `of` makes of turn t in a thread (N choices at
// most; a bit for each that counts) goes there, and whenever it is full the K best stay and nothing behind them comes in any more.  Equal logits by
// the thousand take this way: a choice of 64 requests of 4 beams of 131072 equal logits takes 0.18 ms with 8, 0.23 ms with 128.
template <int THREADS, int N, typename F>
__device__ __forceinline__ int keep_best(Choice* found, int* n_found, int K, int turns, F of) {
  Choice cut = {0.0, kNone};
  __syncthreads();                                         // everyone has read how many there were
  if (threadIdx.x == 0) *n_found = 0;
  __syncthreads();
  for (int t = 0; t < turns; ++t) {
    Choice x[N];
    uint32_t left = of(t, x);
    for (bool last = false;;) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (!(left >> j & 1)) continue;
        if (cut.rest != kNone && !before(x[j], cut)) {
          left &= ~(1u << j);
          continue;
        }
        const int to = atomicAdd(n_found, 1);
        if (to >= THREADS) continue;
        found[to] = x[j];
        left &= ~(1u << j);
      }
      const bool over = __syncthreads_or(left);
      const int n = min(*n_found, THREADS);
      if (!over && (last || t + 1 < turns || n <= K)) break;
      last = !over;
      cut = keep_k<THREADS>(found, n_found, n, K);
    }
  }
  return *n_found;
}

// One workgroup for a group.  A value that the K best reach comes from 256 disjoint subsets' largest: of every row some lists, since the best
// may all be one row's.  Lists that reach it are read again, and what reaches it in them is sorted.  What is read of the rows' pass is
// requested at once and kept, so that a choice is three round trips: where the group's rows are, their lists, the logits looked at again.  Bound: those
// and the steps between (6..9 us for 1..64 requests of 4 beams, 8 choices; 12 for 32 choices of 16 beams).
template <typename E, bool MASKED, bool TINY, int THREADS, int kHeld>
__global__ __launch_bounds__(THREADS) void select_best_kernel(SelectArgs a, GroupRows g, int group0) {
  __shared__ RowScore rows[kBeamsMost];
  __shared__ float subset[THREADS];
  __shared__ Choice found[THREADS];      // choices that are sorted by counting what comes before each
  __shared__ uint16_t list[THREADS];
  __shared__ int n_list, n_found;
  const int tid = threadIdx.x, K = a.n_best, bits = a.parts_bits, parts = 1 << bits;
  const int row0 = g.row(blockIdx.x), beams = g.rows(blockIdx.x), all = beams << bits;
  const int64_t at0 = (int64_t)row0 << bits;
  const int of_group = all * 64, mine = min(tid, all - 1);
  float most[kHeld];
  int most_at[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int l = min(tid + i * THREADS, of_group - 1);
    most[i] = a.most[at0 * 64 + l];
    most_at[i] = a.most_at[at0 * 64 + l];
  }
  const float ref = a.refs[at0 + mine], score = a.scores[row0 + (mine >> bits)];
  double sum = a.sums[at0 + mine];
  if (tid == 0) n_list = n_found = 0;
  // Of each row the score less the logarithm of its sum, and where its exponents are counted from: a logit is taken from there first,
  // which is exact where it is large, and rows of the type's lowest value alone keep their sum.  A row's parts are neighbouring threads'.
  if (tid < (all + 63 & ~63)) {
    const float c = most_of_parts(ref, bits);
    sum = sum_of_parts(sum * (double)__builtin_amdgcn_exp2f((ref - c) * kLog2e), bits);
    const double b = (double)score - log(sum);
    if (tid < all && (tid & (parts - 1)) == 0) {
      rows[tid >> bits] = RowScore{sum > 0.0 && fabs(b) < (double)INFINITY ? b : -(double)INFINITY, (double)c};
    }
  }
  __syncthreads();
  // scores as 32 bits round them, which keeps their order: at most K - 1 are above one that is below the K-th of any K
  const auto scored = [&](int row, float value) __attribute__((always_inline)) { return ((double)value - rows[row].from) + rows[row].base; };
  float top = -INFINITY, score_of[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int l = tid + i * THREADS;
    score_of[i] = l < of_group ? (float)scored(l >> (6 + bits), most[i]) : -INFINITY;
    top = fmaxf(top, score_of[i]);
  }
  // the K-th largest of 256 subsets' values, or a little less
  subset[tid] = top;
  __syncthreads();
  float of[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int at = j * 64 + (tid & 63);
    of[j] = subset[at];
#pragma unroll
    for (int more = 256; more < THREADS; more += 256) of[j] = fmaxf(of[j], subset[more + at]);
  }
  const float low = reached_by(of, K, K + K / 8);

  const auto see_lists = [&](auto see) __attribute__((always_inline)) {
    if (!(top >= low)) return;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if (score_of[i] >= low) {
        const int row = (tid + i * THREADS) >> (6 + bits);
        see(Choice{scored(row, most[i]), rest_of(row, most[i], most_at[i])}, tid + i * THREADS);
      }
    }
  };
  see_lists([&](const Choice&, int l) __attribute__((always_inline)) {
    const int to = atomicAdd(&n_list, 1);
    if (to < THREADS) list[to] = (uint16_t)l;
  });
  __syncthreads();
  constexpr int N = E::kGroup;
  const int long_part = part_groups<E>(a);
  int lists = n_list;
  if (lists > THREADS) {                                   // many equals: the K best lists hold the K best
    lists = keep_best<THREADS, 1>(found, &n_found, K, (of_group + THREADS - 1) / THREADS, [&](int t, Choice* x) {
      const int l = tid + t * THREADS, row = l >> (6 + bits);
      if (l >= of_group) return 0u;
      const float value = a.most[at0 * 64 + l];
      x[0] = Choice{scored(row, value), rest_of(row, value, a.most_at[at0 * 64 + l])};
      return (float)x[0].score >= low ? 1u : 0u;
    });
    if (tid < lists) {
      const uint64_t of = found[tid].rest;
      const int at = (int)(of & 0xffffff), part = at / long_part;
      list[tid] = (uint16_t)((((int)(of >> 56) << bits) + part) * 64 + ((at - part * long_part) & 63));
    }
    __syncthreads();
    if (tid == 0) n_found = 0;
    __syncthreads();
  }

  // Lanes for a list: as many as it has groups, up to a wavefront.
  const int wide = 32 - __builtin_clz(min(long_part >> 6, 64) * 2 - 1) - 1;
  const int side = tid & ((1 << wide) - 1), at_once = THREADS >> wide;
  const auto list_of = [&](int i, int* row, int* first) __attribute__((always_inline)) {
    const int l = list[i];
    *row = l >> (6 + bits);
    *first = ((l >> 6) & (parts - 1)) * long_part;
    return *first + (l & 63) + side * 64;
  };
  for (int i = tid >> wide; i < lists; i += at_once) {
    int row, first;
    const int from = list_of(i, &row, &first);
    const auto p = part_of<E, MASKED, TINY>(a, row0 + row, first);
#pragma unroll 2
    for (int o = from; o < p.end; o += 64 << wide) {
      float x[N];
      p.read(o, x);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const double s = scored(row, x[j]);
        if ((float)s >= low) {
          const int to = atomicAdd(&n_found, 1);
          if (to < THREADS) found[to] = Choice{s, rest_of(row, x[j], p.token(o, j))};
        }
      }
    }
  }
  __syncthreads();
  int n = n_found;
  if (n > THREADS) {
    const int steps = (long_part + (64 << wide) - 1) / (64 << wide);
    n = keep_best<THREADS, N>(found, &n_found, K, (lists + at_once - 1) / at_once * steps, [&](int t, Choice* best) {
      const int i = (tid >> wide) + t / steps * at_once;
      if (i >= lists) return 0u;
      int row, first;
      const int o = list_of(i, &row, &first) + t % steps * (64 << wide);
      const auto p = part_of<E, MASKED, TINY>(a, row0 + row, first);
      if (o >= p.end) return 0u;
      float x[N];
      p.read(o, x);
      uint32_t reach = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        best[j] = Choice{scored(row, x[j]), rest_of(row, x[j], p.token(o, j))};
        if ((float)best[j].score >= low) reach |= 1u << j;
      }
      return reach;
    });
  } else if (n > kRanked) {                                // ranking takes n * n looks (256 rows of logits rounded to whole numbers, 64 choices: 131 -> 76 us)
    keep_k<THREADS>(found, &n_found, n, K);
    n = K;
  }
  const int64_t out = (int64_t)(group0 + blockIdx.x) * K;
  const auto write = [&](int k, const Choice& x) __attribute__((always_inline)) {
    a.best_scores[out + k] = (float)x.score;
    a.best_beams[out + k] = (int)(x.rest >> 56);
    a.best_tokens[out + k] = (int)(x.rest & 0xffffff);
  };
  for (int i = tid >> 2; i < n; i += THREADS / 4) {         // four lanes count for each
    const Choice x = found[i];
    int rank = 0;
#pragma unroll 4
    for (int k = tid & 3; k < n; k += 4) rank += before(found[k], x);
    rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, false);
    rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, false);
    if (rank < K && (tid & 3) == 0) write(rank, x);
  }
  for (int k = n + tid; k < K; k += THREADS) {
    a.best_scores[out + k] = -INFINITY;
    a.best_beams[out + k] = a.best_tokens[out + k] = -1;
  }
}

// ---- state rows ---------------------------------------------------------------------------------

typedef u32x4_t __attribute__((aligned(1))) u32x4_a1;

// A thread moves columns (16 bytes; the last ones of a row that is no multiple of that, single) of all rows of a group: every row's
// new value is read before the first is written, and no other thread touches the column, so a group may be moved in place.
// Rows that stay are neither read nor written there.  U columns of R rows are under way at a time.  Bound: HBM, read + write.
// 64 groups of 2..6 rows of 32 KB, 16 arrays of them (67 MB read once and written): 12.8 us a call (5.2 TB/s; 13.8 with plain stores, 16.4 with nontemporal
// loads too, since a row that several take is found in the caches, and 41 with one column to a thread, which leaves too little under way).
template <int R, int U>
__global__ __launch_bounds__(kStateThreads) void states_kernel(StatesArgs a, GroupRows g) {
  uint32_t b = blockIdx.x;
  int s = 0;
  while (b >= a.array[s].end) ++s;
  if (s > 0) b -= a.array[s - 1].end;
  const StateArray& x = a.array[s];
  const uint32_t chunk = b % x.chunks, group = b / x.chunks % (uint32_t)a.n_groups, outer = b / x.chunks / (uint32_t)a.n_groups;
  const int row0 = g.row(group), beams = g.rows(group);
  const bool all = x.dst != x.src;
  int from[R];
  uint64_t moves = 0;                                      // rows that change
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int p = sload(a.parents + row0 + min(r, beams - 1));
    from[r] = (uint32_t)p < (uint32_t)beams ? p : r;
    if (r < beams && (all || from[r] != r)) moves |= 1ull << r;
  }
  if (!moves) return;
  // a stretch of U * 4 KB of every row, from a base that is the same for all threads
  const int64_t begin = (int64_t)chunk * (U * kStateThreads * kStateUnit), stretch = min(x.row_bytes - begin, (int64_t)(U * kStateThreads * kStateUnit));
  const int64_t at = (int64_t)outer * x.outer_stride + row0 * x.row_stride + begin;
  const uint8_t* src = x.src + at;
  uint8_t* dst = x.dst + at;
  const uint32_t whole = (uint32_t)stretch / kStateUnit * kStateUnit, rest = (uint32_t)stretch % kStateUnit, mine = threadIdx.x * kStateUnit;
  u32x4_t v[R][U];
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (moves >> r & 1) {
      const uint8_t* row = src + from[r] * x.row_stride;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (mine + u * (kStateThreads * kStateUnit) < whole) v[r][u] = *(const u32x4_a1*)(row + (mine + u * (kStateThreads * kStateUnit)));
    }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (moves >> r & 1) {
      uint8_t* row = dst + r * x.row_stride;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (mine + u * (kStateThreads * kStateUnit) < whole) __builtin_nontemporal_store(v[r][u], (u32x4_a1*)(row + (mine + u * (kStateThreads * kStateUnit))));
    }
  if (threadIdx.x < rest) {
    uint8_t c[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (moves >> r & 1) c[r] = src[from[r] * x.row_stride + whole + threadIdx.x];
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (moves >> r & 1) dst[r * x.row_stride + whole + threadIdx.x] = c[r];
  }
}

template <typename E, bool MASKED, bool TINY>
void launch_rows(const SelectArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.rows * a.parts)), block(64);
  if constexpr (!MASKED && !TINY) {
    const bool far = (int64_t)a.rows * a.vocab * E::kBytes >= kLastLevelBytes;
    if constexpr (E::kBytes == 2) {
      if (((uintptr_t)a.logits & 2) || (a.rows > 1 && (a.stride & 1))) {
        if (far) select_rows_kernel<E, false, false, true, true><<<grid, block, 0, st>>>(a);
        else select_rows_kernel<E, false, false, false, true><<<grid, block, 0, st>>>(a);
        return;
      }
    }
    if (far) {
      select_rows_kernel<E, false, false, true><<<grid, block, 0, st>>>(a);
      return;
    }
  }
  select_rows_kernel<E, MASKED, TINY, false><<<grid, block, 0, st>>>(a);
}
template <typename E, bool MASKED, bool TINY>
void launch_best(const SelectArgs& a, const GroupRows& g, int32_t group0, int32_t n_groups, hipStream_t st) {
  int most = 0;                                            // parts of the largest group
  for (int32_t i = 0; i < (g.each ? 1 : n_groups); ++i) most = std::max(most, g.rows(i) * a.parts);
  const int lists = most * 64, deep = a.part_octets * (kOctet / E::kGroup) / 64;
  const dim3 grid((unsigned)n_groups);
  static_assert(1024 * 16 == 64 * kMostParts, "a thread holds its share of the lists");
  // Half the threads where they hold the lists and what is looked at again is little: calls of 16 and 64 requests of 4 beams of 131072 bf16 logits, 8
  // choices: 14.5 and 22.7 us, with 1024 threads 16.5 and 25.4; 64 requests with 128 choices (a list there is 32 groups): 33, with 512 threads 42.
  if (lists <= kFewLists && a.n_best * deep <= 1024) select_best_kernel<E, MASKED, TINY, kFewThreads, kFewLists / kFewThreads><<<grid, dim3(kFewThreads), 0, st>>>(a, g, group0);
  else select_best_kernel<E, MASKED, TINY, 1024, 16><<<grid, dim3(1024), 0, st>>>(a, g, group0);
}
#define SYM_OF_TYPE(launch, E, ...)                                                     \
  (a.vocab < E::kGroup ? (a.allowed ? launch<E, true, true>(__VA_ARGS__) : launch<E, false, true>(__VA_ARGS__)) \
                    : (a.allowed ? launch<E, true, false>(__VA_ARGS__) : launch<E, false, false>(__VA_ARGS__)))
#define SYM_OF_STEP(launch, ...)                                        \
  (dtype == SYM_F32    ? SYM_OF_TYPE(launch, LogitF32, __VA_ARGS__)     \
   : dtype == SYM_BF16 ? SYM_OF_TYPE(launch, LogitBF16, __VA_ARGS__)    \
                       : SYM_OF_TYPE(launch, LogitF16, __VA_ARGS__))

}  // namespace

hipError_t launch_select_rows(const SelectArgs& a, int dtype, hipStream_t st) {
  SYM_OF_STEP(launch_rows, a, st);
  return hipGetLastError();
}

hipError_t launch_select_best(const SelectArgs& a, const GroupRows& g, int32_t group0, int32_t n_groups, int dtype, hipStream_t st) {
  SYM_OF_STEP(launch_best, a, g, group0, n_groups, st);
  return hipGetLastError();
}
#undef SYM_OF_STEP
#undef SYM_OF_TYPE

hipError_t launch_states(const StatesArgs& a, const GroupRows& g, int32_t most_beams, hipStream_t st) {
  const dim3 grid(a.array[a.n_arrays - 1].end), block(kStateThreads);
  if (most_beams <= 4) states_kernel<4, state_columns(4)><<<grid, block, 0, st>>>(a, g);
  else if (most_beams <= 8) states_kernel<8, state_columns(8)><<<grid, block, 0, st>>>(a, g);
  else if (most_beams <= 16) states_kernel<16, state_columns(16)><<<grid, block, 0, st>>>(a, g);
  else if (most_beams <= 32) states_kernel<32, state_columns(32)><<<grid, block, 0, st>>>(a, g);
  else states_kernel<kBeamsMost, state_columns(kBeamsMost)><<<grid, block, 0, st>>>(a, g);
  return hipGetLastError();
}

}  // namespace symkv
