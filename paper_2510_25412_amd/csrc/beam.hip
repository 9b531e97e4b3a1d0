// Beam search beside the cache: the best continuations of a request's beams, and state rows that follow their beams.
#include <cfloat>

#include "../../include/symphony_kv.h"
#include "beam.hpp"
#include "device.hpp"

namespace symkv {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// ---- steps across the lanes of a wavefront ---------------------------------------------------

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return as_f32(__builtin_amdgcn_update_dpp(as_u32(x), as_u32(x), CTRL, 0xf, 0xf, false));
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
__device__ __forceinline__ double wave_sum(double x) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ int lanes_of(uint64_t b) { return __builtin_popcountll(b); }
__device__ __forceinline__ int lanes_below(uint64_t b) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0)); }

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
    if (count(low) <= limit) return low;
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
  static constexpr int kBytes = 2;
  struct Raw {
    u32x4_t w;
  };
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return Raw{*(const u32x4_a2*)p}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = as_f32(r.w[i] << 16);
      x[2 * i + 1] = as_f32(r.w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw few(const uint8_t* p, int n) { return few16<Raw>(p, n); }
};
struct LogitF16 {
  static constexpr int kBytes = 2;
  struct Raw {
    u32x4_t w;
  };
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return Raw{*(const u32x4_a2*)p}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)r.w[i]);
      x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i] >> 16));
    }
  }
  static __device__ __forceinline__ Raw few(const uint8_t* p, int n) { return few16<Raw>(p, n); }
};
struct LogitF32 {
  static constexpr int kBytes = 4;
  struct Raw {
    u32x4_t w, v;
  };
  static __device__ __forceinline__ Raw load(const uint8_t* p) { return Raw{*(const u32x4_a4*)p, *(const u32x4_a4*)(p + 16)}; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = as_f32(r.w[i]);
      x[4 + i] = as_f32(r.v[i]);
    }
  }
  static __device__ __forceinline__ Raw few(const uint8_t* p, int n) {
    Raw r = {};
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < n) (j < 4 ? r.w : r.v)[j & 3] = ((const uint32_t*)p)[j];
    return r;
  }
};

constexpr int kAhead = 4;              // octets of a lane under way; a part's maxima are kept apart by their place among these
constexpr int kFound = 256;            // logits that a wavefront sorts
constexpr int kLists = 4 * 64;         // maxima of a part

// One wavefront: a part of a row, 8 logits (an octet) to a lane at a time.  What it reads is counted from the row's start,
// whatever the address, so equal rows give equal results.  TINY: rows of less than an octet, read one by one.
template <typename E, bool MASKED, bool TINY>
struct Part {
  const uint8_t* row;
  const uint8_t* bits;
  int vocab, first, end;               // octets of this part

  // Octet o.  The last one of a row that does not end with it: the row's last 8 logits.  What is not wanted comes from where others read.
  __device__ __forceinline__ typename E::Raw raw(int o, bool want) const {
    if constexpr (TINY) return E::few(row, vocab);
    const int at = min((want ? o : first) * kOctet, vocab - kOctet);
    return E::load(row + (int64_t)at * E::kBytes);
  }
  __device__ __forceinline__ uint32_t allowed(int o) const {
    const bool in = o < end;
    const uint32_t m = MASKED ? bits[in ? o : first] : 0xffu;
    return in ? m : 0;
  }
  // -inf in the place of what does not count.  m: the octet's allowed bits
  __device__ __forceinline__ void mask(float (&x)[8], int o, uint32_t m) const {
    const int over = (o + 1) * kOctet - vocab;             // more than a row's last octet holds
    if constexpr (TINY) m = over > 0 ? m & (0xffu >> over) : m;
    else m = over > 0 ? m << over : m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t keep = (uint32_t)((int32_t)(m << (31 - j)) >> 31);
      x[j] = as_f32((as_u32(x[j]) & keep) | (0xff800000u & ~keep));
    }
  }
  __device__ __forceinline__ int token(int o, int j) const { return (TINY ? 0 : min(o * kOctet, vocab - kOctet)) + j; }
  // Octet o's logits, masked
  __device__ __forceinline__ void read(int o, float (&x)[8]) const {
    const uint32_t m = allowed(o);
    E::unpack(raw(o, m != 0), x);
    mask(x, o, m);
  }
};

struct Found {
  float value;
  int token;
};
__device__ __forceinline__ bool before(float v, int t, float w, int u) { return v > w || (v == w && t < u); }

// The K best of a part, where more than kFound logits reach the value that should have left about K: exactly the K-th largest is
// found by halves over the whole part, then what is above it and of its equals the first.  Returns how many there are, in f.
template <typename P>
__device__ __attribute__((noinline)) int equals_too(const P& p, int K, float low, float top, Found* f) {
  const int lane = threadIdx.x & 63;
  const auto count = [&](auto reaches) {
    int n = 0;
    for (int o = p.first + lane; o - lane < p.end; o += 64) {
      float x[8];
      p.read(o, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) n += reaches(x[j]);
    }
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    return n;
  };
  uint32_t lo = __builtin_amdgcn_readfirstlane(key_of(low)), hi = __builtin_amdgcn_readfirstlane(key_of(top)) + 1;
  while (hi > lo + 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const float t = of_key(mid);
    if (__builtin_amdgcn_readfirstlane(count([t](float v) { return v >= t; })) >= K) lo = mid;
    else hi = mid;
  }
  const float t = of_key(lo);
  const int above = __builtin_amdgcn_readfirstlane(count([t](float v) { return v > t; }));
  int n_above = 0, n_equal = 0;
  for (int o = p.first + lane; o - lane < p.end; o += 64) {
    float x[8];
    p.read(o, x);
    int equal_before = 0, above_before = 0, equal_all = 0, above_all = 0;      // of lower lanes, of the wavefront
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint64_t e = __ballot(x[j] == t), g = __ballot(x[j] > t);
      equal_before += lanes_below(e);
      equal_all += lanes_of(e);
      above_before += lanes_below(g);
      above_all += lanes_of(g);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (x[j] > t) f[n_above + above_before++] = Found{x[j], p.token(o, j)};
      if (x[j] == t) {
        const int at = above + n_equal + equal_before++;
        if (at < K) f[at] = Found{t, p.token(o, j)};
      }
    }
    n_above += above_all;
    n_equal += equal_all;
  }
  return min(K, above + n_equal);
}

template <typename E, bool MASKED, bool TINY>
__global__ __launch_bounds__(64) void select_rows_kernel(SelectArgs a) {
  __shared__ Found found[kFound];
  __shared__ uint16_t lists[kLists];
  const int lane = threadIdx.x & 63, K = a.n_best;
  const int row = (int)(blockIdx.x / (uint32_t)a.parts), part = (int)(blockIdx.x % (uint32_t)a.parts);
  const int64_t list = blockIdx.x;
  float* values = a.values + list * K;
  int32_t* tokens = a.tokens + list * K;
  const auto nothing = [&](int from) {
    for (int k = from + lane; k < K; k += 64) {
      values[k] = -INFINITY;
      tokens[k] = -1;
    }
  };
  const float score = a.scores[row];
  if (!(fabsf(score) < INFINITY)) {                        // no beam lives here
    if (lane == 0) {
      a.sums[list] = 0.0;
      a.refs[list] = -FLT_MAX;
    }
    nothing(0);
    return;
  }
  Part<E, MASKED, TINY> p;
  p.row = (const uint8_t*)a.logits + (int64_t)row * a.stride * E::kBytes;
  p.bits = MASKED ? a.allowed + (int64_t)row * a.allowed_stride : nullptr;
  p.vocab = a.vocab;
  p.first = part * a.part_octets;
  p.end = min(p.first + a.part_octets, (a.vocab + kOctet - 1) / kOctet);
  const int whole = min(p.end, a.vocab / kOctet);          // octets that need no look at the row's end

  // One pass: sums of exp(x - c), eight to a lane, and the maxima.  c is a lane's largest logit so far, so that no exponent is positive: a
  // rounding of (x - c) log2 e then weighs at most 2^-24 of the sum, where with c some way below the largest it would weigh that many times as much.
  float c = -FLT_MAX, s[8] = {}, most[kAhead];
#pragma unroll
  for (int d = 0; d < kAhead; ++d) most[d] = -INFINITY;
  const int batches = (p.end - p.first + 64 * kAhead - 1) / (64 * kAhead);
  typename E::Raw cur[kAhead], next[kAhead];
  uint32_t m[kAhead], m_next[kAhead], m_later[kAhead];
  const auto octet = [&](int i, int d) __attribute__((always_inline)) { return p.first + (i * kAhead + d) * 64 + lane; };
#pragma unroll
  for (int d = 0; d < kAhead; ++d) m[d] = p.allowed(octet(0, d));
#pragma unroll
  for (int d = 0; d < kAhead; ++d) m_next[d] = p.allowed(octet(1, d));
#pragma unroll
  for (int d = 0; d < kAhead; ++d) cur[d] = p.raw(octet(0, d), m[d] != 0);
  for (int i = 0; i < batches; ++i) {
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
      m_later[d] = p.allowed(octet(i + 2, d));
      next[d] = p.raw(octet(i + 1, d), m_next[d] != 0);
    }
    const bool plain = !MASKED && !TINY && p.first + (i + 1) * kAhead * 64 <= whole;
    float x[kAhead][8], to = c;
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
      E::unpack(cur[d], x[d]);
      if (!plain) p.mask(x[d], octet(i, d), m[d]);
      const float top = fmaxf(fmaxf(fmaxf(x[d][0], x[d][1]), fmaxf(x[d][2], x[d][3])), fmaxf(fmaxf(x[d][4], x[d][5]), fmaxf(x[d][6], x[d][7])));
      most[d] = fmaxf(most[d], top);
      to = fmaxf(to, top);
    }
    const float by = __builtin_amdgcn_exp2f((c - to) * kLog2e);
    c = to;
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] *= by;
#pragma unroll
    for (int d = 0; d < kAhead; ++d)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += __builtin_amdgcn_exp2f((x[d][j] - c) * kLog2e);
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
      cur[d] = next[d];
      m[d] = m_next[d];
      m_next[d] = m_later[d];
    }
  }
  const float ref = across<6>(c, Larger());
  const double sum = wave_sum((double)(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]))) * (double)__builtin_amdgcn_exp2f((c - ref) * kLog2e));
  if (lane == 0) {
    a.sums[list] = sum;
    a.refs[list] = ref;
  }
  if (!(sum > 0.0)) return nothing(0);                     // nothing allowed, or no distribution

  // The K best: only lists (a lane, a place among those ahead) whose maximum is among the K largest can hold one.  These are read
  // again, and what reaches the K-th largest maximum is sorted by counting what comes before it.
  const float top = across<6>(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])), Larger());
  const float low = reached_by(most, K, K + 4);
  int n_lists = 0;
#pragma unroll
  for (int d = 0; d < kAhead; ++d) {
    const bool in = most[d] >= low;
    const uint64_t b = __ballot(in);
    if (in) lists[n_lists + lanes_below(b)] = (uint16_t)(d * 64 + lane);
    n_lists += lanes_of(b);
  }
  __syncthreads();
  int n = 0;
  const int work = n_lists * batches;
  for (int w = lane; w - lane < work; w += 64) {
    float x[8];
    const int at = w < work ? w / batches : 0;
    const int l = lists[at], o = w < work ? p.first + (w - at * batches) * (kAhead * 64) + l : p.end;
    p.read(o, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool in = x[j] >= low;
      const uint64_t b = __ballot(in);
      const int to = n + lanes_below(b);
      if (in && to < kFound) found[to] = Found{x[j], p.token(o, j)};
      n += lanes_of(b);
    }
  }
  if (n > kFound) n = equals_too(p, K, low, top, found);
  __syncthreads();
  for (int k0 = 0; k0 < n; k0 += 64) {
    const Found mine = found[min(k0 + lane, n - 1)];
    int rank = k0 + lane < n ? 0 : K;
    for (int k = 0; k < n; ++k) {
      const Found other = found[k];
      rank += before(other.value, other.token, mine.value, mine.token);
    }
    if (rank < K) {
      values[rank] = mine.value;
      tokens[rank] = mine.token;
    }
  }
  nothing(n);
}

// ---- a group's choice among its rows' parts --------------------------------------------------------

struct Choice {
  double score;
  float value;
  int row, token;
};
// Scores of one row are in the order of its logits even where 64 bits cannot tell them apart.
__device__ __forceinline__ bool before(const Choice& a, const Choice& b) {
  if (a.score != b.score) return a.score > b.score;
  if (a.row != b.row) return a.row < b.row;
  return before(a.value, a.token, b.value, b.token);
}

constexpr int kChoices = 512;
__global__ __launch_bounds__(256) void select_best_kernel(SelectArgs a, GroupRows g, int group0) {
  __shared__ double base[kBeamsMost], sums[kMostLists];
  __shared__ float refs[kMostLists], heads[kMostLists], from[kBeamsMost], least;
  __shared__ Choice choice[kChoices];
  __shared__ int count;
  const int tid = threadIdx.x, K = a.n_best, parts = a.parts;
  const int row0 = g.base + g.first[blockIdx.x], beams = g.first[blockIdx.x + 1] - g.first[blockIdx.x], lists = beams * parts;
  const int64_t list0 = (int64_t)row0 * parts;
  float head = -INFINITY;
  if (tid < lists) {
    refs[tid] = a.refs[list0 + tid];
    sums[tid] = a.sums[list0 + tid];
    head = a.values[(list0 + tid) * K];
  }
  if (tid == 0) count = 0;
  __syncthreads();
  // Of each row the score less the logarithm of its sum, and where its exponents are counted from: a logit is taken from there first,
  // which is exact where it is large, and rows of the type's lowest value alone keep their sum.
  if (tid < beams) {
    float c = -FLT_MAX;
    for (int p = 0; p < parts; ++p) c = fmaxf(c, refs[tid * parts + p]);
    double s = 0.0;
    for (int p = 0; p < parts; ++p) s += sums[tid * parts + p] * (double)__builtin_amdgcn_exp2f((refs[tid * parts + p] - c) * kLog2e);
    const double b = (double)a.scores[row0 + tid] - log(s);
    base[tid] = s > 0.0 && fabs(b) < (double)INFINITY ? b : -(double)INFINITY;
    from[tid] = c;
  }
  __syncthreads();
  // No choice is below the K-th largest of the lists' best, as 32 bits round them.
  heads[tid] = tid < lists ? (float)(((double)head - (double)from[tid / parts]) + base[tid / parts]) : -INFINITY;
  __syncthreads();
  if (tid < 64) {
    const float x[4] = {heads[tid], heads[64 + tid], heads[128 + tid], heads[192 + tid]};
    const float l = reached_by(x, K, K + 16);
    if (tid == 0) least = l;
  }
  __syncthreads();
  const float low = least;
  const int entries = lists * K;
  const auto entry = [&](int e) {
    Choice x;
    x.row = e / K / parts;
    x.value = a.values[list0 * K + e];
    x.token = a.tokens[list0 * K + e];
    x.score = ((double)x.value - (double)from[x.row]) + base[x.row];
    return x;
  };
  for (int e = tid; e < entries; e += 256) {
    const Choice x = entry(e);
    if ((float)x.score >= low) {
      const int at = atomicAdd(&count, 1);
      if (at < kChoices) choice[at] = x;
    }
  }
  __syncthreads();
  const int64_t out = (int64_t)(group0 + blockIdx.x) * K;
  const auto write = [&](int k, const Choice& x) {
    a.best_scores[out + k] = (float)x.score;
    a.best_beams[out + k] = x.row;
    a.best_tokens[out + k] = x.token;
  };
  int n = count;
  if (n <= kChoices) {
    for (int i = tid; i < n; i += 256) {
      const Choice mine = choice[i];
      int rank = 0;
      for (int k = 0; k < n; ++k) rank += before(choice[k], mine);
      if (rank < K) write(rank, mine);
    }
  } else {                                                 // many equals: one choice after the other
    n = K;
    Choice last;
    for (int k = 0; k < K; ++k) {
      Choice best = {-(double)INFINITY, 0.f, -1, -1};
      for (int e = tid; e < entries; e += 256) {
        const Choice x = entry(e);
        if ((float)x.score >= low && (k == 0 || before(last, x)) && (best.row < 0 || before(x, best))) best = x;
      }
      choice[tid] = best;
      __syncthreads();
      for (int d = 128; d; d >>= 1) {
        if (tid < d && choice[tid + d].row >= 0 && (choice[tid].row < 0 || before(choice[tid + d], choice[tid]))) choice[tid] = choice[tid + d];
        __syncthreads();
      }
      last = choice[0];
      if (tid == 0) write(k, last);
      __syncthreads();
    }
  }
  for (int k = n + tid; k < K; k += 256) {
    a.best_scores[out + k] = -INFINITY;
    a.best_beams[out + k] = a.best_tokens[out + k] = -1;
  }
}

// ---- state rows ---------------------------------------------------------------------------------

typedef u32x4_t __attribute__((aligned(1))) u32x4_a1;

// A thread moves one column (16 bytes; the last ones of a row that is no multiple of that, single) of all rows of a group: every row's
// new value is read before the first is written, and no other thread touches the column, so a group may be moved in place.
// Rows that stay are neither read nor written there.  Bound: HBM, read + write.
template <int R, typename V>
__device__ __forceinline__ void move_column(uint8_t* dst, const uint8_t* src, int64_t stride, int beams, const int (&from)[R], bool all) {
  V v[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r < beams && (all || from[r] != r)) v[r] = *(const V*)(src + from[r] * stride);
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r < beams && (all || from[r] != r)) *(V*)(dst + r * stride) = v[r];
}

template <int R>
__global__ __launch_bounds__(kStateThreads) void states_kernel(StatesArgs a, GroupRows g) {
  uint32_t b = blockIdx.x;
  int s = 0;
  while (b >= a.array[s].end) ++s;
  if (s > 0) b -= a.array[s - 1].end;
  const StateArray& x = a.array[s];
  const uint32_t chunk = b % x.chunks, group = b / x.chunks % (uint32_t)a.n_groups, outer = b / x.chunks / (uint32_t)a.n_groups;
  const int row0 = g.base + g.first[group], beams = g.first[group + 1] - g.first[group];
  const bool all = x.dst != x.src;
  int from[R];
  bool moves = all;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    from[r] = r;
    if (r < beams) {
      const int p = sload(a.parents + row0 + r);
      from[r] = (uint32_t)p < (uint32_t)beams ? p : r;
      moves = moves || from[r] != r;
    }
  }
  if (!moves) return;
  const int64_t units = x.row_bytes / kStateUnit, unit = (int64_t)chunk * kStateThreads + threadIdx.x;
  const int64_t rest = x.row_bytes % kStateUnit, at = (int64_t)outer * x.outer_stride + row0 * x.row_stride;
  if (unit < units) move_column<R, u32x4_a1>(x.dst + at + unit * kStateUnit, x.src + at + unit * kStateUnit, x.row_stride, beams, from, all);
  else if (unit < units + rest) {
    const int64_t byte = units * kStateUnit + (unit - units);
    move_column<R, uint8_t>(x.dst + at + byte, x.src + at + byte, x.row_stride, beams, from, all);
  }
}

template <typename E>
void launch_rows(const SelectArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.rows * a.parts)), block(64);
  if (a.vocab < kOctet) {
    if (a.allowed) select_rows_kernel<E, true, true><<<grid, block, 0, st>>>(a);
    else select_rows_kernel<E, false, true><<<grid, block, 0, st>>>(a);
  } else if (a.allowed) {
    select_rows_kernel<E, true, false><<<grid, block, 0, st>>>(a);
  } else {
    select_rows_kernel<E, false, false><<<grid, block, 0, st>>>(a);
  }
}

}  // namespace

hipError_t launch_select_rows(const SelectArgs& a, int dtype, hipStream_t st) {
  if (dtype == SYM_F32) launch_rows<LogitF32>(a, st);
  else if (dtype == SYM_BF16) launch_rows<LogitBF16>(a, st);
  else launch_rows<LogitF16>(a, st);
  return hipGetLastError();
}

hipError_t launch_select_best(const SelectArgs& a, const GroupRows& g, int32_t group0, int32_t n_groups, hipStream_t st) {
  select_best_kernel<<<dim3((unsigned)n_groups), dim3(256), 0, st>>>(a, g, group0);
  return hipGetLastError();
}

hipError_t launch_states(const StatesArgs& a, const GroupRows& g, int32_t most_beams, hipStream_t st) {
  const dim3 grid(a.array[a.n_arrays - 1].end), block(kStateThreads);
  if (most_beams <= 4) states_kernel<4><<<grid, block, 0, st>>>(a, g);
  else if (most_beams <= 8) states_kernel<8><<<grid, block, 0, st>>>(a, g);
  else if (most_beams <= 16) states_kernel<16><<<grid, block, 0, st>>>(a, g);
  else if (most_beams <= 32) states_kernel<32><<<grid, block, 0, st>>>(a, g);
  else states_kernel<kBeamsMost><<<grid, block, 0, st>>>(a, g);
  return hipGetLastError();
}

}  // namespace symkv
