// HIP kernels (gfx950 / CDNA4) of what comes before and beside dense attention on long files: rotary positions of query and key
// rows, appends that turn the keys on their way into the pages, bounds of the pages' keys, the choice of pages by those bounds
// and attention over the chosen pages.
#include <hip/hip_runtime.h>
#include <hip/hip_ext.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "device.hpp"
#include "sparse.hpp"

namespace symkv {

namespace {

#define SYM_AS4 const __attribute__((address_space(4)))

// Storage of two elements in one or two words.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {      // to nearest even, as every conversion to the storage type
  const bf16x2_t v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
// The rounding to 32 bits on the way to 16, which the compiler would otherwise leave out (it rounds 64 bits to bf16 in one go, in a dozen
// instructions): a caller who computes a rotation with elementwise operations gets these bits.
__device__ __forceinline__ float round_f32(double x) {
  float f = (float)x;
  asm("" : "+v"(f));
  return f;
}
template <typename E>
__device__ __forceinline__ u32x4_t pack_chunk(const float* y) {
  if constexpr (E::kDimsPerChunk == 8) return u32x4_t{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
  else return u32x4_t{as_u32(y[0]), as_u32(y[1]), as_u32(y[2]), as_u32(y[3])};
}

// ---------------------------------------------------------------------------------------
// Rotary positions.  Pair (x1, x2) of a row at position p turns by the angle 2 pi p t, t turns per position:
//   y1 = m (x1 cos - x2 sin),  y2 = m (x2 cos + x1 sin).
// In 64 bits: p t loses its fraction in 32 bits at far positions, and a key that is rounded to its neighbour in the storage type
// (it takes an error of 2^-25 in a cosine) shows in the outputs of attention as 1e-5.  The angle is reduced to p t - round(p t) turns, so that
// sincospi's argument is exact.  A workgroup computes the angles of its tokens once, into LDS, for all heads; a thread then keeps
// those of its two 16-byte chunks in registers and walks the token's rows with them.
// Bound: HBM, read + write: 16384 rows of 32 + 8 bf16 heads in 65 us, 336 MB at 5.2 TB/s (a copy of that size reaches 4.8).  64 rows
// take 4.3 us, a launch and one angle's arithmetic.
// ---------------------------------------------------------------------------------------
constexpr int kPairs = 64;                       // pairs of a head at most
constexpr int kRunTokens = kP;                   // most tokens of a workgroup

__device__ __forceinline__ double2 angle_of(SYM_AS4 RopeTable* r, int pos, int i) {
  double x = (double)pos * r->turns[i], s, c;
  x -= rint(x);
  sincospi(2.0 * x, &s, &c);
  return make_double2(r->mag * c, r->mag * s);
}

struct RowAt {
  const uint8_t* src;
  uint8_t* dst;
  int half;                                      // bytes from the first to the second 128-byte half of the destination
  bool turns;
};

// Rows of `ntok` tokens, `rpt` of each, 2^lg of the workgroup's 256 threads to a token: row_at(token, row) says where from and where to.
// Eight threads to a row, two chunks each, so that a thread holds both elements of its pairs (a row may be turned in place).
// angles() fills cs and ends with a barrier; the first U rows of every thread are under way while it runs.
template <typename E, int PATH, int U, typename R, typename A>
__device__ __forceinline__ void turn_rows(const R& row_at, const A& angles, const int rpt, const int ntok, const int lg, const int dims,
                                          const double2 (*cs)[kPairs], uint8_t (*stage)[kRowBytes]) {
  constexpr int C = E::kDimsPerChunk;
  const int tid = threadIdx.x, j = tid & 7;
  const int tok = min(tid >> lg, ntok - 1), rl = (tid & ((1 << lg) - 1)) >> 3, nrl = 1 << (lg - 3);
  const bool mine = (tid >> lg) < ntok;
  const int hr = dims / 2 / C;                   // HALVES: chunks of the first half of what turns
  int c0 = j, c1 = j + 8;
  bool lane_turns = PATH != ROPE_NONE;
  if constexpr (PATH == ROPE_HALVES) {
    lane_turns = j < hr;
    c0 = lane_turns ? j : 2 * j;                 // the rest of the row, two chunks in a row: 2 hr + 2 (j - hr)
    c1 = lane_turns ? j + hr : c0 + 1;
  }
  u32x4_t x[U][2];
  auto request = [&](int row0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {                // past the end the last row is read again and not stored
      const RowAt at = row_at(tok, min(row0 + u * nrl, rpt - 1));
      x[u][0] = *(const u32x4_t*)(at.src + c0 * 16);
      x[u][1] = *(const u32x4_t*)(at.src + c1 * 16);
    }
  };
  request(rl);
  angles();
  double c[C], s[C];
  if constexpr (PATH == ROPE_HALVES || PATH == ROPE_INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const int i = PATH == ROPE_HALVES ? (lane_turns ? j * C + e : 0) : e < C / 2 ? j * (C / 2) + e : (j + 8) * (C / 2) + e - C / 2;
      const double2 t = cs[tok][i];
      c[e] = t.x;
      s[e] = t.y;
    }
  }
  for (int base = 0;; ) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = base + u * nrl + rl;
      const RowAt at = row_at(tok, min(row, rpt - 1));
      u32x4_t y[2] = {x[u][0], x[u][1]};
      if constexpr (PATH == ROPE_HALVES) {
        if (lane_turns && at.turns) {
          float a[C], b[C], ya[C], yb[C];
          E::unpack(__builtin_bit_cast(uint4, x[u][0]), a);
          E::unpack(__builtin_bit_cast(uint4, x[u][1]), b);
#pragma unroll
          for (int e = 0; e < C; ++e) {
            ya[e] = round_f32((double)a[e] * c[e] - (double)b[e] * s[e]);
            yb[e] = round_f32((double)b[e] * c[e] + (double)a[e] * s[e]);
          }
          y[0] = pack_chunk<E>(ya);
          y[1] = pack_chunk<E>(yb);
        }
      } else if constexpr (PATH == ROPE_INTERLEAVED) {
        if (at.turns) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float a[C], ya[C];
            E::unpack(__builtin_bit_cast(uint4, x[u][h]), a);
#pragma unroll
            for (int p = 0; p < C / 2; ++p) {
              const double ce = c[h * (C / 2) + p], se = s[h * (C / 2) + p];
              ya[2 * p] = round_f32((double)a[2 * p] * ce - (double)a[2 * p + 1] * se);
              ya[2 * p + 1] = round_f32((double)a[2 * p + 1] * ce + (double)a[2 * p] * se);
            }
            const u32x4_t t = pack_chunk<E>(ya);
#pragma unroll
            for (int w = 0; w < 4; ++w)          // a word holds one pair (bf16) or half of one
              if (((h ? c1 : c0) * C + w * (C / 4)) < dims) y[h][w] = t[w];
          }
        }
      } else if constexpr (PATH == ROPE_HALVES_ANY) {
        // the other element of a pair lies anywhere in the row: through LDS
        __syncthreads();
        *(u32x4_t*)(stage[tid >> 3] + c0 * 16) = x[u][0];
        *(u32x4_t*)(stage[tid >> 3] + c1 * 16) = x[u][1];
        __syncthreads();
        if (at.turns) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int d0 = (h ? c1 : c0) * C;
            float a[C], ya[C];
            E::unpack(__builtin_bit_cast(uint4, x[u][h]), a);
#pragma unroll
            for (int e = 0; e < C; ++e) {
              const int d = d0 + e, i = d < dims / 2 ? d : d - dims / 2;
              const bool in = d < dims;
              const int other = in ? (d < dims / 2 ? d + dims / 2 : i) : d;
              float o;
              if constexpr (C == 8) o = as_f32((uint32_t)((const uint16_t*)stage[tid >> 3])[other] << 16);
              else o = ((const float*)stage[tid >> 3])[other];
              const double2 t = cs[tok][in ? i : 0];
              ya[e] = in ? round_f32((double)a[e] * t.x + (d < dims / 2 ? -(double)o : (double)o) * t.y) : a[e];
            }
            const u32x4_t t = pack_chunk<E>(ya);
            if (d0 < dims) y[h] = t;
          }
        }
      }
      if (mine && row < rpt) {
        *(u32x4_t*)(at.dst + (c0 >> 3) * at.half + (c0 & 7) * 16) = y[0];
        *(u32x4_t*)(at.dst + (c1 >> 3) * at.half + (c1 & 7) * 16) = y[1];
      }
    }
    base += U * nrl;
    if (base >= rpt) break;
    request(base + rl);
  }
}

// Angles of `n` tokens, at positions pos[..] or from pos0 on, into cs.
template <int PATH>
__device__ __forceinline__ void fill_angles(SYM_AS4 RopeTable* r, const int32_t* pos, const int pos0, const int n, double2 (*cs)[kPairs]) {
  if constexpr (PATH != ROPE_NONE) {
    const int pairs = r->dims / 2;
    for (int i = threadIdx.x; i < n * kPairs; i += 256)
      if (i % kPairs < pairs) cs[i / kPairs][i % kPairs] = angle_of(r, pos ? pos[i / kPairs] : pos0 + i / kPairs, i % kPairs);
  }
  __syncthreads();
}

// Query and key rows of a batch, turned on their own.  Bound: HBM, read + write.
struct RopeRowsKernelArgs {
  RopeRowsArgs a;
  RopeTable r;
};
template <typename E, int PATH>
__global__ __launch_bounds__(256) void rope_rows_kernel(RopeRowsKernelArgs) {
  __shared__ double2 cs[4][kPairs];
  __shared__ __align__(16) uint8_t stage[PATH == ROPE_HALVES_ANY ? 32 : 1][kRowBytes];
  // the arguments where they lie: named as a parameter and indexed by the thread, the table would be copied to scratch
  auto ka = (SYM_AS4 RopeRowsKernelArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  const int per = ka->a.tokens, t0 = blockIdx.x * per, n = min(per, ka->a.n - t0);
  const int hq = ka->a.q ? ka->a.Hq : 0, hk = ka->a.k ? ka->a.Hkv : 0;
  const uint8_t* q = (const uint8_t*)ka->a.q + (int64_t)t0 * hq * kRowBytes;
  const uint8_t* k = (const uint8_t*)ka->a.k + (int64_t)t0 * hk * kRowBytes;
  uint8_t* qo = (uint8_t*)ka->a.q_out + (int64_t)t0 * hq * kRowBytes;
  uint8_t* ko = (uint8_t*)ka->a.k_out + (int64_t)t0 * hk * kRowBytes;
  const int32_t* pos = ka->a.pos + t0;
  turn_rows<E, PATH, 4>(
      [&](int tok, int row) __attribute__((always_inline)) {
        const bool is_q = row < hq;
        const int64_t off = (int64_t)(is_q ? tok * hq + row : tok * hk + row - hq) * kRowBytes;
        return RowAt{(is_q ? q : k) + off, (is_q ? qo : ko) + off, kHalfBytes, true};
      },
      [&]() __attribute__((always_inline)) { fill_angles<PATH>(&ka->r, pos, 0, n, cs); }, hq + hk, n, per == 1 ? 8 : 6, ka->r.dims, cs, stage);
}

// Bounds of one (page, kv head): elementwise minimum and maximum of its 16 keys, by one wavefront.  Lane (r, j) reads chunk j of
// both halves of tokens r and 8 + r; the eight lanes of a chunk are combined by halving exchanges over the list [lo, -hi]
// (the minimum of -x is -maximum), which leave lane r with entries r V/8 .. of it.  A NaN makes both bounds of its element NaN.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
struct PageKeys {
  uint4 k[4];                                    // index = row half * 2 + token half
};
template <bool STREAM>
__device__ __forceinline__ void load_keys(PageKeys& R, const uint8_t* slab) {
#pragma unroll
  for (int x = 0; x < 4; ++x) R.k[x] = ld16<STREAM>(slab + x * 1024 + (threadIdx.x & 63) * 16);
}
template <typename E>
__device__ __forceinline__ void write_bounds(const PageKeys& R, uint8_t* out) {
  constexpr int C = E::kDimsPerChunk, V = 4 * C;
  const int lane = threadIdx.x & 63, r = lane >> 3, j = lane & 7;
  const uint4* k = R.k;
  float v[V];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float a[C], b[C];
    E::unpack(k[2 * h], a);
    E::unpack(k[2 * h + 1], b);
#pragma unroll
    for (int e = 0; e < C; ++e) {
      v[h * C + e] = least(a[e], b[e]);
      v[V / 2 + h * C + e] = least(-a[e], -b[e]);
    }
  }
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    const auto sw = __builtin_amdgcn_permlane32_swap(as_u32(v[i]), as_u32(v[i + V / 2]), false, false);
    v[i] = least(as_f32(sw[0]), as_f32(sw[1]));
  }
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    const auto sw = __builtin_amdgcn_permlane16_swap(as_u32(v[i]), as_u32(v[i + V / 4]), false, false);
    v[i] = least(as_f32(sw[0]), as_f32(sw[1]));
  }
  const bool b3 = (lane & 8) != 0;
#pragma unroll
  for (int i = 0; i < V / 8; ++i) {
    const float keep = b3 ? v[i + V / 8] : v[i], send = b3 ? v[i] : v[i + V / 8];
    v[i] = least(keep, row_xor8(send));
  }
  const bool top = r >= 4;
  const int at = (r & 3) * (V / 8);              // entry of lo (or hi): dim (at / C) 8 C + j C + at % C
#pragma unroll
  for (int i = 0; i < V / 8; ++i) v[i] = top ? -v[i] : v[i];
  uint2 w;
  if constexpr (C == 8) w = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  else w = make_uint2(as_u32(v[0]), as_u32(v[1]));
  *(uint2*)(out + (top ? kRowBytes : 0) + (at / C) * kHalfBytes + j * 16 + (at % C) * (16 / C)) = w;
}

// ---------------------------------------------------------------------------------------
// Append with the keys turned on the way.  A workgroup takes a run, the new tokens of a file that go to consecutive slots of one page, one
// layer: its keys and values, or one of them where runs are long.  Few runs travel with the kernel's arguments, so that no request over
// the host link stands before the first load.  When the run completes its page, the workgroup of the keys writes the page's bounds
// behind its own stores.  Bound: HBM, read + write: 7500 tokens of 8 bf16 heads in 16 us, 63 MB at 3.9 TB/s (940 workgroups that all run at
// once: start, list, rows, angles and bounds show); 64 files of one token 4.8 us: the launch and a chain of two loads, an angle and a store.
// ---------------------------------------------------------------------------------------
struct ArgRuns {
  int32_t w[kArgRuns * RUN_WORDS];
};
struct AppendKernelArgs {
  AppendRopeArgs a;
  RopeTable r;
};
struct AppendRunsKernelArgs {
  AppendKernelArgs k;
  ArgRuns runs;
};
template <typename E, int PATH>
__device__ __forceinline__ void append_run(SYM_AS4 AppendKernelArgs* ka, const int t0, const int slot, const int nf, const int pos0, const int layer, const int part, const int parts, const bool apart,
                                           double2 (*cs)[kPairs], uint8_t (*stage)[kRowBytes]) {
  const int n = nf & 0xff, Hkv = ka->a.Hkv, Hq = ka->a.q ? ka->a.Hq : 0;
  // this workgroup's rows of a token: keys and values (part -1) or, where they are apart, keys (-2) or values (-1); or a part of the query rows
  const int first = part >= 0 ? 2 * Hkv + Hq * part / parts : apart && part == -1 ? Hkv : 0;
  const int rows = (part >= 0 ? 2 * Hkv + Hq * (part + 1) / parts : part == -2 ? Hkv : 2 * Hkv) - first;
  if (rows <= 0) return;
  uint8_t* page = ka->a.pool + layer * ka->a.layer_bytes + (int64_t)(slot / kP) * ka->a.page_bytes;
  const int ts = slot % kP;
  const uint8_t* k = (const uint8_t*)ka->a.k + layer * ka->a.layer_rows + (int64_t)t0 * Hkv * kRowBytes;
  const uint8_t* v = (const uint8_t*)ka->a.v + layer * ka->a.layer_rows + (int64_t)t0 * Hkv * kRowBytes;
  const uint8_t* q = (const uint8_t*)ka->a.q + (int64_t)t0 * Hq * kRowBytes;
  uint8_t* qo = (uint8_t*)ka->a.q_out + (int64_t)t0 * Hq * kRowBytes;
  const int32_t* pos = ka->a.pos ? ka->a.pos + t0 : nullptr;
  const int lg = n == 1 ? 8 : n == 2 ? 7 : n <= 4 ? 6 : n <= 8 ? 5 : 4;
  turn_rows<E, PATH, 4>(
      [=](int tok, int x) __attribute__((always_inline)) {
        const int row = first + x;
        // all three of everything, then the choice: under branches the compiler chooses between addresses of the captured variables,
        // and these go to memory
        const bool is_q = row >= 2 * Hkv, is_v = row >= Hkv;
        const int g = is_v ? row - Hkv : row;
        const int64_t from_q = (int64_t)(tok * Hq + row - 2 * Hkv) * kRowBytes, from = (int64_t)(tok * Hkv + g) * kRowBytes;
        const uint8_t *sq = q + from_q, *sv = v + from, *sk = k + from;
        uint8_t *dq = qo + from_q, *dk = page + (int64_t)g * kSlab + (is_v ? kBlk : 0) + (ts + tok) * kHalfBytes;
        return RowAt{is_q ? sq : is_v ? sv : sk, is_q ? dq : dk, is_q ? kHalfBytes : kP * kHalfBytes, is_q || !is_v};
      },
      [=]() __attribute__((always_inline)) {
        if (!apart || part != -1) fill_angles<PATH>(&ka->r, pos, pos0, n, cs);      // (values do not turn: what is read of cs is not used)
      }, rows, n, lg, ka->r.dims, cs, stage);
  if ((nf >> 8) && ka->a.bounds && part == (apart ? -2 : -1)) {
    __syncthreads();                             // the page's last keys are written; the others were there
    uint8_t* b = ka->a.bounds + layer * ka->a.layer_bounds + (int64_t)(slot / kP) * Hkv * (2 * kRowBytes);
    for (int g = threadIdx.x >> 6; g < Hkv; g += 4) {
      PageKeys R;
      load_keys<false>(R, page + (int64_t)g * kSlab);
      write_bounds<E>(R, b + g * (2 * kRowBytes));
    }
  }
}
// Query rows of a batch are turned beside, in workgroups of their own.
// The workgroups behind the runs' copy a batch's lists to the workspace for the launches that follow, 16 bytes per thread.
__device__ __forceinline__ bool copy_lists(SYM_AS4 AppendKernelArgs* ka) {
  const int blk = (int)blockIdx.x - ka->a.n_runs;
  if (blk < 0) return false;
  const uint4* src = (const uint4*)ka->a.host_words;
  uint4* dst = (uint4*)ka->a.dev_words;
  const int64_t n16 = (ka->a.copy_words + 3) / 4;      // the staging buffer is padded to 16 bytes
  if (blockIdx.y == 0 && blockIdx.z == 0)
    for (int64_t i = (int64_t)blk * 256 + threadIdx.x; i < n16; i += (int64_t)(gridDim.x - ka->a.n_runs) * 256) dst[i] = src[i];
  return true;
}
template <typename E, int PATH>
__global__ __launch_bounds__(256) void append_rope_kernel(AppendKernelArgs) {
  __shared__ double2 cs[PATH == ROPE_NONE ? 1 : kRunTokens][kPairs];
  __shared__ __align__(16) uint8_t stage[PATH == ROPE_HALVES_ANY ? 32 : 1][kRowBytes];
  auto ka = (SYM_AS4 AppendKernelArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  if (copy_lists(ka)) return;
  const int32_t* w = ka->a.runs + (int64_t)blockIdx.x * RUN_WORDS;
  append_run<E, PATH>(ka, sload(w), sload(w + 1), sload(w + 2), sload(w + 3), blockIdx.y, (int)blockIdx.z - 1 - ka->a.apart, (int)gridDim.z - 1 - ka->a.apart, ka->a.apart, cs, stage);
}
template <typename E, int PATH>
__global__ __launch_bounds__(256) void append_rope_runs_kernel(AppendRunsKernelArgs) {
  __shared__ double2 cs[PATH == ROPE_NONE ? 1 : kRunTokens][kPairs];
  __shared__ __align__(16) uint8_t stage[PATH == ROPE_HALVES_ANY ? 32 : 1][kRowBytes];
  auto ka = (SYM_AS4 AppendRunsKernelArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  if (copy_lists(&ka->k)) return;
  const auto* w = ka->runs.w + blockIdx.x * RUN_WORDS;
  append_run<E, PATH>(&ka->k, w[0], w[1], w[2], w[3], blockIdx.y, (int)blockIdx.z - 1 - ka->k.a.apart, (int)gridDim.z - 1 - ka->k.a.apart, ka->k.a.apart, cs, stage);
}

// ---------------------------------------------------------------------------------------
// Bounds of a list of pages.  A workgroup of W wavefronts takes an equal share of the pages (at most 64, an id to each lane) in one layer; its
// wavefronts take the (page, kv head) in turn, the next one's keys under way while one is reduced.  W = 4, a page to a workgroup, for few
// pages, whose ids travel with the arguments; W = 8 for many, as many workgroups as compute units, whose list may stay in pinned
// host memory: a share is one request over the host link.  Bound: HBM (4 KiB read for 512 bytes written): 64 files of 512..4096
// tokens in 57 us, 297 MB at 5.2 TB/s (pieces of 4 KiB at a stride of 8 KiB are read at 6.0 to 6.6 TB/s when nothing is written).
// ---------------------------------------------------------------------------------------
struct BoundsKernelArgs {
  BoundsArgs a;
  int32_t ids[kArgPages];
};
template <typename E, bool ARGS, int W>
__global__ __launch_bounds__(64 * W) void bounds_kernel(std::conditional_t<ARGS, BoundsKernelArgs, BoundsArgs>) {
  auto ka = (SYM_AS4 BoundsKernelArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  const int first = (int)((int64_t)ka->a.n_pages * blockIdx.x / gridDim.x), end = (int)((int64_t)ka->a.n_pages * (blockIdx.x + 1) / gridDim.x);
  const int Hkv = ka->a.Hkv, n = (end - first) * Hkv, at = min(first + (int)(threadIdx.x & 63), end - 1);
  int ids;                                       // lane l: page l of the workgroup's
  if constexpr (ARGS) ids = ka->ids[at];
  else ids = ka->a.pages[at];
  const uint8_t* pool = ka->a.pool + blockIdx.y * ka->a.layer_bytes;
  uint8_t* bounds = ka->a.bounds + blockIdx.y * ka->a.layer_bounds;
  const int64_t page_bytes = ka->a.page_bytes;
  const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  auto page = [&](int u) __attribute__((always_inline)) { return (int64_t)__builtin_amdgcn_readlane(ids, u / Hkv); };
  if (w >= n) return;
  PageKeys A, B;
  load_keys<true>(A, pool + page(w) * page_bytes + (w % Hkv) * kSlab);
  for (int u = w; u < n; u += 2 * W) {
    const int v = u + W, x = v + W, vv = min(v, n - 1), xx = min(x, n - 1);      // (past the end: the last one again, not used)
    load_keys<true>(B, pool + page(vv) * page_bytes + (vv % Hkv) * kSlab);
    write_bounds<E>(A, bounds + (page(u) * Hkv + u % Hkv) * (2 * kRowBytes));
    if (v >= n) break;
    load_keys<true>(A, pool + page(xx) * page_bytes + (xx % Hkv) * kSlab);
    write_bounds<E>(B, bounds + (page(v) * Hkv + v % Hkv) * (2 * kRowBytes));
  }
}

// ---------------------------------------------------------------------------------------
// Choice of pages.  For a new token and kv head, page p scores  sum_d A_d hi_d + B_d lo_d  with A_d = sum_h max(q_hd, 0), B_d = sum_h min(q_hd, 0)
// over the G query heads of the kv head: what the sum of their logits with any key of the page does not exceed.  Products and sums in 64
// bits (the choice hangs on comparisons of scores that lie close together; with sums in 32 bits it would depend on their order),
// rounded to 32 at the end and written down as whole numbers of the same order.
// A wavefront takes one kv head and 32 pages; 32 lanes share a page's 512 bytes, a 16-byte chunk each, with the chunk's coefficients
// in registers; eight pages a lane are then added up over the 32 lanes by halving exchanges.  A wavefront's coefficients could serve
// more of a row's pages, but fewer wavefronts then hide less: 8 files of 32k..131k tokens, 8 heads, 41, 40, 45 and 44 us with 32, 64,
// 128 and 256 pages to a wavefront, one file 9, 12, 17 and 27.  Bound: between HBM (161 MB in 39.5 us, 4.1 TB/s) and the vector units (busy
// for 57 % of it: conversions and products in 64 bits).
// ---------------------------------------------------------------------------------------
constexpr int kScorePages = 32;                  // of a wavefront
__device__ __forceinline__ double as_f64(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return as_f64((uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, false), (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, false));
}

// A score as a whole number of the same order (NaN above all; never 0, which stands for none).
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = as_u32(x + 0.0f);           // -0 and 0 are equal
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// A wavefront's scores of 2 STEPS pages at a time, for one kv head of a token.
template <typename E, int STEPS = kScorePages / 2>
struct Scorer {
  static constexpr int C = E::kDimsPerChunk;
  double cf[C];                                  // coefficients of this lane's chunk: lanes 0..15 of a page hold lo, 16..31 hi
  int id[STEPS];                                 // pages 2 s + (upper half of the wavefront)

  __device__ __forceinline__ void coefficients(const SparseArgs& a, const int row, const int head) {
    const int hl = threadIdx.x & 31, part = hl >> 4, chunk = hl & 15, G = a.Hq / a.Hkv;
    const uint8_t* q = (const uint8_t*)a.q + ((int64_t)row * a.Hq + head * G) * kRowBytes + chunk * 16;
#pragma unroll
    for (int e = 0; e < C; ++e) cf[e] = 0.0;
    for (int h = 0; h < G; ++h) add(part, *(const uint4*)(q + h * kRowBytes));
  }
  // one query head's chunk
  __device__ __forceinline__ void add(const int part, const uint4& row) {
    float x[C];
    E::unpack(row, x);
#pragma unroll
    for (int e = 0; e < C; ++e) cf[e] += (double)(part ? (x[e] < 0.f ? 0.f : x[e]) : (x[e] > 0.f ? 0.f : x[e]));
  }
  __device__ __forceinline__ void ids(const int32_t* pt, const int p0, const int end) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) id[s] = pt[min(p0 + 2 * s + (int)((threadIdx.x & 63) >> 5), end - 1)];
  }
  // put(page, key) of the pages p0 .. of id, below end; next() runs when id has been used
  template <typename N, typename P>
  __device__ __forceinline__ void score(const SparseArgs& a, const int head, const int p0, const int end, const N& next, const P& put) {
    const int lane = threadIdx.x & 63, sub = lane >> 5, hl = lane & 31;
    const uint8_t* rec = a.bounds + head * (2 * kRowBytes) + hl * 16;
    const int64_t page_rec = (int64_t)a.Hkv * (2 * kRowBytes);
#pragma unroll
    for (int b = 0; b < STEPS / 8; ++b) {
      uint4 x[8];
#pragma unroll
      for (int s = 0; s < 8; ++s) x[s] = *(const uint4*)(rec + (int64_t)id[b * 8 + s] * page_rec);
      if (b == STEPS / 8 - 1) next();
      double v[8];
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        float f[C];
        E::unpack(x[s], f);
        v[s] = 0.0;
#pragma unroll
        for (int e = 0; e < C; ++e) v[s] = __builtin_fma(cf[e], (double)f[e], v[s]);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {              // lane bit 4: even rows of 16 lanes keep pages 0..3, odd ones 4..7
        const uint64_t p = __builtin_bit_cast(uint64_t, v[s]), q = __builtin_bit_cast(uint64_t, v[s + 4]);
        const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)p, (uint32_t)q, false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(p >> 32), (uint32_t)(q >> 32), false, false);
        v[s] = as_f64(lo[0], hi[0]) + as_f64(lo[1], hi[1]);
      }
      const bool b3 = (lane & 8) != 0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {              // lane bit 3
        const double keep = b3 ? v[s + 2] : v[s], send = b3 ? v[s] : v[s + 2];
        v[s] = keep + dpp_f64<0x128>(send);      // row_ror:8
        v[s] += dpp_f64<0xB1>(v[s]);             // the octet's sum
        v[s] += dpp_f64<0x4E>(v[s]);
        v[s] += dpp_f64<0x141>(v[s]);
      }
      // lane octet (bit 4, bit 3) holds steps 4 bit4 + 2 bit3 + {0, 1} of the eight
      const int step = b * 8 + ((lane >> 4) & 1) * 4 + ((lane >> 3) & 1) * 2 + (lane & 1), p = p0 + 2 * step + sub;
      if ((lane & 7) < 2 && p < end) put(p, order_of((float)((lane & 1) ? v[1] : v[0])));
    }
  }
};

template <typename E>
__global__ __launch_bounds__(256) void sparse_scores_kernel(SparseArgs a) {
  hold(a.scored, a.tables, a.bounds, a.q, a.scores, a.Hq, a.Hkv, a.first, a.score_stride);
  const int32_t* w = a.scored + (int64_t)(a.scored0 + blockIdx.y) * SPARSE_SCORED_WORDS;
  const int row = sload(w), tbl = sload(w + 1), end = sload(w + 2);
  const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int head = wave % a.Hkv, p0 = a.first + wave / a.Hkv * kScorePages;
  if (p0 >= end) return;
  uint32_t* scores = a.scores + ((int64_t)(row - a.row0) * a.Hkv + head) * a.score_stride;
  Scorer<E> sc;
  sc.ids(a.tables + tbl, p0, end);
  sc.coefficients(a, row, head);
  sc.score(a, head, p0, end, [] {}, [&](int p, uint32_t key) { scores[p - a.first] = key; });
}

// ---------------------------------------------------------------------------------------
// Append and scores of a small batch in one launch: single new tokens, few pages to score.  The first workgroups append as above; the
// others score 16 pages to a wavefront and turn the query rows for themselves, because those that the others write are not there yet.
// (The pages that the tokens complete are their rows' last ones, which nobody scores.)  What it saves is a launch's start and end: one
// file of 30000 tokens, 8 heads, 9.0 us instead of 4.1 and 8.7.  Bound: latency (arguments, lists, query rows, an angle, records).
// ---------------------------------------------------------------------------------------
struct FirstKernelArgs {
  AppendKernelArgs k;
  SparseArgs s;
  int32_t parts, append_blocks, row_blocks;        // workgroups of a run's query rows, of all runs, of a scored row
};
// Chunk `c` of a row, turned: its own 16 bytes and those that hold its pairs' other elements.
template <typename E, int PATH>
__device__ __forceinline__ uint4 turned_chunk(const uint4& own, const uint4& other, const int c, const int dims, const double2* cs) {
  constexpr int C = E::kDimsPerChunk;
  float a[C], b[C], y[C];
  E::unpack(own, a);
  E::unpack(other, b);
  u32x4_t r = __builtin_bit_cast(u32x4_t, own);
  if constexpr (PATH == ROPE_HALVES) {
    const int hr = dims / 2 / C;
    if (c >= 2 * hr) return own;
    const bool upper = c >= hr;
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const double2 t = cs[(upper ? c - hr : c) * C + e];
      y[e] = round_f32(upper ? (double)a[e] * t.x + (double)b[e] * t.y : (double)a[e] * t.x - (double)b[e] * t.y);
    }
    r = pack_chunk<E>(y);
  } else if constexpr (PATH == ROPE_INTERLEAVED) {
#pragma unroll
    for (int p = 0; p < C / 2; ++p) {
      const double2 t = cs[c * (C / 2) + p];
      y[2 * p] = round_f32((double)a[2 * p] * t.x - (double)a[2 * p + 1] * t.y);
      y[2 * p + 1] = round_f32((double)a[2 * p + 1] * t.x + (double)a[2 * p] * t.y);
    }
    const u32x4_t t = pack_chunk<E>(y);
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (c * C + w * (C / 4) < dims) r[w] = t[w];
  }
  return __builtin_bit_cast(uint4, r);
}
template <typename E, int PATH>
__global__ __launch_bounds__(256) void sparse_first_kernel(FirstKernelArgs) {
  constexpr int C = E::kDimsPerChunk;
  __shared__ double2 cs[1][kPairs];
  auto ka = (SYM_AS4 FirstKernelArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  if ((int)blockIdx.x < ka->append_blocks) {
    const int run = (int)blockIdx.x / (1 + ka->parts), part = (int)blockIdx.x % (1 + ka->parts) - 1;
    const int32_t* w = ka->k.a.runs + (int64_t)run * RUN_WORDS;
    append_run<E, PATH>(&ka->k, sload(w), sload(w + 1), sload(w + 2), sload(w + 3), 0, part, ka->parts, false, cs, nullptr);
    return;
  }
  const int blk = (int)blockIdx.x - ka->append_blocks, at_row = blk / ka->row_blocks, Hkv = ka->s.Hkv, first = ka->s.first;
  const int32_t* w = ka->s.scored + (int64_t)at_row * SPARSE_SCORED_WORDS;
  const int row = sload(w), tbl = sload(w + 1), end = sload(w + 2);
  const int wave = __builtin_amdgcn_readfirstlane(blk % ka->row_blocks * 4 + (int)(threadIdx.x >> 6));
  const int head = wave % Hkv, p0 = first + wave / Hkv * kFirstPages, G = ka->s.Hq / Hkv;
  const int chunk = threadIdx.x & 15, part = (threadIdx.x >> 4) & 1, hr = ka->k.r.dims / 2 / C;
  const int other = PATH == ROPE_HALVES ? (chunk < hr ? chunk + hr : chunk < 2 * hr ? chunk - hr : chunk) : chunk;
  SparseArgs a{};                                // (what score() reads of it)
  a.bounds = ka->s.bounds;
  a.Hkv = Hkv;
  Scorer<E, kFirstPages / 2> sc;
  sc.ids(ka->s.tables + tbl, min(p0, end - 1), end);
  const uint8_t* q = (const uint8_t*)ka->k.a.q + ((int64_t)row * ka->s.Hq + head * G) * kRowBytes;
  uint4 x[8], y[8];                                // (G <= 8)
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    x[h] = *(const uint4*)(q + min(h, G - 1) * kRowBytes + chunk * 16);
    if constexpr (PATH == ROPE_HALVES) y[h] = *(const uint4*)(q + min(h, G - 1) * kRowBytes + other * 16);
    else y[h] = x[h];
  }
  const int32_t* pos = ka->k.a.pos;
  const int at = pos ? pos[row] : sload(ka->s.rows + (int64_t)row * SPARSE_ROW_WORDS + 1) - 1;
  if ((int)threadIdx.x < ka->k.r.dims / 2) cs[0][threadIdx.x] = angle_of(&ka->k.r, at, threadIdx.x);
  __syncthreads();
  if (p0 >= end) return;
#pragma unroll
  for (int e = 0; e < C; ++e) sc.cf[e] = 0.0;
#pragma unroll
  for (int h = 0; h < 8; ++h)
    if (h < G) sc.add(part, turned_chunk<E, PATH>(x[h], y[h], chunk, ka->k.r.dims, cs[0]));
  uint32_t* scores = ka->s.scores + ((int64_t)row * Hkv + head) * ka->s.score_stride;
  sc.score(a, head, p0, end, [] {}, [&](int p, uint32_t key) { scores[p - first] = key; });
}

constexpr int kMostWaves = 8;                   // of a workgroup that attends
struct ChooseLds {
  __align__(16) uint32_t hist[kChoiceRounds][256];                // one for every round
  uint2 total[kMostWaves];                       // of every wavefront: greatest and least score, then how many are above and equal to the least chosen
};

// Sum over this lane and the higher ones of the wavefront: four DPP adds inside rows of 16 lanes, then the rows' totals.
__device__ __forceinline__ uint32_t suffix_sum(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x101, 0xf, 0xf, true);      // row_shl: 0 past the row's end
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x102, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x104, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x108, 0xf, 0xf, true);
  const uint32_t t1 = (uint32_t)__builtin_amdgcn_readlane((int)x, 16), t2 = (uint32_t)__builtin_amdgcn_readlane((int)x, 32), t3 = (uint32_t)__builtin_amdgcn_readlane((int)x, 48);
  const int row = (threadIdx.x & 63) >> 4;
  return x + (row < 1 ? t1 : 0) + (row < 2 ? t2 : 0) + (row < 3 ? t3 : 0);
}
// Sum over this lane and the lower ones.
__device__ __forceinline__ uint32_t prefix_sum(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true);      // row_shr
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true);
  const uint32_t t0 = (uint32_t)__builtin_amdgcn_readlane((int)x, 15), t1 = (uint32_t)__builtin_amdgcn_readlane((int)x, 31), t2 = (uint32_t)__builtin_amdgcn_readlane((int)x, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return x + (row > 0 ? t0 : 0) + (row > 1 ? t1 : 0) + (row > 2 ? t2 : 0);
}
// The greatest x of the wavefront, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));      // row_ror
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));
  return max(max((uint32_t)__builtin_amdgcn_readlane((int)x, 0), (uint32_t)__builtin_amdgcn_readlane((int)x, 16)),
             max((uint32_t)__builtin_amdgcn_readlane((int)x, 32), (uint32_t)__builtin_amdgcn_readlane((int)x, 48)));
}

// The `want` highest of the m scores (want < m), by the whole workgroup: put(i-th chosen, its index), in order of the index.
// The smallest chosen score is found in at most four rounds (ScoreRange): a histogram of 256 equal steps between the least and the greatest
// that it can be, and the step in which the wanted one lies.  Usually a step that is wanted whole ends it.  A thread holds EPT scores in a row, so that
// places are counted thread by thread; EPT = 0: any number of scores, sixteen at a time, read again for every round.
template <int W, int EPT, typename P>
__device__ __forceinline__ void pick_highest(const uint32_t* sc, const int m, const int want, ChooseLds& s, const P& put) {
  constexpr int NT = 64 * W, N = EPT > 0 ? EPT : 16;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int per = EPT > 0 ? EPT : (m + 16 * NT - 1) / (16 * NT) * 16, i0 = tid * per;
  uint32_t key[N];
  auto fetch = [&](int from) __attribute__((always_inline)) {      // scores from .. from + N - 1; 0 past the end
    if constexpr (EPT == 1) {
      key[0] = sc[min(from, m - 1)];
    } else {
#pragma unroll
      for (int v = 0; v < N / 4; ++v) {
        const uint4 k = *(const uint4*)(sc + min(from + 4 * v, (m - 1) & ~3));
        key[4 * v] = k.x;
        key[4 * v + 1] = k.y;
        key[4 * v + 2] = k.z;
        key[4 * v + 3] = k.w;
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) key[e] = from + e < m ? key[e] : 0u;
  };
  if constexpr (EPT > 0) fetch(i0);
  auto each = [&](auto f) __attribute__((always_inline)) {          // f(index, key)
    if constexpr (EPT > 0) {
#pragma unroll
      for (int e = 0; e < EPT; ++e) f(i0 + e, key[e]);
    } else {
      for (int x = 0; x < per; x += 16) {
        fetch(i0 + x);
#pragma unroll
        for (int e = 0; e < 16; ++e) f(i0 + x + e, key[e]);
      }
    }
  };
  for (int i = tid; i < kChoiceRounds * 256; i += NT) (&s.hist[0][0])[i] = 0;
  uint32_t hi = 0, top = 0;                      // top: the greatest ~key
  each([&](int, uint32_t k) {
    hi = max(hi, k);
    top = max(top, k ? ~k : 0u);
  });
  hi = wave_max(hi);
  top = wave_max(top);
  if (lane == 0) s.total[w] = make_uint2(hi, top);
  __syncthreads();
#pragma unroll
  for (int x = 0; x < W; ++x) {
    hi = max(hi, s.total[x].x);
    top = max(top, s.total[x].y);
  }
  ScoreRange r{(uint32_t)__builtin_amdgcn_readfirstlane(~top), (uint32_t)__builtin_amdgcn_readfirstlane(hi)};
  uint32_t need = (uint32_t)want, t = 0;         // chosen: above t, and the first `need` of those equal to it
#pragma unroll 1
  for (int round = 0; round < kChoiceRounds; ++round) {
    const int shift = r.shift();
    uint32_t* h = s.hist[round];
    each([&](int, uint32_t k) {
      if (r.holds(k)) atomicAdd(&h[r.step(k, shift)], 1u);      // (0, for none, is below every lo)
    });
    __syncthreads();
    // every wavefront for itself: lane l has steps 4 l .. 4 l + 3
    const uint4 c = *(const uint4*)(h + 4 * lane);
    const uint32_t own = c.x + c.y + c.z + c.w;
    const uint32_t sum = suffix_sum(own);
    const int at = 63 - __clzll((long long)__builtin_amdgcn_ballot_w64(sum >= need));      // the highest lane with enough from its steps on
    uint32_t above = (uint32_t)__builtin_amdgcn_readlane((int)(sum - own), at);
    const uint32_t cx = (uint32_t)__builtin_amdgcn_readlane((int)c.x, at), cy = (uint32_t)__builtin_amdgcn_readlane((int)c.y, at);
    const uint32_t cz = (uint32_t)__builtin_amdgcn_readlane((int)c.z, at), cw = (uint32_t)__builtin_amdgcn_readlane((int)c.w, at);
    uint32_t step = 4 * at + 3, count = cw;
    if (above + count < need) above += count, --step, count = cz;
    if (above + count < need) above += count, --step, count = cy;
    if (above + count < need) above += count, --step, count = cx;
    need -= above;
    r.narrow(step, shift);
    if (need == count) {                         // the whole step
      t = r.lo - 1;
      need = 0;
      break;
    }
    t = r.lo;
    if (shift == 0) break;                       // all of one value
  }
  // Place of a chosen one: those above t before it, and at most `need` of the equal ones before it.
  uint32_t gt = 0, eq = 0;
  each([&](int, uint32_t k) {
    gt += k > t ? 1 : 0;
    eq += k == t ? 1 : 0;
  });
  const uint32_t g_to = prefix_sum(gt), q_to = prefix_sum(eq);
  __syncthreads();                               // (s.total is read above)
  if (lane == 63) s.total[w] = make_uint2(g_to, q_to);
  __syncthreads();
  uint32_t g = g_to - gt, q = q_to - eq;
#pragma unroll
  for (int x = 0; x < W; ++x) {
    g += x < w ? s.total[x].x : 0;
    q += x < w ? s.total[x].y : 0;
  }
  each([&](int i, uint32_t k) {
    if (k < t || k == 0) return;
    if (k > t || q < need) put((int)(g + min(q, need)), i);
    g += k > t ? 1 : 0;
    q += k == t ? 1 : 0;
  });
}

// ---------------------------------------------------------------------------------------
// Attention over the chosen pages of a (new token, kv head): a workgroup of W wavefronts to each of `splits` equal parts of their list.
// Every workgroup chooses from the row's scores for itself and keeps its part of the list in LDS, where it reads like a
// file's page table: only the last page may be partly filled.  One pass over the pages, with the running maximum and sum of the softmax in
// fp32; the wavefronts' results are combined through LDS.  The workgroup that finishes last of a row's parts joins them, so that no
// launch follows.  STREAM: nontemporal loads, where no two rows read the same pages (64 files 62.4 -> 59.3 us a call); where they do (several
// tokens of a file, forks) the next row finds them in a cache (chunks 72 us, with nontemporal loads 95).
// Bound: HBM (8 KiB for 4 D 16 G flops): 64 files of 512..4096 tokens, 1024 tokens read of each, in 53 us, 306 MB at 5.8 TB/s, the scoring
// of bounds with it; 138 rows of 8 files in 66 us, 440 MB of which the caches serve the most.  One row of one file is latency: 14 us, of
// which the choice 3.8, pages 1.9, combining 2.1, handing over 2.4.
// ---------------------------------------------------------------------------------------
// What workgroups of one launch hand to each other goes past the caches that they do not share, in both directions, and a workgroup
// counts itself done when its stores have arrived.  (A release fence instead writes back everything in the L2: with one from every
// wavefront the choice among 5000 pages took 470 us instead of 40.)
__device__ __forceinline__ void hand_over(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float take(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// Whether this workgroup is the last of `all` to come; every thread calls it, behind its stores.  The counter is 0 again for the next launch.
__device__ __forceinline__ bool comes_last(int32_t* counter, const int all, int& shared) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    shared = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == all - 1;
    if (shared) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return shared;
}

// bf16 storage: on the matrix cores, an fp32 weight cut into three bf16 numbers (8 bits each: exact), as in decode_bins_mx.  Where 3 G columns fit
// into 16 each takes a column of one product.  With 8 heads per kv head there are two products to the same sums: the upper part halved in columns 0..7
// of both (0 there would make an infinite V NaN), the middle and the lower part in columns 8..15.  (Weights cut to 16 bits in one
// product: error against 64 bits 4.8e-6 instead of 2e-7.)
template <int G, bool STREAM>
struct AttendMx {
  typedef ElemBF16 Elem;
  static constexpr int D = 128;
  static constexpr bool TWICE = G == 8;
  bf16x8_t q[4];
  f32x4_t O[8];
  float m, l;
  int col, grp, part;
  uint32_t cut1, cut2;
  float scale;

  __device__ __forceinline__ void start(const uint8_t* qrows, float scale_log2e) {
    const int lane = threadIdx.x & 63;
    col = lane & 15;
    grp = lane >> 4;
    part = col / G;
    cut1 = part >= 1 ? 0xffff0000u : 0u;
    cut2 = part >= 2 ? 0xffff0000u : 0u;
    scale = scale_log2e;
    const uint8_t* qp = qrows + (col % G) * kRowBytes + grp * 16;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) q[ks] = __builtin_bit_cast(bf16x8_t, *(const u32x4_t*)(qp + ks * 64));
    m = -1e30f;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) O[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // (a lane's place in a page hangs on nothing that start() sets: the first page is requested before it)
  __device__ __forceinline__ void request(PageRegs& R, const uint8_t* slab) const {
    const int col = threadIdx.x & 15, grp = (threadIdx.x & 63) >> 4;
    const uint8_t* kb = slab + col * kHalfBytes + grp * 16;
    const uint8_t* vb = slab + kBlk + (col >> 3) * (kP * kHalfBytes) + (4 * grp) * kHalfBytes + (col & 7) * 16;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) R.k[ks] = ld16<STREAM>(kb + (ks >> 1) * (kP * kHalfBytes) + (ks & 1) * 64);
#pragma unroll
    for (int u = 0; u < 4; ++u) R.v[u] = ld16<STREAM>(vb + u * kHalfBytes);
  }
  __device__ __forceinline__ void page(PageRegs& R, const int nvalid) {
    f32x4_t S = {0.f, 0.f, 0.f, 0.f}, S2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      S = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, R.k[ks]), q[ks], S, 0, 0, 0);
      S2 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, R.k[2 + ks]), q[2 + ks], S2, 0, 0, 0);
    }
    S = S + S2;
    if (nvalid < kP) {                           // slots past the file's end hold anything; weight 0, but 0 * NaN is NaN
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (4 * grp + u >= nvalid) {
          S[u] = -__builtin_inff();
          R.v[u] = make_uint4(0, 0, 0, 0);
        }
    }
    const float mx = fmaxf(fmaxf(S[0], S[1]), fmaxf(S[2], S[3])) * scale;
    if (__builtin_amdgcn_ballot_w64(mx > m + kTau) != 0) {
      const float mn = pair32_max(pair16_max(fmaxf(m, mx)));
      const float al = __builtin_amdgcn_exp2f(m - mn);
      l *= al;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int v = 0; v < 4; ++v) O[e][v] *= al;
      m = mn;
    }
    uint32_t w[4], w2[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      float x = __builtin_amdgcn_exp2f(__builtin_fmaf(S[v], scale, -m));
      l += x;
      if constexpr (TWICE) {
        const float up = as_f32(as_u32(x) & 0xffff0000u), mid = x - up;
        w[v] = as_u32(part ? mid : 0.5f * up);
        w2[v] = as_u32(part ? mid - as_f32(as_u32(mid) & 0xffff0000u) : 0.5f * up);
      } else {
        x -= as_f32(as_u32(x) & cut1);
        x -= as_f32(as_u32(x) & cut2);
        w[v] = as_u32(x);
      }
    }
    auto upper = [](const uint32_t* x) __attribute__((always_inline)) {
      return __builtin_bit_cast(s16x4_t, make_uint2(__builtin_amdgcn_perm(x[1], x[0], 0x07060302), __builtin_amdgcn_perm(x[3], x[2], 0x07060302)));
    };
    const s16x4_t W = upper(w), W2 = TWICE ? upper(w2) : W;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t sel = (e & 1) ? 0x07060302 : 0x05040100;
      auto word = [&](int u) { return (e >> 1) == 0 ? R.v[u].x : (e >> 1) == 1 ? R.v[u].y : (e >> 1) == 2 ? R.v[u].z : R.v[u].w; };
      const s16x4_t vt = __builtin_bit_cast(s16x4_t, make_uint2(__builtin_amdgcn_perm(word(1), word(0), sel), __builtin_amdgcn_perm(word(3), word(2), sel)));
      O[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, W, O[e], 0, 0, 0);
      if constexpr (TWICE) O[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, W2, O[e], 0, 0, 0);
    }
  }
  // this wavefront's unnormalised result, [G][D] and (max, sum) per head
  __device__ __forceinline__ void finish(float* acc, float* ml) {
    const float ls = pair32_sum(pair16_sum(l));
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float low = row_shl<G>(O[e][v]);
        if constexpr (!TWICE) low += row_shl<2 * G>(O[e][v]);
        O[e][v] += low == low ? low : 0.f;       // (an infinite V at a lower part of 0: the upper part says what it makes of the output)
      }
    if (col < G) {
      float* o = acc + col * D + 32 * grp;       // + 8 v + e
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        *(float4*)(o + 8 * v) = make_float4(O[0][v], O[1][v], O[2][v], O[3][v]);
        *(float4*)(o + 8 * v + 4) = make_float4(O[4][v], O[5][v], O[6][v], O[7][v]);
      }
      if (grp == 0) *(float2*)(ml + 2 * col) = make_float2(m, ls);
    }
  }
};

// fp32 storage: on the vector units, lane (r, j) holds tokens r and 8 + r of a page and 8 dims; running maximum and sum are each lane's own.
template <int G, bool STREAM>
struct AttendF32 {
  typedef ElemF32 Elem;
  static constexpr int C = 4, DPL = 8, D = 64;
  uint4 q[G][2];
  float m[G], l[G], acc[G][DPL];
  int r, j;
  float scale;

  __device__ __forceinline__ void start(const uint8_t* qrows, float scale_log2e) {
    const int lane = threadIdx.x & 63;
    r = lane >> 3;
    j = lane & 7;
    scale = scale_log2e;
#pragma unroll
    for (int h = 0; h < G; ++h) {
      q[h][0] = *(const uint4*)(qrows + h * kRowBytes + j * 16);
      q[h][1] = *(const uint4*)(qrows + h * kRowBytes + kHalfBytes + j * 16);
      m[h] = -1e30f;
      l[h] = 0.f;
#pragma unroll
      for (int d = 0; d < DPL; ++d) acc[h][d] = 0.f;
    }
  }
  __device__ __forceinline__ void request(PageRegs& R, const uint8_t* slab) const {
    const uint8_t* b = slab + (threadIdx.x & 63) * 16;
#pragma unroll
    for (int x = 0; x < 4; ++x) R.k[x] = ld16<STREAM>(b + x * 1024);
#pragma unroll
    for (int x = 0; x < 4; ++x) R.v[x] = ld16<STREAM>(b + kBlk + x * 1024);
  }
  __device__ __forceinline__ void page(PageRegs& R, const int nvalid) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
      if (hf * 8 + r >= nvalid) {
        R.v[hf] = make_uint4(0, 0, 0, 0);
        R.v[2 + hf] = make_uint4(0, 0, 0, 0);
      }
    float s[2][G];
    bool need = false;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int h = 0; h < G; ++h) {
        float x = ElemF32::dot(R.k[2 + hf], q[h][1], ElemF32::dot(R.k[hf], q[h][0], 0.f));
        x = octet_sum(x) * scale;
        s[hf][h] = hf * 8 + r < nvalid ? x : -__builtin_inff();
      }
#pragma unroll
    for (int h = 0; h < G; ++h) need |= fmaxf(s[0][h], s[1][h]) > m[h] + kTau;
    if (__builtin_amdgcn_ballot_w64(need) != 0) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
        const float mn = fmaxf(m[h], fmaxf(s[0][h], s[1][h])), al = __builtin_amdgcn_exp2f(m[h] - mn);
        l[h] *= al;
#pragma unroll
        for (int d = 0; d < DPL; ++d) acc[h][d] *= al;
        m[h] = mn;
      }
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      float w[G];
#pragma unroll
      for (int h = 0; h < G; ++h) {
        w[h] = __builtin_amdgcn_exp2f(s[hf][h] - m[h]);
        l[h] += w[h];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float v[C];
        ElemF32::unpack(R.v[i * 2 + hf], v);
#pragma unroll
        for (int h = 0; h < G; ++h)
#pragma unroll
          for (int e = 0; e < C; ++e) acc[h][i * C + e] = __builtin_fmaf(w[h], v[e], acc[h][i * C + e]);
      }
    }
  }
  __device__ __forceinline__ void finish(float* out, float* ml) {
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const float M = pair32_max(pair16_max(fmaxf(m[h], row_xor8(m[h]))));
      const float f = __builtin_amdgcn_exp2f(m[h] - M);
      float ls = l[h] * f;
      ls = pair32_sum(pair16_sum(ls + row_xor8(ls)));
      // the eight token slots of a chunk: halving exchanges over lane bits 5, 4, 3 leave lane r with entry r
      float x[DPL];
#pragma unroll
      for (int d = 0; d < DPL; ++d) x[d] = acc[h][d] * f;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const auto sw = __builtin_amdgcn_permlane32_swap(as_u32(x[d]), as_u32(x[d + 4]), false, false);
        x[d] = as_f32(sw[0]) + as_f32(sw[1]);
      }
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const auto sw = __builtin_amdgcn_permlane16_swap(as_u32(x[d]), as_u32(x[d + 2]), false, false);
        x[d] = as_f32(sw[0]) + as_f32(sw[1]);
      }
      const bool b3 = (r & 1) != 0;
      const float keep = b3 ? x[1] : x[0], send = b3 ? x[0] : x[1];
      out[h * D + (r / C) * (D / 2) + j * C + r % C] = keep + row_xor8(send);
      if ((threadIdx.x & 63) == 0) *(float2*)(ml + 2 * h) = make_float2(M, ls);
    }
  }
};

// SCORES: the workgroup scores the row's pages itself, where they are few.
template <typename AT, int G, bool SCORES, int W>
__global__ __launch_bounds__(64 * W, 8 / W) void sparse_attend_kernel(SparseArgs a) {
  constexpr int D = AT::D, NT = 64 * W;
  // the choice's counts, then the wavefronts' results
  constexpr int kResult = W * G * D * 4;
  __shared__ __align__(16) uint8_t s_mem[kResult > (int)sizeof(ChooseLds) ? kResult : (int)sizeof(ChooseLds)];
  __shared__ __align__(16) float s_ml[W][2 * G];
  __shared__ int32_t s_list[kPartPages];
  __shared__ int s_last;
  __shared__ __align__(16) uint32_t s_keys[SCORES ? kOwnScores : 4];
  hold(a.rows, a.tables, a.scores, a.pool, a.page_bytes, a.q, a.out, a.picked, a.Hq, a.Hkv, a.budget, a.first, a.last, a.splits);
  const int unit = (int)blockIdx.x / a.splits, split = (int)blockIdx.x - unit * a.splits;
  const int row = a.row0 + unit / a.Hkv, head = unit % a.Hkv;
  const int32_t* rw = a.rows + (int64_t)row * SPARSE_ROW_WORDS;
  const int32_t* pt = a.tables + sload(rw);
  const int vis = sload(rw + 1), n = (vis + kP - 1) / kP, kept = min(n, a.budget);
  const int tail = (vis - 1) % kP + 1;           // tokens of the last page
  const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  AT at;
  at.start((const uint8_t*)a.q + ((int64_t)row * a.Hq + head * G) * kRowBytes, a.scale_log2e);
  // this workgroup's part of the list
  const int lo = (int)((int64_t)kept * split / a.splits), hi = (int)((int64_t)kept * (split + 1) / a.splits);
  int32_t* picked = a.picked ? a.picked + ((int64_t)row * a.Hkv + head) * a.budget : nullptr;
  auto put = [&](int i, int p) __attribute__((always_inline)) {
    if (i < lo || i >= hi) return;
    s_list[i - lo] = pt[p];
    if (picked) picked[i] = p;
  };
  if (n <= a.budget) {
    for (int i = lo + threadIdx.x; i < hi; i += NT) put(i, i);
    if (picked && split == 0)
      for (int i = n + threadIdx.x; i < a.budget; i += NT) picked[i] = -1;
  } else {
    for (int i = threadIdx.x; i < a.first + a.last; i += NT) {
      if (i < a.first) put(i, i);
      else put(kept - a.last + i - a.first, n - a.last + i - a.first);
    }
    const int m = n - a.first - a.last, want = kept - a.first - a.last;
    // places that the choice fills: a page of the pool in each until then (the choice has barriers before it fills them)
    for (int i = max(lo, a.first) + threadIdx.x; i < min(hi, kept - a.last); i += NT) s_list[i - lo] = 0;
    auto chosen = [&](int i, int p) __attribute__((always_inline)) { put(a.first + i, a.first + p); };
    ChooseLds& s = *(ChooseLds*)s_mem;
    const uint32_t* sc = a.scores + (int64_t)unit * a.score_stride;
    if constexpr (SCORES) {
      if (want > 0) {
        int p0 = a.first + wv * kScorePages;
        const int end = n - a.last;
        Scorer<typename AT::Elem> own;
        if (p0 < end) {
          own.ids(pt, p0, end);
          own.coefficients(a, row, head);
        }
        for (; p0 < end; p0 += W * kScorePages)
          own.score(a, head, p0, end, [&] { own.ids(pt, p0 + W * kScorePages, end); }, [&](int p, uint32_t key) { s_keys[p - a.first] = key; });
        __syncthreads();
        if (m <= NT) pick_highest<W, 1>(s_keys, m, want, s, chosen);
        else pick_highest<W, kOwnScores / NT < 4 ? 4 : kOwnScores / NT>(s_keys, m, want, s, chosen);
      }
    } else if (want == 0) {
    } else if (m <= NT) {
      pick_highest<W, 1>(sc, m, want, s, chosen);
    } else if (m <= 4 * NT) {
      pick_highest<W, 4>(sc, m, want, s, chosen);
    } else if (m <= 8 * NT) {
      pick_highest<W, 8>(sc, m, want, s, chosen);
    } else if (m <= 16 * NT) {
      pick_highest<W, 16>(sc, m, want, s, chosen);
    } else if (m <= 32 * NT) {
      pick_highest<W, 32>(sc, m, want, s, chosen);
    } else {
      pick_highest<W, 0>(sc, m, want, s, chosen);
    }
  }
  if (lo >= hi && threadIdx.x == 0) s_list[0] = pt[0];      // a part without pages (a short file among long ones)
  __syncthreads();
  int p = lo + (int)((int64_t)(hi - lo) * wv / W);
  const int pe = lo + (int)((int64_t)(hi - lo) * (wv + 1) / W);
  const uint8_t* pool = a.pool + (int64_t)head * kSlab;
  PageRegs A, B;
  // (past the wavefront's pages, and without any: another page, read and not used)
  auto id = [&](int i) __attribute__((always_inline)) { return (int64_t)__builtin_amdgcn_readfirstlane(s_list[max(min(i, hi - 1) - lo, 0)]); };
  at.request(A, pool + id(p) * a.page_bytes);
  while (p < pe) {
    at.request(B, pool + id(p + 1) * a.page_bytes);
    at.page(A, p == kept - 1 ? tail : kP);
    if (++p >= pe) break;
    at.request(A, pool + id(p + 1) * a.page_bytes);
    at.page(B, p == kept - 1 ? tail : kP);
    ++p;
  }
  float (*s_acc)[G * D] = (float (*)[G * D])s_mem;
  at.finish(s_acc[wv], s_ml[wv]);
  __syncthreads();
  float* out = a.out + ((int64_t)row * a.Hq + head * G) * D;
  const int64_t slot = (int64_t)unit * a.splits + split;
  for (int x = threadIdx.x; x < G * D; x += NT) {
    const int h = x / D;
    float M = s_ml[0][2 * h], num = 0.f, den = 0.f;
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, s_ml[w][2 * h]);
#pragma unroll
    for (int w = 0; w < W; ++w) {     // (a wavefront without pages: maximum -1e30, sum 0, zeros)
      const float f = __builtin_amdgcn_exp2f(s_ml[w][2 * h] - M);
      num = __builtin_fmaf(s_acc[w][x], f, num);
      den = __builtin_fmaf(s_ml[w][2 * h + 1], f, den);
    }
    if (a.splits == 1) {
      out[x] = num / den;
    } else {
      hand_over(a.part_acc + slot * G * D + x, num);
      if (x % D == 0) {
        hand_over(a.part_ml + (slot * G + h) * 2, M);
        hand_over(a.part_ml + (slot * G + h) * 2 + 1, den);
      }
    }
  }
  if (a.splits == 1 || !comes_last(a.counters + unit, a.splits, s_last)) return;
  const int64_t first = (int64_t)unit * a.splits;
  for (int x = threadIdx.x; x < G * D; x += NT) {      // the parts in their order, whoever came last
    const int h = x / D;
    float M = -1e30f, num = 0.f, den = 0.f;
    for (int i0 = 0; i0 < a.splits; i0 += 8) {         // eight parts' loads in flight
      float2 ml[8];
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int64_t i = first + min(i0 + u, a.splits - 1);
        ml[u] = make_float2(take(a.part_ml + (i * G + h) * 2), take(a.part_ml + (i * G + h) * 2 + 1));
        v[u] = take(a.part_acc + i * G * D + x);
      }
      float mn = M;
#pragma unroll
      for (int u = 0; u < 8; ++u) mn = fmaxf(mn, ml[u].x);
      const float f0 = __builtin_amdgcn_exp2f(M - mn);
      num *= f0;
      den *= f0;
      M = mn;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float f = i0 + u < a.splits ? __builtin_amdgcn_exp2f(ml[u].x - M) : 0.f;
        num = __builtin_fmaf(i0 + u < a.splits ? v[u] : 0.f, f, num);      // (0 * Inf is NaN)
        den = __builtin_fmaf(ml[u].y, f, den);
      }
    }
    out[x] = num / den;
  }
}

}  // namespace

// The element type and the way of turning, as template arguments.
#define SYM_ROPE_CASES(LAUNCH) \
  if (dtype == 0) { \
    switch (r.path) { \
      case ROPE_NONE: LAUNCH(ElemF32, ROPE_NONE); break; \
      case ROPE_HALVES: LAUNCH(ElemF32, ROPE_HALVES); break; \
      case ROPE_HALVES_ANY: LAUNCH(ElemF32, ROPE_HALVES_ANY); break; \
      case ROPE_INTERLEAVED: LAUNCH(ElemF32, ROPE_INTERLEAVED); break; \
      default: return hipErrorInvalidValue; \
    } \
  } else { \
    switch (r.path) { \
      case ROPE_NONE: LAUNCH(ElemBF16, ROPE_NONE); break; \
      case ROPE_HALVES: LAUNCH(ElemBF16, ROPE_HALVES); break; \
      case ROPE_HALVES_ANY: LAUNCH(ElemBF16, ROPE_HALVES_ANY); break; \
      case ROPE_INTERLEAVED: LAUNCH(ElemBF16, ROPE_INTERLEAVED); break; \
      default: return hipErrorInvalidValue; \
    } \
  }

hipError_t launch_rope_rows(RopeRowsArgs a, const RopeTable& r, int dtype, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  if (a.n > kMostRopeRows) return hipErrorInvalidValue;
  // enough rows for every compute unit: 1024 bf16 rows of 32 + 8 heads 7.0 us a call (7.8 with one token), 2048 10.4 (12.5), 16384 65 (75)
  a.tokens = a.n >= 1024 ? 4 : 1;
  const RopeRowsKernelArgs ka{a, r};
  const dim3 grid((unsigned)((a.n + a.tokens - 1) / a.tokens)), block(256);
#define SYM_LAUNCH(E, PATH) hipLaunchKernelGGL((rope_rows_kernel<E, PATH>), grid, block, 0, st, ka)
  SYM_ROPE_CASES(SYM_LAUNCH)
#undef SYM_LAUNCH
  return hipGetLastError();
}

hipError_t launch_append_rope(AppendRopeArgs a, const RopeTable& r, int dtype, hipStream_t st) {
  if (a.n_runs <= 0) return a.done ? hipEventRecord(a.done, st) : hipSuccess;
  if (a.n_layers < 1 || a.n_layers > 65535) return hipErrorInvalidValue;
  const int64_t copy = std::min<int64_t>((a.copy_words / 4 + 255) / 256 + (a.copy_words > 0), 256);
  // the query rows of a run in parts of about four passes of a workgroup (8 files of up to 33 new tokens 72.5 us a pred; one part to a run 75.3)
  const int parts = a.q ? std::min(std::max(a.Hq * std::min(a.run_tokens, kRunTokens) / 128, 1), std::min(a.Hq, 16)) : 0;
  // keys and values of long runs apart: values need not wait for angles (8000 tokens of a file 16.9 us a call, 17.8 in one; 8 files of 2..33 tokens
  // 70.6 and 71.9; 2 tokens of 8 files 29.5 and 28.8, one of 64 files 62.1 and 61.6)
  a.apart = a.run_tokens > 8;
  const dim3 grid((unsigned)(a.n_runs + copy), (unsigned)a.n_layers, (unsigned)(1 + a.apart + parts)), block(256);
  if (a.by_args) {
    if (a.n_runs > kArgRuns) return hipErrorInvalidValue;
    AppendRunsKernelArgs ka;
    ka.k = AppendKernelArgs{a, r};
    std::copy_n(a.runs, a.n_runs * RUN_WORDS, ka.runs.w);
    std::fill(ka.runs.w + a.n_runs * RUN_WORDS, ka.runs.w + kArgRuns * RUN_WORDS, 0);
    hipError_t e = hipSuccess;
#define SYM_LAUNCH(E, PATH) e = launch_done(append_rope_runs_kernel<E, PATH>, grid, block, st, a.done, ka)
    SYM_ROPE_CASES(SYM_LAUNCH)
#undef SYM_LAUNCH
    return e;
  }
  const AppendKernelArgs ka{a, r};
  hipError_t e = hipSuccess;
#define SYM_LAUNCH(E, PATH) e = launch_done(append_rope_kernel<E, PATH>, grid, block, st, a.done, ka)
  SYM_ROPE_CASES(SYM_LAUNCH)
#undef SYM_LAUNCH
  return e;
}

hipError_t launch_bounds(const BoundsArgs& a, int dtype, hipStream_t st) {
  if (a.n_pages <= 0) return hipSuccess;
  if (a.n_layers < 1 || a.n_layers > 65535) return hipErrorInvalidValue;
  if (a.by_args) {
    if (a.n_pages > kArgPages) return hipErrorInvalidValue;
    BoundsKernelArgs ka;
    ka.a = a;
    std::copy_n(a.pages, a.n_pages, ka.ids);
    std::fill(ka.ids + a.n_pages, ka.ids + kArgPages, 0);
    const dim3 grid((unsigned)a.n_pages, (unsigned)a.n_layers);
    if (dtype == 0) return launch_done(bounds_kernel<ElemF32, true, 4>, grid, dim3(256), st, a.done, ka);
    return launch_done(bounds_kernel<ElemBF16, true, 4>, grid, dim3(256), st, a.done, ka);
  }
  // a workgroup to a compute unit: files of 10000, 20000, 120000 tokens of 8 heads 7.3, 10.8, 53.2 us a call, with four 8.0, 11.9, 54.9;
  // 64 files of 512..4096 tokens 58.7 and 60.0 (71 with half as many, 68 with 320)
  const int blocks = std::min(a.n_pages, std::max(std::max(256 / a.n_layers, 1), (a.n_pages + 63) / 64));
  const dim3 grid((unsigned)blocks, (unsigned)a.n_layers);
  if (dtype == 0) return launch_done(bounds_kernel<ElemF32, false, 8>, grid, dim3(512), st, a.done, a);
  return launch_done(bounds_kernel<ElemBF16, false, 8>, grid, dim3(512), st, a.done, a);
}

hipError_t launch_sparse_first(const AppendRopeArgs& a, const RopeTable& r, const SparseArgs& s, int dtype, hipStream_t st) {
  FirstKernelArgs ka{{a, r}, s, std::max(a.Hq / 128, 1), 0, 0};
  ka.append_blocks = a.n_runs * (1 + ka.parts);
  ka.row_blocks = ((s.most_scored + kFirstPages - 1) / kFirstPages * s.Hkv + 3) / 4;
  const dim3 grid((unsigned)(ka.append_blocks + ka.row_blocks * s.n_scored)), block(256);
#define SYM_LAUNCH(E) \
  if (r.path == ROPE_HALVES) hipLaunchKernelGGL((sparse_first_kernel<E, ROPE_HALVES>), grid, block, 0, st, ka); \
  else hipLaunchKernelGGL((sparse_first_kernel<E, ROPE_INTERLEAVED>), grid, block, 0, st, ka)
  if (dtype == 0) {
    SYM_LAUNCH(ElemF32);
  } else {
    SYM_LAUNCH(ElemBF16);
  }
#undef SYM_LAUNCH
  return hipGetLastError();
}

hipError_t launch_sparse_scores(const SparseArgs& a, int dtype, hipStream_t st) {
  if (a.n_scored <= 0) return hipSuccess;
  const int64_t waves = (int64_t)((a.most_scored + kScorePages - 1) / kScorePages) * a.Hkv;
  if (a.n_scored > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((waves + 3) / 4), (unsigned)a.n_scored), block(256);
  if (dtype == 0) hipLaunchKernelGGL((sparse_scores_kernel<ElemF32>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((sparse_scores_kernel<ElemBF16>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_sparse_attend(const SparseArgs& a, int dtype, hipStream_t st) {
  if (a.n_rows <= 0) return hipSuccess;
  const dim3 grid((unsigned)(a.n_rows * a.Hkv * a.splits)), block(64 * a.waves);
#define SYM_ATTEND_ROWS(AT, GG, STREAM) \
  if (a.own) hipLaunchKernelGGL((sparse_attend_kernel<AT<GG, STREAM>, GG, true, 4>), grid, block, 0, st, a); \
  else if (a.waves == 4) hipLaunchKernelGGL((sparse_attend_kernel<AT<GG, STREAM>, GG, false, 4>), grid, block, 0, st, a); \
  else hipLaunchKernelGGL((sparse_attend_kernel<AT<GG, STREAM>, GG, false, 8>), grid, block, 0, st, a)
#define SYM_ATTEND(GG) \
  case GG: \
    if (dtype == 0) { \
      if (a.stream) SYM_ATTEND_ROWS(AttendF32, GG, true); \
      else SYM_ATTEND_ROWS(AttendF32, GG, false); \
    } else { \
      if (a.stream) SYM_ATTEND_ROWS(AttendMx, GG, true); \
      else SYM_ATTEND_ROWS(AttendMx, GG, false); \
    } \
    break;
  switch (a.Hq / a.Hkv) {
    SYM_ATTEND(1) SYM_ATTEND(2) SYM_ATTEND(4) SYM_ATTEND(8)
    default: return hipErrorInvalidValue;
  }
#undef SYM_ATTEND
#undef SYM_ATTEND_ROWS
  return hipGetLastError();
}

int enter_device(int device) {
  int cur = device;
  if (hipGetDevice(&cur) != hipSuccess || cur == device) return -1;
  return hipSetDevice(device) == hipSuccess ? cur : -1;
}
void leave_device(int before) {
  if (before >= 0) (void)hipSetDevice(before);
}

bool stream_captures(hipStream_t st) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(st, &cs) != hipSuccess) {
    (void)hipGetLastError();
    return true;
  }
  return cs != hipStreamCaptureStatusNone;
}

}  // namespace symkv
