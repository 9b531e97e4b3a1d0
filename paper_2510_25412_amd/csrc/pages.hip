// Page copies: forked and reordered files' last pages, pages that leave a range of the pool.
#include "beam.hpp"
#include "device.hpp"

namespace symkv {

namespace {

template <int N>
struct CopyList {
  int32_t word[3 * N];
};

// The filled slots of pages, bit for bit.  A page is 4 * Hkv pieces (kv head, K or V, row half) of 16 slots of 128 bytes; the first r
// slots of a piece lie together, so the 16-byte chunks of a copy are counted through, r * 8 to a piece.  Sources and destinations are
// different pages.  Bound: HBM, read + write.  Half of a server's pool (9837 pages, 2 layers, 1.29 GB read, as much written) 409..422 us = 6.1..6.3 TB/s,
// with two chunks to a thread, past the caches both ways (plain stores 438, plain loads 425, four chunks 420..437, eight 445..468).
// Few copies are of last pages, which several forks take: plain loads (239 copies x 8 layers, a call 24.2 us; 26.0 past the caches).
// The grid is a full page's whatever the slots, and of a copy of few slots most workgroups start, read the list and leave: 240 copies x 8 layers x 8
// heads of 1, 4, 8, 15 slots take 13, 26, 26, 36 us (8, 31, 63, 118 MB written); with a grid for the longest copy of the list 3.6, 8.8, 20, 36. The
// calls that copy so are the host's time (next to which this is not seen).
constexpr int kCopyChunks = 2;         // chunks of a thread
template <bool PAST>
__device__ __forceinline__ u32x4_t load16(const uint8_t* p) {
  if constexpr (PAST) return __builtin_nontemporal_load((const u32x4_t*)p);
  else return *(const u32x4_t*)p;
}
template <bool BY_ARGS, int N>
__global__ __launch_bounds__(256) void copy_kernel(CopyArgs a, CopyList<N> l) {
  const int e = 3 * (int)blockIdx.y;
  int src, dst, what;
  if constexpr (BY_ARGS) {
    src = l.word[e], dst = l.word[e + 1], what = l.word[e + 2];
  } else {
    src = sload(a.list + e), dst = sload(a.list + e + 1), what = sload(a.list + e + 2);
  }
  const uint32_t per = (uint32_t)(what & 0xff) * 8, total = per * (uint32_t)a.Hkv * 4;      // chunks of a piece, of the copy
  uint8_t* pool = a.pool + (int64_t)blockIdx.z * a.layer_bytes;
  const uint8_t* s = pool + (int64_t)src * a.page_bytes;
  uint8_t* d = pool + (int64_t)dst * a.page_bytes;
  const uint32_t first = blockIdx.x * (256 * kCopyChunks) + threadIdx.x;
  if (blockIdx.x * (256 * kCopyChunks) < total) {
    const float inv = 1.0f / (float)per;
    u32x4_t v[kCopyChunks];
    uint32_t at[kCopyChunks];
#pragma unroll
    for (int u = 0; u < kCopyChunks; ++u) {
      const uint32_t i = min(first + u * 256, total - 1);
      // i / per: with a half added, no quotient of an i below 2^21 is within its roundings of a whole number
      const uint32_t piece = (uint32_t)(((float)i + 0.5f) * inv);
      at[u] = (i + piece * (kP * 8 - per)) * 16;
      v[u] = load16<!BY_ARGS>(s + at[u]);
    }
#pragma unroll
    for (int u = 0; u < kCopyChunks; ++u)
      if (first + u * 256 < total) __builtin_nontemporal_store(v[u], (u32x4_t*)(d + at[u]));
  }
  if (blockIdx.x == 0 && (what >> 8) && a.bounds) {
    uint8_t* b = a.bounds + (int64_t)blockIdx.z * a.layer_bounds;
    const int64_t n = (int64_t)a.Hkv * 512;
    for (int64_t i = threadIdx.x * 16; i < n; i += 256 * 16) *(u32x4_t*)(b + dst * n + i) = *(const u32x4_t*)(b + src * n + i);
  }
}

}  // namespace

template <int N>
static hipError_t launch_listed(const CopyArgs& a, dim3 grid, hipStream_t st) {
  CopyList<N> l = {};
  std::copy(a.list, a.list + 3 * a.n_copies, l.word);
  return launch_done(copy_kernel<true, N>, grid, dim3(256), st, a.done, a, l);
}

hipError_t launch_copies(const CopyArgs& a, hipStream_t st) {
  if (a.n_copies <= 0) return hipSuccess;
  if (a.page_bytes / 16 > (1 << 21) || (a.by_args && a.n_copies > kArgCopies)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((a.page_bytes / 16 + 256 * kCopyChunks - 1) / (256 * kCopyChunks)), (unsigned)a.n_copies, (unsigned)a.n_layers);
  if (a.by_args) return a.n_copies <= 32 ? launch_listed<32>(a, grid, st) : launch_listed<kArgCopies>(a, grid, st);
  return launch_done(copy_kernel<false, 1>, grid, dim3(256), st, a.done, a, CopyList<1>{});
}

}  // namespace symkv
