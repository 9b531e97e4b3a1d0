// What the kernels share: the page geometry, loads of descriptor words, cross-lane steps, element types, launches that complete an event.
//
// Geometry shared by all kernels (also stated in include/symphony_kv.h): a K or V row of
// one token and one kv head is 256 bytes; a (page, kv head) slab is [K|V][row half 0|1]
// [16 tokens][128 bytes], 8 KiB, so 8 tokens of one row half are 1 KiB contiguous.
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <cstdint>

namespace symkv {

namespace {

constexpr int kP = 16;              // tokens per page
constexpr int kRowBytes = 256;      // bytes of one K or V row (one token, one kv head)
constexpr int kHalfBytes = 128;     // a row half
constexpr int kBlk = kP * kRowBytes;   // 4096: K (or V) of one (page, head)
constexpr int kSlab = 2 * kBlk;        // 8192: K+V of one (page, head)
constexpr int kWavesPerBlock = 4;
constexpr float kTau = 8.0f;        // the running max may lag the true max by up to 2^kTau

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float as_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __builtin_bit_cast(uint32_t, f); }

// One word of the batch descriptor at a wavefront-uniform address, through the scalar cache.  The constant address space says
// what the compiler cannot see: nothing writes the descriptor while a kernel runs.  Without it these loads are vector loads as
// soon as the kernel stores anything, and since vector loads return in order, waiting for a page id then meant waiting for every
// K/V load in flight (s_waitcnt vmcnt(0) once per page; whole calls without / with: long contexts, 8 heads per kv head 754 / 716
// us; one file of 2000 tokens x 32 layers 494 / 473; drafts of 4 on 64 files 136.4 / 134.4; the mixed batch 1845 / 1824).
typedef const __attribute__((address_space(4))) int32_t* const_word_t;
__device__ __forceinline__ int sload(const int32_t* ptr) { return __builtin_amdgcn_readfirstlane(*(const_word_t)(uintptr_t)ptr); }

// Kernel arguments that a start needs, all requested before the first of them is waited for.  Left to itself the compiler fetches
// each where it is used, and a start is then a chain of up to six misses of the scalar cache before the first K/V load.
template <typename... T>
__device__ __forceinline__ void hold(const T&... x) {
  (..., [](auto v) __attribute__((always_inline)) { asm volatile("" ::"s"(v)); }(x));
}

// Sum over the 8 lanes of a lane octet (lanes 8k .. 8k+7): three DPP adds.
__device__ __forceinline__ float octet_sum(float x) {
  x += as_f32(__builtin_amdgcn_update_dpp(0, as_u32(x), 0xB1, 0xf, 0xf, false));    // quad_perm [1,0,3,2]
  x += as_f32(__builtin_amdgcn_update_dpp(0, as_u32(x), 0x4E, 0xf, 0xf, false));    // quad_perm [2,3,0,1]
  x += as_f32(__builtin_amdgcn_update_dpp(0, as_u32(x), 0x141, 0xf, 0xf, false));   // row_half_mirror
  return x;
}

// Value of the lane 8 away inside the 16-lane row (lane ^ 8): DPP row rotate by 8.
__device__ __forceinline__ float row_xor8(float x) {
  return as_f32(__builtin_amdgcn_update_dpp(0, as_u32(x), 0x128, 0xf, 0xf, false));   // row_ror:8
}

// max / sum of x over the lane pairs (l, l ^ 32) and (l, l ^ 16), in every lane, with the lane-swap instructions: swapping
// the upper 32 lanes of x with the lower 32 of a copy leaves one register holding the lower half twice and the other the
// upper half twice (likewise the odd and even rows of 16 lanes), so combining the two needs no select.
__device__ __forceinline__ float pair32_max(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(as_u32(x), as_u32(x), false, false);
  return fmaxf(as_f32(sw[0]), as_f32(sw[1]));
}
__device__ __forceinline__ float pair16_max(float x) {
  const auto sw = __builtin_amdgcn_permlane16_swap(as_u32(x), as_u32(x), false, false);
  return fmaxf(as_f32(sw[0]), as_f32(sw[1]));
}
__device__ __forceinline__ float pair32_sum(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(as_u32(x), as_u32(x), false, false);
  return as_f32(sw[0]) + as_f32(sw[1]);
}
__device__ __forceinline__ float pair16_sum(float x) {
  const auto sw = __builtin_amdgcn_permlane16_swap(as_u32(x), as_u32(x), false, false);
  return as_f32(sw[0]) + as_f32(sw[1]);
}

// Element-type traits.  A lane holds, per row half, one 16-byte chunk of a K/V row.
struct ElemBF16 {
  static constexpr int kDimsPerChunk = 8;
  // dot of one 16-byte chunk of K with the matching chunk of q, accumulated into s
  static __device__ __forceinline__ float dot(const uint4& k, const uint4& q, float s) {
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, k.x), __builtin_bit_cast(bf16x2_t, q.x), s, false);
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, k.y), __builtin_bit_cast(bf16x2_t, q.y), s, false);
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, k.z), __builtin_bit_cast(bf16x2_t, q.z), s, false);
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, k.w), __builtin_bit_cast(bf16x2_t, q.w), s, false);
    return s;
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
    f[0] = as_f32(v.x << 16); f[1] = as_f32(v.x & 0xffff0000u);
    f[2] = as_f32(v.y << 16); f[3] = as_f32(v.y & 0xffff0000u);
    f[4] = as_f32(v.z << 16); f[5] = as_f32(v.z & 0xffff0000u);
    f[6] = as_f32(v.w << 16); f[7] = as_f32(v.w & 0xffff0000u);
  }
};
struct ElemF32 {
  static constexpr int kDimsPerChunk = 4;
  static __device__ __forceinline__ float dot(const uint4& k, const uint4& q, float s) {
    s = __builtin_fmaf(as_f32(k.x), as_f32(q.x), s);
    s = __builtin_fmaf(as_f32(k.y), as_f32(q.y), s);
    s = __builtin_fmaf(as_f32(k.z), as_f32(q.z), s);
    s = __builtin_fmaf(as_f32(k.w), as_f32(q.w), s);
    return s;
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
    f[0] = as_f32(v.x); f[1] = as_f32(v.y); f[2] = as_f32(v.z); f[3] = as_f32(v.w);
  }
};

// 16 bytes of K or V.  STREAM: nontemporal, which streams a batch larger than the caches fastest; a compute unit that reads
// with few others gets its lines sooner without it.
template <bool STREAM>
__device__ __forceinline__ uint4 ld16(const uint8_t* p) {
  if constexpr (STREAM) return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4_t*)p));
  else return *(const uint4*)p;
}

struct PageRegs {
  uint4 k[4];   // index = row_half * 2 + token_half
  uint4 v[4];
};

// Operands of the matrix instructions.
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

template <int N>
__device__ __forceinline__ float row_shl(float x) {     // value of the lane N further up in the 16-lane row (0 past its end)
  return as_f32(__builtin_amdgcn_update_dpp(0, as_u32(x), 0x100 + N, 0xf, 0xf, true));
}

// A launch that completes the event `done` (or none).  The event hangs on the dispatch itself: recorded behind the launch it is a
// packet of its own, which the next kernel waits for, 3.0 us in every call whatever its size (two kernels of 10 us with an event
// recorded between them 25.4 us, with it attached and without a system fence 22.4, with no event at all 22.4; as a record without a
// system fence 23.6).  A stream that is being captured takes it as a record: a graph's kernel nodes carry no events.
template <typename K, typename... A>
hipError_t launch_done(K kernel, dim3 grid, dim3 block, hipStream_t st, hipEvent_t done, const A&... a) {
  if (done) {
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &cs) != hipSuccess) {
      (void)hipGetLastError();
      cs = hipStreamCaptureStatusActive;
    }
    if (cs == hipStreamCaptureStatusNone) {
      hipExtLaunchKernelGGL(kernel, grid, block, 0, st, nullptr, done, 0, a...);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL(kernel, grid, block, 0, st, a...);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && done ? hipEventRecord(done, st) : e;
}

}  // namespace

}  // namespace symkv
