// Helpers that the gfx950 kernels share: vector types, bf16 conversions, streaming
// loads, and the launch with optional timing events.
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "pced_internal.h"

namespace pced {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));  // at any float's address

constexpr float kNegInf = -INFINITY;

__device__ __forceinline__ float bf2f(uint32_t b) { return __uint_as_float(b << 16); }

// round-to-nearest-even float -> bf16 bits (finite inputs)
__device__ __forceinline__ uint32_t f2bf(float f) {
  uint32_t u = __float_as_uint(f);
  u += 0x7FFFu + ((u >> 16) & 1u);
  return u >> 16;
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 16-byte load of data a launch reads once (KV pages, LM-head and projection
// weights in a decode step): with STREAM it carries the non-temporal hint and
// streams through the caches without displacing what is reused (partial
// states, outputs, q and x rows). Launches that read the same bytes several
// times (the prefill's row groups and virtual rows, the LM head's row groups)
// use plain loads, so that the repeats hit the caches.
template <bool STREAM>
__device__ __forceinline__ uint4 ld_w(const uint4* p) {
  if constexpr (STREAM) {
    const u32x4 v = __builtin_nontemporal_load((const u32x4*)p);
    return make_uint4(v.x, v.y, v.z, v.w);
  } else {
    return *p;
  }
}

// element e (of 8) of a 16-byte row piece
__device__ __forceinline__ uint32_t el16(const u32x4& v, int e) { return (v[e >> 1] >> (16 * (e & 1))) & 0xFFFFu; }

// Run r of a bf16 V tile (see k_load): kv-head, token quad and first dim
struct RunPos {
  int g, q, d0;
};
__device__ __forceinline__ RunPos run_pos(int run, int D) {
  const int rpt = D / 4, r = run % rpt;
  return RunPos{run / rpt, (r >> 1) & 3, 32 * (r >> 3) + 8 * (r & 1)};
}

// This wave's LDS accesses so far are complete and ordered before the next ones
// (other lanes' data is read next).
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Launch; timing events, when given, are attached to the dispatch itself
// (start when the kernel begins, stop when it completes), so they measure the
// kernel and not the queue around it.
template <typename Kern, typename... Args>
hipError_t go(Kern kernel, dim3 grid, dim3 block, size_t shm, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1,
              Args... args) {
  if (ev0 || ev1) hipExtLaunchKernelGGL(kernel, grid, block, (uint32_t)shm, st, ev0, ev1, 0u, args...);
  else hipLaunchKernelGGL(kernel, grid, block, shm, st, args...);
  return hipGetLastError();
}
hipEvent_t t0(const Timing* tm) { return tm ? tm->start : nullptr; }
hipEvent_t t1(const Timing* tm) { return tm ? tm->stop : nullptr; }

}  // namespace
}  // namespace pced
