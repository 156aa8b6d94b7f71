// 8-bit codes of cache blocks (16 tokens of one layer and kv-head, K or V): encoding a
// bf16 tile, decoding to bf16. See pced_cache8 in pced.h for the definition.
//
// A tile of codes keeps the bf16 tile's order (kswz, vswz): a lane's 16-byte units 2j and
// 2j + 1 of the bf16 tile are the two halves of its unit j of codes, so that both operands of
// the attention's products come from 16-byte loads of one wave-contiguous KiB.
#pragma once
#include "pced_device.h"

namespace pced {
namespace {

constexpr int kE4m3 = 1, kInt8 = 2;  // pced_code

// Codes of a tile that a wave holds as NU units per lane. *scale: the block's scale as bf16 bits,
//   s = clamp(max |x|, 2^-100, 2^127) / M rounded up to bf16,  code = x (1 / s) to the nearest, within +-M.
// Rounded up, so that no code is cut off by more than an fp32 rounding; two bytes, whose relative
// step of 2^-7 costs no precision: a value is its code times exactly this scale. The limits keep
// 1 / s and codes times s within fp32. NaN counts as 0.
template <int CODE, int NU>
__device__ __forceinline__ void encode_tile(const u32x4 (&u)[NU], u32x4 (&c)[NU / 2], uint32_t* scale) {
  constexpr float M = CODE == kE4m3 ? 448.f : 127.f;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(bf2f(el16(u[i], e))));  // (NaN: the other one)
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  top = fminf(fmaxf(top, 0x1p-100f), 0x1p127f);
  const uint32_t sb = (__float_as_uint(top / M) + 0xFFFFu) >> 16;
  const float inv = 1.f / bf2f(sb);
  *scale = sb;
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = bf2f(el16(u[i], e)), z = fminf(fmaxf(x * inv, -M), M);
      y[e] = x == x ? z : 0.f;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint32_t r = 0;
      if constexpr (CODE == kE4m3) {
        r = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], (int)r, false);
        r = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], (int)r, true);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r |= ((uint32_t)(int)rintf(y[4 * w + e]) & 0xFFu) << (8 * e);
      }
      c[i >> 1][2 * (i & 1) + w] = r;
    }
  }
}

// Four codes as four bf16 (exactly: at most 8 significant bits)
template <int CODE>
__device__ __forceinline__ uint2 decode4(uint32_t w) {
  bf16x2 lo, hi;
  if constexpr (CODE == kE4m3) {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true);
  } else {
    lo = bf16x2{(__bf16)(float)(int8_t)w, (__bf16)(float)(int8_t)(w >> 8)};
    hi = bf16x2{(__bf16)(float)(int8_t)(w >> 16), (__bf16)(float)(int8_t)(w >> 24)};
  }
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

}  // namespace
}  // namespace pced
