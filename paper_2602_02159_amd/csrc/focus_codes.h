// e4m3 rows with one power of two each, in registers: what the kernels that write and read such rows share.
#pragma once

#include "focus_attn.h"
#include "focus_common.h"

namespace focus {

constexpr int kExpMin = 127 - 110, kExpMax = 127 + 119;  // as stored

__device__ __forceinline__ float exp_value(uint32_t byte) { return __uint_as_float(byte << 23); }  // 2^(byte - 127), 0 for 0

// A value of a row as its code takes it; `inv` = 2^-E.  The limit matters for rows whose E is at its upper end only; infinities and NaN
// take the NaN code.
__device__ __forceinline__ float scaled_for_code(float v, float inv) {
  const float y = fminf(fmaxf(v * inv, -448.f), 448.f);
  return fabsf(v) < INFINITY ? y : __builtin_nanf("");
}
__device__ __forceinline__ uint32_t decode2(uint32_t codes, bool high, float scale) {  // two of the four codes as a bf16 pair, times 2^E
  return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
}
__device__ __forceinline__ uint4 decode8(const uint2& c, float scale) {
  return make_uint4(decode2(c.x, false, scale), decode2(c.x, true, scale), decode2(c.y, false, scale), decode2(c.y, true, scale));
}

// STREAM: rows that one workgroup alone reads pass the caches by (load_stream16)
template <bool STREAM, class V>
__device__ __forceinline__ V load_row_piece(const uint8_t* p) {
  return STREAM ? __builtin_nontemporal_load(reinterpret_cast<const V*>(p)) : *reinterpret_cast<const V*>(p);
}
template <int D, bool STREAM>
__device__ __forceinline__ void load_codes(uint32_t (&v)[D / 64], const uint8_t* p) {
  if constexpr (D == 128) {
    const uintx2 w = load_row_piece<STREAM, uintx2>(p);
    v[0] = w.x;
    v[1] = w.y;
  } else {
    v[0] = load_row_piece<STREAM, uint32_t>(p);
  }
}
template <bool STREAM>
__device__ __forceinline__ uint4 load_codes16(const uint8_t* p) {
  return __builtin_bit_cast(uint4, load_row_piece<STREAM, uintx4>(p));
}

}  // namespace focus
