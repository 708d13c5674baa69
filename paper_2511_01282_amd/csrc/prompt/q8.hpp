// A cache of e4m3 values with a power-of-two scale for each block of rows: where its scales lie, and what its values are.
#pragma once

#include "chunk.hpp"

namespace respec {

typedef float q8_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 q8_bf16x2 __attribute__((ext_vector_type(2)));

// Offset of row r's scale byte, in the page of id `id` (out of range: page 0's, as offset_in) and KV head g.
__device__ __forceinline__ int64_t scale_offset(const ChunkBatch& c, const Q8Scales& q8, int32_t id, uint32_t r, int g) {
  const int64_t page = (uint32_t)id < (uint32_t)c.n_pages ? id : 0;
  return page * q8.page_stride + (int64_t)g * q8.head_stride + (int64_t)((r - div_by(r, c.page) * c.page.d) >> q8.shift);
}
__device__ __forceinline__ int64_t scale_offset(const ChunkAttnArgs& a, int32_t id, uint32_t r, int g) {
  return scale_offset(a.b, a.q8, id, r, g);
}

// Four values as float32: exact, but for what float32 itself cannot hold.
__device__ __forceinline__ u32x4 q8_floats(uint32_t codes, uint32_t byte) {
  const q8_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  const int e = (int)byte - 127;
  return u32x4{__float_as_uint(__builtin_amdgcn_ldexpf(lo.x, e)), __float_as_uint(__builtin_amdgcn_ldexpf(lo.y, e)),
               __float_as_uint(__builtin_amdgcn_ldexpf(hi.x, e)), __float_as_uint(__builtin_amdgcn_ldexpf(hi.y, e))};
}

// Eight values (two words of codes) as bf16, which holds them exactly; `scale`: the float 2^(byte - 127), of which the
// instruction takes the exponent.
__device__ __forceinline__ u32x4 q8_bf16(u32x2 codes, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, true))};
}

}  // namespace respec
