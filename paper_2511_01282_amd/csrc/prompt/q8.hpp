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

// Eight values (two words of codes) as bf16, which holds them exactly under bytes 3 to 246: below, steps of 2^(byte - 136) are
// smaller than bf16's least, 2^-133, and above, large codes reach 2^128, an infinity.  `scale`: the float 2^(byte - 127), of which
// the instruction takes the exponent.
__device__ __forceinline__ u32x4 q8_bf16(u32x2 codes, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.x, scale, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes.y, scale, true))};
}

// Values of any size.  A sum over rows, of values times weights of up to 2^8, may leave float32 where the mean is well inside
// it.  Rows that a pass over the cache leaves at kLarge or above, or not finite, are not stored but taken again in a second pass
// with V's scales kUnit powers of two lower (but byte 0 at least: 2^-54 of a value's error, beside sums of 2^114), which no sum leaves float32
// with, and put right where they are stored.  Partial results stay below kLarge, so that 64 of them join
// without leaving float32.  The second pass is code of its own behind the first and reads its arguments anew: with what both
// start from kept in registers, 32 query rows of 128 columns took 8% more; like this 18 calls take -5 to +1.5% of what they took.
constexpr float kLarge = 1.329227996e36f;  // 2^120
constexpr int kUnit = 64;
// Sum of sizes: at kLarge or above where one is, NaN where one is.
template <typename V>
__device__ __forceinline__ void add_sizes(float& sum, const V& v) {
#pragma unroll
  for (int e = 0; e < (int)(sizeof(V) / 4); ++e) sum += fabsf(v[e]);
}
__device__ __forceinline__ int lane_id() { return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)); }

// What the second pass starts from, the kernel's arguments and a wave's number, read anew: nothing else is kept in registers for it.
struct Again {
  const ChunkAttnArgs& a;
  int x, wave;
};
__device__ __forceinline__ Again again_from(int x, int wave) {
  uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();  // (the kernel's one argument)
  asm volatile("" : "+s"(p), "+s"(x), "+s"(wave));
  return Again{*(const ChunkAttnArgs*)(const __attribute__((address_space(4))) ChunkAttnArgs*)p, x, wave};
}

// A split's reference maximum and sum beside values in units of 2^unit: o 2^unit 2^m is o 2^(m + unit), so the sum counts 2^-unit as
// much; what the reference's rounding leaves out goes into both (`to_o`: factor of o).
__device__ __forceinline__ void move_unit(int unit, float& m, float& l, float& to_o) {
#pragma clang fp contract(off)
  const float u = (float)unit, to = m + u, b = to - m, rest = (m - (to - b)) + (u - b);
  to_o = __builtin_amdgcn_exp2f(rest);
  l = __builtin_amdgcn_ldexpf(l * to_o, -unit);
  m = to;
}

}  // namespace respec
