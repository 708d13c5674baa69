// Rotary positions of queries and keys.
//
// A row of a head at position p: pair i of its columns, (x_a, x_b), is turned by the angle p w_i and stretched by the
// amplitude.  Every row is read and written once, and memory bounds it if the angles cost little:
//
// Angles.  w_i is held in turns per position, as a 64-bit fraction; p w_i mod 1 turn is then the low word of an integer
// product, within 2^-31 at any position, where a float's product would be off by p 2^-24.  Its upper 32 bits split into a quadrant and
// a rest of at most an eighth of a turn either way, whose sine and cosine are Taylor's polynomials up to x^9 and x^10 (what is
// left out is below 2^-25).
//
// A unit of work is 32 bytes of a row that hold 16 / (bytes per element) whole pairs: two 16-byte pieces, rotary_dim / 2
// columns apart (half) or side by side (interleaved).  A thread takes one unit's place in up to R heads of one token, so the
// angles are taken once for R units, while the loads of these are under way.
//
// 8192 tokens of 32 + 8 heads of 128, bf16 (168 MB): 34 to 37 us, 4.5 to 4.9 TB/s, as a large copy; the vector instructions stand
// behind it.  65 nodes of 28 + 4 heads: 4.1 us, which is a launch.  Float32, 4096 tokens of 16 + 16 heads of 64 (67 MB): 13.5 us a call.
// Lengths, not positions: a token's workgroup walks over the batch, 1024 sequences of a token each 11 us a call, 4096 35, 16384 205.
#include "cache.hpp"

namespace respec {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Sine and cosine of `phase` 2^-32 turns.
__device__ __forceinline__ void sincos_turns(uint32_t phase, float& s, float& c) {
  const uint32_t quadrant = (phase + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(phase - (quadrant << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float y = x * x;
  const float sn = x * __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
  const float cs = __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float a = quadrant & 1 ? cs : sn, b = quadrant & 1 ? sn : cs;
  s = quadrant & 2 ? -a : a;
  c = (quadrant + 1) & 2 ? -b : b;
}

template <int ES>
__device__ __forceinline__ float element(const u32x4& p, int i) {
  if constexpr (ES == 4) return __uint_as_float(p[i]);
  return __uint_as_float(i & 1 ? p[i / 2] & 0xFFFF0000u : p[i / 2] << 16);
}
template <int ES>
__device__ __forceinline__ void put_pair(u32x4& p, int i, float lo, float hi) {  // elements i (even) and i + 1
  if constexpr (ES == 4) {
    p[i] = __float_as_uint(lo);
    p[i + 1] = __float_as_uint(hi);
  } else {
    p[i / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
  }
}

// Status of a batch's sequences (64-bit sums: nothing of the device's words wraps).
__device__ __forceinline__ void rotary_status(const ChunkBatch& c, int wg) {
  const int b = wg * kRotaryThreads + (int)threadIdx.x;
  if (b < c.batch) c.status[b] = chunk_seq(c, b).status;
}

template <int ES, int D, bool HALF, int R>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
  constexpr int U = D * ES / 32;     // units of a head
  constexpr int P = 16 / ES;         // pairs of a unit, elements of a piece
  if ((int)blockIdx.x < a.status_wgs) {
    if (blockIdx.y == 0) rotary_status(a.b, blockIdx.x);
    return;
  }
  const int t0 = ((int)blockIdx.x - a.status_wgs) * a.tok_per_wg;
  const int slots = (int)a.stride.d * U;  // threads of a token
  int slot = (int)threadIdx.x + (int)blockIdx.y * kRotaryThreads, i = 0;
  if (a.tok_per_wg > 1) {
    i = (int)div_by((uint32_t)slot / U, a.stride);
    slot -= i * slots;
  }
  const int t = t0 + i, unit = slot % U, j = slot / U;
  const bool mine = i < a.tok_per_wg && t < a.tokens && j < (int)a.stride.d;
  const bool turned = unit < a.turned;
  // bytes of the unit's two pieces within a row
  int lo, hi;
  if (turned && HALF) {
    lo = unit * 16;
    hi = lo + a.turned * 16;
  } else {
    lo = unit * 32;
    hi = lo + 16;
  }
  u32x4 x[R][2];
  bool there[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int head = j + r * (int)a.stride.d;
    there[r] = mine && head < a.heads;
    if (there[r]) {
      const bool of_q = head < a.q_heads;
      const RotaryRows& z = of_q ? a.q : a.k;
      const char* p = z.x + (int64_t)t * z.x_tok + (int64_t)(of_q ? head : head - a.q_heads) * z.x_head;
      x[r][0] = ld16(p + lo);
      x[r][1] = ld16(p + hi);
    }
  }
  int pos = -1;
  if (a.positions) {
    if (mine) pos = a.positions[t];
  } else {
    __shared__ int32_t at[kRotaryThreads];
    for (int k = threadIdx.x >> 6; k < a.tok_per_wg; k += kRotaryThreads / 64) {
      int b;
      const ChunkSeq s = seq_of_token(a.b, t0 + k, b);  // (past the last token: none)
      if ((threadIdx.x & 63) == 0) at[k] = s.n > 0 ? s.L + (t0 + k - s.t0) : -1;
    }
    __syncthreads();
    if (mine) pos = at[i];
  }
  if (pos < 0) return;
  if (turned) {
    float sn[P], cs[P];
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const uint64_t turns = (uint64_t)(uint32_t)pos * a.turns[unit * P + e] + 0x80000000u;
      sincos_turns((uint32_t)(turns >> 32), sn[e], cs[e]);
      sn[e] *= a.amplitude;
      cs[e] *= a.amplitude;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!there[r]) continue;
      u32x4 y[2];
      if constexpr (HALF) {
#pragma unroll
        for (int e = 0; e < P; e += 2) {
          float u[2], v[2];
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const float xa = element<ES>(x[r][0], e + w), xb = element<ES>(x[r][1], e + w);
            u[w] = xa * cs[e + w] - xb * sn[e + w];
            v[w] = xb * cs[e + w] + xa * sn[e + w];
          }
          put_pair<ES>(y[0], e, u[0], u[1]);
          put_pair<ES>(y[1], e, v[0], v[1]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const int piece = 2 * e / P, at = 2 * e % P;
          const float xa = element<ES>(x[r][piece], at), xb = element<ES>(x[r][piece], at + 1);
          put_pair<ES>(y[piece], at, xa * cs[e] - xb * sn[e], xb * cs[e] + xa * sn[e]);
        }
      }
      x[r][0] = y[0];
      x[r][1] = y[1];
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (!there[r]) continue;
    const int head = j + r * (int)a.stride.d;
    const bool of_q = head < a.q_heads;
    const RotaryRows& z = of_q ? a.q : a.k;
    char* p = z.y + (int64_t)t * z.y_tok + (int64_t)(of_q ? head : head - a.q_heads) * z.y_head;
    *reinterpret_cast<u32x4*>(p + lo) = x[r][0];
    *reinterpret_cast<u32x4*>(p + hi) = x[r][1];
  }
}

template <int ES, int D>
hipError_t go(bool half, int r, dim3 grid, const RotaryArgs& a, hipStream_t s) {
  if (half && r == 1) hipLaunchKernelGGL((rotary_kernel<ES, D, true, 1>), grid, dim3(kRotaryThreads), 0, s, a);
  else if (half) hipLaunchKernelGGL((rotary_kernel<ES, D, true, 4>), grid, dim3(kRotaryThreads), 0, s, a);
  else if (r == 1) hipLaunchKernelGGL((rotary_kernel<ES, D, false, 1>), grid, dim3(kRotaryThreads), 0, s, a);
  else hipLaunchKernelGGL((rotary_kernel<ES, D, false, 4>), grid, dim3(kRotaryThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(int es, int head_dim, bool half, int heads_per_thread, int wgs, int wgs_of_token, const RotaryArgs& a,
                         hipStream_t s) {
  const dim3 grid(wgs, wgs_of_token);
  if (es == 2) return head_dim == 128 ? go<2, 128>(half, heads_per_thread, grid, a, s) : go<2, 64>(half, heads_per_thread, grid, a, s);
  return head_dim == 128 ? go<4, 128>(half, heads_per_thread, grid, a, s) : go<4, 64>(half, heads_per_thread, grid, a, s);
}

}  // namespace respec
