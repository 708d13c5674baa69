// Log probability and rank of a given token, entropy and top alternatives, per row of logits.
//
//   m = max z, S = sum e^(z-m), T = sum e^(z-m) (z-m)
//   lse = m + log S, H = log S - T/S, log p(t) = (z_t - m) - log S
//   rank(t) = #{u : z_u > z_t} + #{u < t : z_u = z_t}
//
// One pass over the row.  A thread keeps the largest logit so far, S and T against it, the count for the rank, the
// 16-byte vector that held its largest logit first, and the largest of its other vectors.  (A reference maximum that
// is raised only now and then would save rescalings, but not here: T against a reference 16 below the maximum loses
// 4 bits of the entropy when it is moved.)  The top alternatives need little bookkeeping in the pass: the K-th largest
// of the threads' maxima, H, is at most the K-th largest logit, so every one of the top K is in a vector of one of the
// few threads whose maximum reaches H.  They have the vector with that maximum at hand; only where the largest of a
// thread's others reaches H, too, are its vectors read again (those of all of these threads: 20% more bytes, as eight
// threads share a line, 118 against 114 us).
//
// Memory bounds it, with the vector instructions close behind: 2048 rows of 128256 bf16 logits (526 MB), 108 to 110 us a call
// among others, 4.8 TB/s (bounds checked in every step, not in the last alone: 114), 109 to 121 in a profiler's trace; 65
// rows of 152064 float32 logits (40 MB, in parts), 15 us and 4 us to join them.  The rank counted by the scalar unit off the compare masks, and bf16's best
// vector read again instead of kept: 121 against 114 us.
//
// Keys: (value, id) pairs as 64-bit integers (common.hpp), all distinct, so ties go to the lowest id.
#include <type_traits>

#include "topk.hpp"
#include "prompt.hpp"

namespace respec {
namespace {

constexpr int kThreads = kScoreThreads, kWaves = kThreads / 64;
constexpr int kUnroll = 4;         // vectors of a thread per step
constexpr int kMaxKeys = kScoreMaxKeys;  // keys that reach H and are sorted (more: by repeated passes)
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp_f(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Statistics of a set of logits: the largest one, and S and T against reference ref (-inf: none finite yet).
struct Stats {
  float top, ref, S, T;
  int cnt;
};

// The same with the sums against a larger maximum.  (A difference below -200, beside which e is 0, counts as -200: a
// masked vocabulary's lowest values times S would be an infinity, and 0 times that a NaN.)
__device__ __forceinline__ void rebase(Stats& s, float to) {
  const bool none = s.ref == kNegInf;
  const float d = none ? 0.f : s.ref - to, e = none ? 1.f : exp_f(d);
  s.T = e * (s.T + fmaxf(d, -200.f) * s.S);
  s.S *= e;
  s.ref = to;
}

// Sum over a wave's lanes (moves inside rows of 16 lanes and row swaps: common.hpp).
__device__ __forceinline__ void wave_stats(Stats& s) {
  s.top = fmaxf(s.top, xchg<0>(s.top));
  s.top = fmaxf(s.top, xchg<1>(s.top));
  s.top = fmaxf(s.top, xchg<2>(s.top));
  s.top = fmaxf(s.top, xchg<3>(s.top));
  s.top = fmaxf(s.top, xchg<4>(s.top));
  s.top = fmaxf(s.top, xchg<5>(s.top));
  rebase(s, s.top);
  s.S += xchg<0>(s.S); s.T += xchg<0>(s.T); s.cnt += xchg<0>(s.cnt);
  s.S += xchg<1>(s.S); s.T += xchg<1>(s.T); s.cnt += xchg<1>(s.cnt);
  s.S += xchg<2>(s.S); s.T += xchg<2>(s.T); s.cnt += xchg<2>(s.cnt);
  s.S += xchg<3>(s.S); s.T += xchg<3>(s.T); s.cnt += xchg<3>(s.cnt);
  s.S += xchg<4>(s.S); s.T += xchg<4>(s.T); s.cnt += xchg<4>(s.cnt);
  s.S += xchg<5>(s.S); s.T += xchg<5>(s.T); s.cnt += xchg<5>(s.cnt);
}
// Sum over the records of a workgroup's waves (or a row's parts, at most 64), lane by lane; in every lane.
__device__ __forceinline__ Stats sum_records(const Stats* records, int n) {
  const int lane = threadIdx.x & 63;
  Stats s{kNegInf, kNegInf, 0.f, 0.f, 0};
  if (lane < n) s = records[lane];
  wave_stats(s);
  return s;
}

// The K largest of up to kMaxKeys keys in LDS: wave 0's lane k returns the k-th (0: fewer keys).
template <int KO>
__device__ __forceinline__ uint64_t largest(const uint64_t* keys, int n, uint64_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int at = wave * 64 + lane;
  uint64_t k = sort_lanes_desc(at < n ? keys[at] : 0ull);
  if (n <= 64) return k;  // (uniform)
  if (lane < KO) lds[wave * KO + lane] = k;
  __syncthreads();
  return sort_lanes_desc(lane < kWaves * KO ? lds[lane] : 0ull);
}

// A row's results from its statistics and top keys (wave 0).
__device__ __forceinline__ void write_row(const ScoreArgs& a, int row, const Stats& s, bool has_tok, bool tok_ok, float zt,
                                          uint64_t key) {
  const int lane = threadIdx.x & 63;
  const float nan = __builtin_nanf("");
  const bool bad = !(s.S == s.S), none = s.top == kNegInf;
  const float log_s = logf(s.S);
  if (lane == 0) {
    if (a.lse) a.lse[row] = bad ? nan : none ? kNegInf : s.top + log_s;
    if (a.entropy) a.entropy[row] = bad ? nan : none ? 0.f : log_s - s.T / s.S;
    if (a.tok_logprob)
      a.tok_logprob[row] = bad || (has_tok && !tok_ok) ? nan : !has_tok ? 0.f : none ? kNegInf : (zt - s.top) - log_s;
    if (a.tok_rank) a.tok_rank[row] = bad || !tok_ok ? -1 : s.cnt;
  }
  if (lane < a.topk_out) {
    const int64_t at = (int64_t)row * a.topk_out + lane;
    if (a.topk_id) a.topk_id[at] = bad ? -1 : key_id(key);
    if (a.topk_logprob) a.topk_logprob[at] = bad ? nan : none ? kNegInf : (key_value(key) - s.top) - log_s;
  }
}

template <typename T>
struct Vec {
  static constexpr int N = 16 / Elem<T>::kBytes;
  float z[N];
  __device__ __forceinline__ void load(const char* p) { set(ld16(p)); }
  __device__ __forceinline__ void set(u32x4 x) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (N == 4) z[e] = __uint_as_float(x[e]);
      else z[e] = __uint_as_float(e % 2 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16);
    }
  }
};

// The least float above x (x no NaN and not +inf).
__device__ __forceinline__ float next_above(float x) {
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return __uint_as_float(x < 0.f ? u - 1 : u + 1);
}

template <typename T, int KO>
__global__ __launch_bounds__(kThreads) void score_kernel(ScoreArgs a) {
  constexpr int N = Vec<T>::N, ES = Elem<T>::kBytes;
  __shared__ Stats l_stats[kWaves];
  __shared__ uint64_t l_top[kWaves * KO], l_keys[kMaxKeys];
  __shared__ int l_cand[KO];
  __shared__ int l_n[2];
  const int row = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x % (unsigned)a.parts);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
  const char* z = reinterpret_cast<const char*>(a.z) + (int64_t)row * a.row_stride * ES;
  // Vectors of N logits, aligned to 16 bytes: vector j holds logits j N - off .. ; those cut by the
  // row's ends ("edges", the first and the last) go element by element.
  const int off = (int)(((uintptr_t)z / ES) % N);
  const char* base = z - off * ES;
  const int v_lo = off ? 1 : 0, v_hi = (a.vocab + off) / N, nv = max(0, v_hi - v_lo);
  const int j0 = v_lo + (int)((int64_t)nv * part / a.parts), j1 = v_lo + (int)((int64_t)nv * (part + 1) / a.parts);
  const int tok = a.token ? a.token[row] : -1;
  const bool has_tok = tok != -1, tok_ok = tok >= 0 && tok < a.vocab;
  const float zt = tok_ok ? Elem<T>::to_f32(z, tok) : 0.f;
  // a logit counts for the rank if it is at least z_t before the token's vector, and more than z_t from
  // there on (the vector's own ties are added below)
  const int jt = tok_ok ? (tok + off) / N : 0;
  const float thr_lo = tok_ok ? zt : __builtin_huge_valf(), thr_hi = tok_ok ? next_above(zt) : __builtin_huge_valf();

  Stats s{kNegInf, kNegInf, 0.f, 0.f, 0};
  int jb = j0 + tid < j1 ? j0 + tid : -1;  // vector that held the thread's largest logit first ...
  u32x4 best = {0u, 0u, 0u, 0u};           // ... and what it holds
  float second = kNegInf;                  // the largest logit of the thread's other vectors
  auto step = [&](auto whole_c, int j) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(whole_c)::value;
    u32x4 raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      raw[u] = ld16(base + (int64_t)(WHOLE ? j + u * kThreads : max(min(j + u * kThreads, j1 - 1), j0)) * 16);
    if (j == j0 + tid) best = raw[0];
    Vec<T> x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      x[u].set(raw[u]);
      const int ju = j + u * kThreads;
      const bool in = WHOLE || ju < j1;
      float top = x[u].z[0];
#pragma unroll
      for (int e = 1; e < N; ++e) top = fmaxf(top, x[u].z[e]);
      const bool more = in && top > s.top;
      second = __builtin_amdgcn_fmed3f(second, s.top, in ? top : kNegInf);
      s.top = more ? top : s.top;
      jb = more ? ju : jb;
#pragma unroll
      for (int e = 0; e < 4; ++e) best[e] = more ? raw[u][e] : best[e];
      const float thr = in ? (ju < jt ? thr_lo : thr_hi) : __builtin_huge_valf();
#pragma unroll
      for (int e = 0; e < N; ++e) {
        x[u].z[e] = in ? x[u].z[e] : kNegInf;
        s.cnt += x[u].z[e] >= thr ? 1 : 0;
      }
    }
    if (__any(s.top > s.ref)) {
      if (s.top > s.ref) rebase(s, s.top);
    }
    const float ref = s.ref == kNegInf ? 0.f : s.ref;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = x[u].z[e] - ref, p = exp_f(d);  // (a NaN or +inf makes S a NaN)
        s.S += p;
        s.T = __builtin_fmaf(p, fmaxf(d, -200.f), s.T);  // (-inf: 0 times a finite number)
      }
  };
  int j = j0 + tid;
#pragma unroll 1
  for (; j - tid + kThreads * kUnroll <= j1; j += kThreads * kUnroll) step(std::integral_constant<bool, true>{}, j);
  if (j - tid < j1) step(std::integral_constant<bool, false>{}, j);
  // edges: thread e < N the row's first logits, N <= e < 2 N its last
  uint64_t edge = 0;
  if (tid < 2 * N) {
    const int id = tid < N ? (part == 0 && off && tid < N - off ? tid : -1)
                           : (part == a.parts - 1 ? v_hi * N - off + tid - N : -1);
    // (a row of less than one vector: its only logits are the last ones)
    if (id >= 0 && id < a.vocab && !(tid < N && v_hi < v_lo)) {
      const float x = Elem<T>::to_f32(z, id);
      edge = make_key(x, id);
      if (x > s.top) s.top = x;
      if (s.top > s.ref) rebase(s, s.top);
      const float d = x - (s.ref == kNegInf ? 0.f : s.ref), p = exp_f(d);
      s.S += p;
      s.T = __builtin_fmaf(p, fmaxf(d, -200.f), s.T);
      s.cnt += tok_ok && (x > zt || (x == zt && id < tok)) ? 1 : 0;
    }
  }
  // ties of the token's own vector in front of it
  if (tok_ok && jt >= j0 && jt < j1 && tid < N) {
    const int id = jt * N - off + tid;
    s.cnt += id < tok && Elem<T>::to_f32(z, id) == zt ? 1 : 0;
  }

  wave_stats(s);
  if (lane == 0) l_stats[wave] = s;

  // ---- top K of the part ----
  const bool want_top = a.topk_id || a.topk_logprob;
  uint64_t key = 0;
  if (want_top) {
    uint64_t mine = 0;
    if (jb >= 0) {
      Vec<T> x;
      x.set(best);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint64_t k = make_key(x.z[e], jb * N - off + e);
        mine = x.z[e] == x.z[e] && k > mine ? k : mine;
      }
    }
    const uint64_t sorted = sort_lanes_desc(mine);
    if (lane < KO) l_top[wave * KO + lane] = sorted;
    if (tid < 2) l_n[tid] = 0;
    __syncthreads();
    // (all of the waves' K largest: the largest of the waves' K-th would save a sort, and have up to four times the threads)
    const uint64_t H = key_of_lane(sort_lanes_desc(lane < kWaves * KO ? l_top[lane] : 0ull), KO - 1);
    if (mine != 0 && mine >= H) {  // (at most KO threads: keys are distinct)
      if (H == 0 || second >= key_value(H)) {
        l_cand[atomicAdd(&l_n[0], 1)] = tid;
      } else {
        Vec<T> v;
        v.set(best);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const uint64_t k = make_key(v.z[e], jb * N - off + e);
          if (k >= H && v.z[e] == v.z[e]) l_keys[atomicAdd(&l_n[1], 1)] = k;  // (with the edges' at most (KO + 2) N)
        }
      }
    }
    if (edge != 0 && edge >= H) l_keys[atomicAdd(&l_n[1], 1)] = edge;
    static_assert((KO + 2) * N <= kMaxKeys);
    __syncthreads();
    const int per = (j1 - j0 + kThreads - 1) / kThreads, total = l_n[0] * per;
    for (int x = tid; x < total; x += kThreads) {
      const int j = j0 + l_cand[x / per] + (x % per) * kThreads;
      if (j >= j1) continue;
      Vec<T> v;
      v.load(base + (int64_t)j * 16);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint64_t k = make_key(v.z[e], j * N - off + e);
        if (k >= H && v.z[e] == v.z[e]) {
          const int at = atomicAdd(&l_n[1], 1);
          if (at < kMaxKeys) l_keys[at] = k;
        }
      }
    }
    __syncthreads();
    const int n = l_n[1];
    if (n <= kMaxKeys) {
      key = largest<KO>(l_keys, n, l_top);
    } else {
      // more than that reach H (values in an order that favours few threads): the largest key below
      // the one before, KO times over
      const int e_lo = part == 0 ? 0 : j0 * N - off, e_hi = part == a.parts - 1 ? a.vocab : j1 * N - off;
      uint64_t below = ~0ull;
      for (int r = 0; r < KO; ++r) {
        uint64_t top = 0;
        for (int e = e_lo + tid; e < e_hi; e += kThreads) {
          const float x = Elem<T>::to_f32(z, e);
          const uint64_t k = make_key(x, e);
          top = x == x && k < below && k > top ? k : top;
        }
        top = key_of_lane(sort_lanes_desc(top), 0);
        __syncthreads();
        if (lane == 0) l_top[wave] = top;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) top = l_top[w] > top ? l_top[w] : top;
        below = top;
        key = lane == r ? top : key;
      }
    }
  }
  if (!want_top) __syncthreads();
  if (wave != 0) return;
  s = sum_records(l_stats, kWaves);
  if (a.parts == 1) {
    write_row(a, row, s, has_tok, tok_ok, zt, key);
  } else {
    float* p = a.part + ((int64_t)row * a.parts + part) * (kScoreWords + 2 * KO);
    if (lane == 0) *reinterpret_cast<f32x4*>(p) = f32x4{s.top, s.S, s.T, __int_as_float(s.cnt)};
    if (lane < KO) reinterpret_cast<uint64_t*>(p + kScoreWords)[lane] = key;
  }
}

// Rows that were scored in parts (kMaxKeys / KO at most).
template <typename T, int KO>
__global__ __launch_bounds__(kThreads) void score_join_kernel(ScoreArgs a) {
  __shared__ uint64_t l_top[kWaves * KO], l_keys[kMaxKeys];
  const int row = blockIdx.x, tid = threadIdx.x;
  const float* p = a.part + (int64_t)row * a.parts * (kScoreWords + 2 * KO);
  Stats s{kNegInf, kNegInf, 0.f, 0.f, 0};
  if (tid < a.parts) {  // (wave 0: at most 64)
    const f32x4 x = *reinterpret_cast<const f32x4*>(p + tid * (kScoreWords + 2 * KO));
    s = Stats{x[0], x[0], x[1], x[2], __float_as_int(x[3])};
  }
  if (tid < a.parts * KO)
    l_keys[tid] = reinterpret_cast<const uint64_t*>(p + (tid / KO) * (kScoreWords + 2 * KO) + kScoreWords)[tid % KO];
  __syncthreads();
  wave_stats(s);
  const uint64_t key = largest<KO>(l_keys, a.parts * KO, l_top);
  if (tid >= 64) return;
  const int tok = a.token ? a.token[row] : -1;
  const bool tok_ok = tok >= 0 && tok < a.vocab;
  const float zt = tok_ok ? Elem<T>::to_f32(a.z, (size_t)((int64_t)row * a.row_stride + tok)) : 0.f;
  write_row(a, row, s, tok != -1, tok_ok, zt, key);
}

template <typename T, int KO>
hipError_t go(const ScoreArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((score_kernel<T, KO>), dim3((unsigned)a.rows * a.parts), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  hipLaunchKernelGGL((score_join_kernel<T, KO>), dim3(a.rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_score(int dtype, int ko, const ScoreArgs& a, hipStream_t s) {
  if (dtype == 1) return ko == 8 ? go<bf16_t, 8>(a, s) : go<bf16_t, 16>(a, s);
  return ko == 8 ? go<float, 8>(a, s) : go<float, 16>(a, s);
}

}  // namespace respec
