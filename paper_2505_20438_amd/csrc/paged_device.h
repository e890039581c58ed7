// Device code shared by the kernels of the paged KV cache: packed rows, pages, values that are not finite.
#pragma once
#include "kernels_paged.h"
#include "lane_ops.h"

namespace ham {

// Where a workgroup's share of packed rows lies.  Each row has need(r) of them, in the order of the rows; share `i` is number
// `at` of row `r` (r < 0: there are no more).  All NT threads call it; `scratch` is NT / 32 + 2 ints of LDS, free again after it.
// Up to 64 rows every wave looks for itself.  Past that the waves do it together, PER chunks of 64 rows each at a time: 4,096 rows
// of a token appended 119 us, their attention behind 300 slots 1,139; with every wave by itself, chunk after chunk, 659 and 1,602.
struct Share {
  int r, at;
};
template <int NT, typename Need>
__device__ __forceinline__ Share find_share(int R, int i, int* scratch, const Need& need) {
  const int lane = threadIdx.x & 63;
  if (R <= 64) {
    const int n = lane < R ? need(lane) : 0, end = wave_scan(n);
    const uint64_t hit = __ballot(end > i);
    if (hit == 0) return Share{-1, 0};
    const int l = __builtin_ctzll(hit);
    return Share{l, i - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(n, l))};
  }
  constexpr int NW = NT / 64, PER = 4;
  int* found = scratch + 2 * NW;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int r0 = 0, turn = 0; r0 < R; r0 += NT * PER, turn ^= 1) {
    int n[PER], end[PER], total = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int r = r0 + (w * PER + k) * 64 + lane;
      n[k] = r < R ? need(r) : 0;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      end[k] = total + wave_scan(n[k]);
      total = __builtin_amdgcn_readlane(end[k], 63);
    }
    if (lane == 0) scratch[turn * NW + w] = total;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const int x = scratch[turn * NW + k];
      before += k < w ? x : 0;
      all += x;
    }
    if (i < all) {
      const int mine = i - before;
      if (mine >= 0 && mine < total) {
        bool done = false;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const uint64_t hit = __ballot(end[k] > mine);
          if (!done && hit != 0) {
            done = true;
            if (lane == (int)__builtin_ctzll(hit)) {
              found[0] = r0 + (w * PER + k) * 64 + lane;
              found[1] = mine - (end[k] - n[k]);
            }
          }
        }
      }
      __syncthreads();
      const Share s{__builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[1])};
      __syncthreads();
      return s;
    }
    i -= all;
  }
  return Share{-1, 0};
}

// A row's packed tokens [o, o + c): c < 0 where they do not lie in the call's N.
__device__ __forceinline__ int packed_count(const int* offsets, int r, int N) {
  const int o = offsets[r], e = offsets[r + 1];
  return o >= 0 && e >= o && e <= N ? e - o : -1;
}
// ... of a prompt's row, which also needs them among its n slots
__device__ __forceinline__ int prompt_count(const PagedAttnArgs& a, int r) {
  const int c = packed_count(a.offsets, r, a.N), n = a.kv_len[r];
  return n <= a.kv_max && c <= n ? c : -1;
}

// A page id of a table.  One outside the pool is an error, and page 0 is read in its place.
__device__ __forceinline__ int checked_page(int id, const PagedSizes& z, int* err) {
  if ((unsigned)id < (unsigned)z.n_pages) return id;
  atomicOr(err, 32);
  return 0;
}

// An int at a wave-uniform index that no one writes during the kernel, by a scalar load: in a scalar register, and the wait for
// it is none for the vector loads under way.
__device__ __forceinline__ int scalar_at(const int* table, int i) {
  typedef const __attribute__((address_space(4))) int* ConstInt;
  return ((ConstInt)(uintptr_t)table)[__builtin_amdgcn_readfirstlane(i)];
}

// This lane's number, formed anew: a register kept for it, or for what follows from it, through a loop that needs them all
// would be stored in memory, and the wait for its return is one for all loads under way.
__device__ __forceinline__ int lane_anew() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

// Whether any of the E values of 16 bytes is an infinity or NaN
template <typename T> __device__ __forceinline__ bool any_nonfinite(const u4& v);
template <> __device__ __forceinline__ bool any_nonfinite<bf16>(const u4& v) {
  uint32_t f = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) f |= (v[i] & 0x7F807F80u) + 0x00800080u;  // carries into the sign bit from an exponent of ones
  return (f & 0x80008000u) != 0;
}
template <> __device__ __forceinline__ bool any_nonfinite<float>(const u4& v) {
  uint32_t f = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) f |= (v[i] & 0x7F800000u) + 0x00800000u;
  return (f & 0x80000000u) != 0;
}

// Rows of one product see different slots, and a value that a row does not see has weight 0, but 0 times an infinity or NaN
// is NaN.  Such values are marked by a 1 in an operand for infinity (sign 0) or -infinity (sign 1), NaN in both, and taken
// out of v; products of the marks with the slots that a row sees count them, and what a row has seen is added to its sums.
template <typename T> __device__ __forceinline__ u4 mark_nonfinite(const u4& v, int sign) {
  constexpr uint32_t ONE = sizeof(T) == 2 ? 0x3F80u : 0x3F800000u, EXP = sizeof(T) == 2 ? 0x7F80u : 0x7F800000u;
  constexpr uint32_t MANT = sizeof(T) == 2 ? 0x7Fu : 0x7FFFFFu, SIGN = sizeof(T) == 2 ? 0x8000u : 0x80000000u;
  u4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = 0;
#pragma unroll
    for (int h = 0; h < 32; h += (int)sizeof(T) * 8) {
      const uint32_t x = v[i] >> h;
      if ((x & EXP) == EXP && ((x & MANT) != 0 || ((x & SIGN) != 0) == (sign != 0))) m[i] |= ONE << h;
    }
  }
  return m;
}
template <typename T> __device__ __forceinline__ void drop_nonfinite(u4& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      if ((v[i] & 0x7F80u) == 0x7F80u) v[i] &= 0xFFFF0000u;
      if ((v[i] & 0x7F800000u) == 0x7F800000u) v[i] &= 0x0000FFFFu;
    } else {
      if ((v[i] & 0x7F800000u) == 0x7F800000u) v[i] = 0;
    }
  }
}

// Eight fp32 values as three bf16 planes, each the 8 leading bits of what the ones before it leave: 24 bits in all.  (What a plane
// leaves of a value as a 2-term bf16 dot product, one instruction for two, is slower: 7 packed prompts 780 us for 731.)
__device__ __forceinline__ void weight_planes(const float* p, u4* pp) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t x = __float_as_uint(p[2 * i]), y = __float_as_uint(p[2 * i + 1]);
#pragma unroll
    for (int n = 0; n < 3; ++n) {
      pp[n][i] = __builtin_amdgcn_perm(y, x, 0x07060302u);  // the upper halves
      if (n == 2) break;
      x = __float_as_uint(__uint_as_float(x) - __uint_as_float(x & 0xFFFF0000u));
      y = __float_as_uint(__uint_as_float(y) - __uint_as_float(y & 0xFFFF0000u));
    }
  }
}

// Joins the splits' records of one query row: the weights of split s in lane s, relative to the greatest maximum; a lane's
// values of hd / 64 channels are added up in the order of the splits.
template <int HD>
__device__ __forceinline__ void join_row(const float* part, const float* ml, size_t rec, size_t step, int ns, float* o) {
  constexpr int V = HD / 64, UN = 8;
  const int lane = threadIdx.x & 63;
  const float* p = part + rec * HD + lane * V;
  float x[UN][V];
#pragma unroll
  for (int u = 0; u < UN; ++u)
#pragma unroll
    for (int v = 0; v < V; ++v) x[u][v] = u < ns ? p[(size_t)u * step * HD + v] : 0.f;
  float m = -INFINITY, l = 0.f;
  if (lane < ns) {
    m = ml[2 * (rec + (size_t)lane * step)];
    l = ml[2 * (rec + (size_t)lane * step) + 1];
  }
  const float M = group_max(row_max(m)), mz = M == -INFINITY ? 0.f : M;
  const float e = __builtin_amdgcn_exp2f(m - mz);
  const float L = group_sum(row_sum(e * l));
  const float w = L == 0.f ? 0.f : e / L;
#pragma unroll
  for (int v = 0; v < V; ++v) o[v] = 0.f;
#pragma unroll
  for (int u = 0; u < UN; ++u)
    if (u < ns) {
      const float wu = __shfl(w, u, WAVE);
#pragma unroll
      for (int v = 0; v < V; ++v) o[v] += wu * x[u][v];
    }
  for (int s = UN; s < ns; ++s) {
    const float ws = __shfl(w, s, WAVE);
#pragma unroll
    for (int v = 0; v < V; ++v) o[v] += ws * p[(size_t)s * step * HD + v];
  }
}

}  // namespace ham
