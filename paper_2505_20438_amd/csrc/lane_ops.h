// Device helpers shared by the cache operators (kernels_kv8.hip, kernels_paged*.hip): values of the storage type and
// activation rows in registers, sums and maxima over the lanes of a wave.
#pragma once
#include "device_common.h"

namespace ham {

// four values of the storage type as fp32
template <typename T> __device__ __forceinline__ f4 ld4(const T* p);
template <> __device__ __forceinline__ f4 ld4<float>(const float* p) { return *reinterpret_cast<const f4*>(p); }
template <> __device__ __forceinline__ f4 ld4<bf16>(const bf16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return f4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
            __uint_as_float(u.y & 0xFFFF0000u)};
}
template <typename T> __device__ __forceinline__ void st4(T* p, f4 v);
template <> __device__ __forceinline__ void st4<float>(float* p, f4 v) { *reinterpret_cast<f4*>(p) = v; }
template <> __device__ __forceinline__ void st4<bf16>(bf16* p, f4 v) {
  *reinterpret_cast<uint2*>(p) = uint2{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
}
template <typename T> __device__ __forceinline__ f4 stored4(f4 v) {  // rounded to the storage type
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = to_f<T>(from_f<T>(v[e]));
  return v;
}
// eight values of an activation row of width W
template <typename T> __device__ __forceinline__ void put_act8(void* base, size_t row, int W, int i, const f4* v) {
  if constexpr (Act<T>::SPLIT) {
    T* p = (T*)base + row * 2 * W + i;
    u4 hi, lo;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f4 h = stored4<T>(v[u]), d = v[u] - h;
      hi[2 * u] = f2bf2(h[0], h[1]);
      hi[2 * u + 1] = f2bf2(h[2], h[3]);
      lo[2 * u] = f2bf2(d[0], d[1]);
      lo[2 * u + 1] = f2bf2(d[2], d[3]);
    }
    *reinterpret_cast<u4*>(p) = hi;
    *reinterpret_cast<u4*>(p + W) = lo;
  } else {
    T* p = (T*)base + row * W + i;
    st4<T>(p, v[0]);
    st4<T>(p + 4, v[1]);
  }
}

// N values of the storage type as they lie in memory: a load without a conversion, which would wait for it
template <typename T, int N>
struct Raw {
  static constexpr int W = N * (int)sizeof(T) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W % 4 == 0) {
#pragma unroll
      for (int i = 0; i < W / 4; ++i) {
        const u4 v = ld16((const uint32_t*)p + 4 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * i + e] = v[e];
      }
    } else {
      static_assert(W == 2, "8 or a multiple of 16 bytes");
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x;
      w[1] = v.y;
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};

// the sum and the maximum over the 16 lanes of a row, in each of them
template <int ROR> __device__ __forceinline__ float row_ror(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + ROR, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_sum(float v) {
  v += row_ror<8>(v);
  v += row_ror<4>(v);
  v += row_ror<2>(v);
  return v + row_ror<1>(v);
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, row_ror<8>(v));
  v = fmaxf(v, row_ror<4>(v));
  v = fmaxf(v, row_ror<2>(v));
  return fmaxf(v, row_ror<1>(v));
}

// the greater of v in the four lane groups, in every lane (lanes 16 and 32 apart swapped on the vector units)
__device__ __forceinline__ float group_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float pair16_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float pair32_sum(float v) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float group_sum(float v) { return pair32_sum(pair16_sum(v)); }

// inclusive sum over the lanes up to this one, of a row of 16 and of the wave
__device__ __forceinline__ int row_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  return v + __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
}
__device__ __forceinline__ int wave_scan(int v) {
  v = row_scan(v);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // lane 15 of rows 0 and 2 to the rows after them
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31 to the upper half
  return v;
}

// Rotate-half RoPE of the pair (x, y): products and sums are rounded one by one (no fused multiply-add), so that what is
// rounded to fewer bits next does not depend on how the compiler contracts.
__device__ __forceinline__ void rotate(f4& x, f4& y, f4 c, f4 s) {
#pragma clang fp contract(off)
  const f4 xc = x * c, ys = y * s, yc = y * c, xs = x * s;
  x = xc - ys;
  y = yc + xs;
}

// fp32 values as N bf16 planes, v = p0 + p1 (+ p2): 16 or 24 significant bits
template <int N>
__device__ __forceinline__ void to_planes(const float* v, u4* p) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    p[n] = pack_frag_bf16(r);
    if (n + 1 < N) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] -= bf2f((bf16)((e & 1) ? (p[n][e >> 1] >> 16) : (p[n][e >> 1] & 0xFFFFu)));
    }
  }
}

}  // namespace ham
