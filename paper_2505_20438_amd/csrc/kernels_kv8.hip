// Operators on a KV cache in 8 bits (layout: kernels_kv8.h).
//
// A closed block of 32 slots of a kv head is held as e4m3 codes with one fp32 scale for K and one for V:
//   a = max |x| over the block's 32 x hd values (rounded to the storage type first), scale = a / 448,
//   code = e4m3(clamp(x / scale)), nearest even, as x * (1 / scale);
// a scale below the least normal fp32 value makes every code 0, and a block with an infinity or NaN has scale NaN, so
// that every row that reads it becomes NaN.  The slots past the last full block are in the open block, in the storage
// type; a block is coded once, when its 32nd slot arrives, so the cache does not depend on how its tokens arrived.
//
// k_kv8_append   RoPE of projection rows, K and V into the cache, q out.
// k_kv8_pack     a filled cache of the storage type into the 8-bit cache.
// k_kv8_scores, k_kv8_pick   the blocks whose keys' upper bounds are greatest (k_kv8_pick_few: short rows in one launch).
// k_kv8_attn, k_kv8_combine  attention of one query row per sequence over all or listed blocks and the open one.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "kernels_kv8.h"
#include "launch_rules.h"

namespace ham {

namespace {

// ---------------------------------------------------------------- values and codes
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

// the greatest over a row of 16 lanes and over a wave, in each lane (lanes 16 and 32 apart are swapped on the vector units)
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, true));  // row_ror 8, 4, 2, 1
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x122, 0xF, 0xF, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x121, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = row_max(v);
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((uint32_t)b[0], (uint32_t)b[1]);
}

// Rotate-half RoPE of the pair (x, y): products and sums are rounded one by one (no fused multiply-add), so that what is
// rounded to 8 bits next does not depend on how the compiler contracts.
__device__ __forceinline__ void rotate(f4& x, f4& y, f4 c, f4 s) {
#pragma clang fp contract(off)
  const f4 xc = x * c, ys = y * s, yc = y * c, xs = x * s;
  x = xc - ys;
  y = yc + xs;
}

// Scale of a block from the bits of its greatest magnitude, and what its values are multiplied by.
__device__ __forceinline__ void block_scale(uint32_t top, float& scale, float& inv) {
  scale = top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(top) / KV8_MAX;
  inv = scale >= 1.17549435e-38f ? 1.0f / scale : 0.0f;
}
// |x inv| is at most 448 and two roundings; the conversion takes what is below 464 to 448
__device__ __forceinline__ uint32_t code4(const float* x, float inv) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
}
__device__ __forceinline__ uint32_t magnitude(uint32_t top, float v) { return max(top, __float_as_uint(v) & 0x7FFFFFFFu); }

// A full block is coded by 2 HD threads from their registers.  The first HD hold K: thread (t, g, r) of slot 8 (r / 4) + 4 t
// + r % 4 the 16 channels from 16 g on and those HD / 2 after them (the other half of their RoPE pairs), which are two
// 16-byte pieces of the codes.  The others hold V, and find the least and greatest value of K in each channel from a copy
// in LDS.
template <int HD>
struct CodeLds {
  uint32_t top[2 * HD / 64];
  float k[KV8_BLOCK][HD + 4];
};
template <int HD> struct KeyThread {  // of thread tid < HD
  int t, g, r, slot, d0;
  __device__ __forceinline__ explicit KeyThread(int tid) {
    constexpr int G = HD / 32;  // channel groups of 16 in half a head
    t = tid / (16 * G);
    g = tid / 16 % G;
    r = tid % 16;
    slot = 8 * (r / 4) + 4 * t + r % 4;
    d0 = 16 * g;
  }
};
template <int HD>
__device__ __forceinline__ void share_keys(CodeLds<HD>& sh, const KeyThread<HD>& kt, const float* k0, const float* k1) {
#pragma unroll
  for (int e = 0; e < 16; e += 4) {
    *reinterpret_cast<f4*>(&sh.k[kt.slot][kt.d0 + e]) = f4{k0[e], k0[e + 1], k0[e + 2], k0[e + 3]};
    *reinterpret_cast<f4*>(&sh.k[kt.slot][kt.d0 + HD / 2 + e]) = f4{k1[e], k1[e + 1], k1[e + 2], k1[e + 3]};
  }
}
__device__ __forceinline__ void wave_top(uint32_t* tops, uint32_t top) {
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
}
// after a barrier: the scales of the block, written by one thread
template <int HD>
__device__ __forceinline__ void block_scales(const CodeLds<HD>& sh, const Kv8Cache& c, size_t blk, float& ki, float& vi) {
  float ks, vs;
  uint32_t k = sh.top[0], v = sh.top[HD / 64];
  if constexpr (HD == 128) {
    k = max(k, sh.top[1]);
    v = max(v, sh.top[3]);
  }
  block_scale(k, ks, ki);
  block_scale(v, vs, vi);
  if (threadIdx.x == 0) {
    c.scales[2 * blk] = ks;
    c.scales[2 * blk + 1] = vs;
  }
}
template <int HD>
__device__ __forceinline__ void write_keys(const KeyThread<HD>& kt, const float* k0, const float* k1, float ki, const Kv8Cache& c,
                                           size_t blk) {
  uint8_t* out = c.codes + blk * (2 * KV8_BLOCK * HD);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = code4((h ? k1 : k0) + 4 * e, ki);
    *reinterpret_cast<u4*>(out + kv8_k_index(kt.slot, kt.d0 + h * (HD / 2), HD)) = w;
  }
}
// bounds of channel d; coding keeps the order, so the least code is that of the least value
template <int HD>
__device__ __forceinline__ void write_bounds(const CodeLds<HD>& sh, int d, float ki, const Kv8Cache& c, size_t blk) {
  float lo = sh.k[0][d], hi = lo;
#pragma unroll
  for (int s = 1; s < KV8_BLOCK; ++s) {
    lo = fminf(lo, sh.k[s][d]);
    hi = fmaxf(hi, sh.k[s][d]);
  }
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(lo * ki, hi * ki, 0, false);
  uint8_t* b = c.bounds + blk * (2 * HD) + d / 8 * 16 + d % 8;
  b[0] = (uint8_t)w;
  b[8] = (uint8_t)(w >> 8);
}

// ---------------------------------------------------------------- append
// Two kinds of workgroup for each of the nb steps of 32 tokens, row and kv head.  One: block `first + x` of the row if the
// new tokens fill it; that of step 0 also puts the tokens past the last full block into the open one, after it has read
// what the open block held (so no other workgroup touches it).  The other (if q is wanted): q of 32 tokens, 8 pairs a
// thread.  All of one step of a row run on one XCD (workgroups go round the eight of them), whose L2 then holds the step's
// RoPE factors: with a row's heads on every XCD 22% more bytes were read.  Bound by memory: 8 kv heads of 128, 4 q-heads each,
// bf16, 4 rows x 4,001 tokens 133 us (645 MB, 4.9 TB/s; K and V alone 43 us); 32 rows x 1 token 2.8 us, 5.7 where all 256
// blocks fill up (a chain of loads, maximum, barrier and stores, once).
template <typename T, int HD>
__global__ __launch_bounds__(2 * HD) void k_kv8_append(Kv8AppendArgs a, int nb) {
  constexpr int B = KV8_BLOCK, HALF = HD / 2, QPS = HALF / 4, THREADS = 2 * HD;  // QPS: quads of pairs per head
  __shared__ CodeLds<HD> sh;
  const int tid = threadIdx.x, grp = a.grp, kinds = a.q ? 2 : 1;
  const uint32_t s8 = blockIdx.x / 8, step = s8 / (uint32_t)(kinds * a.Hk) * 8 + blockIdx.x % 8, head = s8 % (uint32_t)(kinds * a.Hk);
  const int r = (int)(step / (uint32_t)nb), x0 = (int)(step % (uint32_t)nb), kvh = (int)head % a.Hk;
  if (r >= a.R) return;
  const int n0 = a.start[r], cnt = a.count[r];
  if (n0 < 0 || cnt < 0 || cnt > a.T || (long long)n0 + cnt > a.slots) {
    if (x0 == 0 && head == 0 && tid == 0) atomicOr(a.err + r, 8);
    return;
  }
  const int ld = (a.H + 2 * a.Hk) * HD;
  const float* src = a.qkv + (size_t)r * a.T * ld;
  const float* cs = a.cos + (size_t)r * a.T * HALF;
  const float* sn = a.sin + (size_t)r * a.T * HALF;
  if ((int)head >= a.Hk) {  // q
    const int t0 = x0 * 32, t1 = min(cnt, t0 + 32), items = (t1 - t0) * grp * (HALF / 8);
    for (int q = tid; q < items; q += THREADS) {
      const int i = q % (HALF / 8) * 8, hq = q / (HALF / 8), t = t0 + hq / grp, h = kvh * grp + hq % grp;
      const float* p = src + (size_t)t * ld + h * HD + i;
      f4 x[2], y[2], c[2], s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        x[u] = *reinterpret_cast<const f4*>(p + 4 * u);
        y[u] = *reinterpret_cast<const f4*>(p + HALF + 4 * u);
        c[u] = *reinterpret_cast<const f4*>(cs + (size_t)t * HALF + i + 4 * u);
        s[u] = *reinterpret_cast<const f4*>(sn + (size_t)t * HALF + i + 4 * u);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) rotate(x[u], y[u], c[u], s[u]);
      const size_t row = (size_t)r * a.T + t;
      put_act8<T>(a.q, row, a.H * HD, h * HD + i, x);
      put_act8<T>(a.q, row, a.H * HD, h * HD + i + HALF, y);
    }
    return;
  }
  const int end = n0 + cnt, first = n0 / B, last = end / B;
  const size_t pair = (size_t)r * a.Hk + kvh;
  T* open = (T*)a.c.open + pair * 2 * B * HD;  // K, then V
  const float* ksrc = src + (size_t)(a.H + kvh) * HD;
  const float* vsrc = ksrc + (size_t)a.Hk * HD;
  const auto key = [&](int t, int i, f4& x, f4& y) {
    const float* p = ksrc + (size_t)t * ld + i;
    x = *reinterpret_cast<const f4*>(p);
    y = *reinterpret_cast<const f4*>(p + HALF);
    rotate(x, y, *reinterpret_cast<const f4*>(cs + (size_t)t * HALF + i), *reinterpret_cast<const f4*>(sn + (size_t)t * HALF + i));
  };
  if (x0 < last - first) {
    const size_t blk = pair * a.c.NB + first + x0;
    const int base = (first + x0) * B - n0;  // token of the block's slot 0
    float ki, vi;
    if (tid < HD) {
      const KeyThread<HD> kt(tid);
      // every load first (a token for every lane, also where the slot is an old one), then the arithmetic
      const int t = max(base + kt.slot, 0);
      const float* p = ksrc + (size_t)t * ld + kt.d0;
      f4 x[4], y[4], c[4], sv[4];
      Raw<T, 4> ox[4], oy[4];
      if (base < 0) {  // the row's first block: slots from the open one
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ox[i].load(open + kt.slot * HD + kt.d0 + 4 * i);
          oy[i].load(open + kt.slot * HD + kt.d0 + HALF + 4 * i);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = *reinterpret_cast<const f4*>(p + 4 * i);
        y[i] = *reinterpret_cast<const f4*>(p + HALF + 4 * i);
        c[i] = *reinterpret_cast<const f4*>(cs + (size_t)t * HALF + kt.d0 + 4 * i);
        sv[i] = *reinterpret_cast<const f4*>(sn + (size_t)t * HALF + kt.d0 + 4 * i);
      }
      float k0[16], k1[16];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        rotate(x[i], y[i], c[i], sv[i]);
        x[i] = stored4<T>(x[i]);
        y[i] = stored4<T>(y[i]);
        if (base < 0 && base + kt.slot < 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[i][e] = ox[i].at(e);
            y[i][e] = oy[i].at(e);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          top = magnitude(magnitude(top, x[i][e]), y[i][e]);
          k0[4 * i + e] = x[i][e];
          k1[4 * i + e] = y[i][e];
        }
      }
      share_keys<HD>(sh, kt, k0, k1);
      wave_top(sh.top, top);
      __syncthreads();
      block_scales<HD>(sh, a.c, blk, ki, vi);
      write_keys<HD>(kt, k0, k1, ki, a.c, blk);
    } else {  // V: channels d .. d + 3 of slots 8 g ..
      const int d = (tid - HD) % (HD / 4) * 4, g = (tid - HD) / (HD / 4);
      f4 v[8];
      Raw<T, 4> ov[8];
      uint32_t top = 0;
      if (base < 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) ov[i].load(open + (B + 8 * g + i) * HD + d);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f4*>(vsrc + (size_t)max(base + 8 * g + i, 0) * ld + d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = stored4<T>(v[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (base < 0 && base + 8 * g + i < 0) v[i][e] = ov[i].at(e);
          top = magnitude(top, v[i][e]);
        }
      }
      wave_top(sh.top, top);
      __syncthreads();
      block_scales<HD>(sh, a.c, blk, ki, vi);
      uint8_t* out = a.c.codes + blk * (2 * B * HD) + B * HD;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo[4] = {v[0][e], v[1][e], v[2][e], v[3][e]}, hi[4] = {v[4][e], v[5][e], v[6][e], v[7][e]};
        *reinterpret_cast<uint2*>(out + kv8_v_index(8 * g, d + e)) = uint2{code4(lo, vi), code4(hi, vi)};
      }
      write_bounds<HD>(sh, tid - HD, ki, a.c, blk);
    }
  }
  if (x0 == 0) {  // slots of the open block: tokens t of slots max(n0, 32 last) .. end (what it held has been read: a barrier)
    const int s0 = max(n0, last * B), ns = end - s0;
    for (int q = tid; q < ns * QPS; q += THREADS) {
      const int s = s0 + q / QPS, i = q % QPS * 4, w = s - last * B;
      f4 x, y;
      key(s - n0, i, x, y);
      st4<T>(open + w * HD + i, x);
      st4<T>(open + w * HD + i + HALF, y);
    }
    for (int q = tid; q < ns * (HD / 4); q += THREADS) {
      const int s = s0 + q / (HD / 4), i = q % (HD / 4) * 4, w = s - last * B;
      st4<T>(open + (B + w) * HD + i, *reinterpret_cast<const f4*>(vsrc + (size_t)(s - n0) * ld + i));
    }
  }
}

// ---------------------------------------------------------------- pack
// One workgroup per (block, kv head, row): a full block is coded, the slots past the last full block go to the open one.
// Every value is read once, into registers, and coded from there.  Bound by memory: 4 rows of up to 8,190 slots, 8 kv heads of
// 128, bf16, 36 us (120 MB read, 62 written, 5.0 TB/s).
template <typename T, int HD>
__global__ __launch_bounds__(2 * HD) void k_kv8_pack(Kv8PackArgs a) {
  constexpr int B = KV8_BLOCK, THREADS = 2 * HD;
  __shared__ CodeLds<HD> sh;
  const int tid = threadIdx.x, b = blockIdx.x, kvh = blockIdx.y, r = blockIdx.z, n = a.kv_len[r];
  if (n < 0 || n > a.kv_max) {
    if (b == 0 && kvh == 0 && tid == 0) atomicOr(a.err + r, 8);
    return;
  }
  const int closed = n / B, ns = min(B, n - b * B);
  if (ns <= 0) return;
  const size_t pair = (size_t)r * a.Hk + kvh, blk = pair * a.c.NB + b;
  const T* K = (const T*)a.K + (pair * a.S + (size_t)b * B) * HD;
  const T* VT = (const T*)a.VT + (pair * a.S + (size_t)b * B) * HD;  // [hd][32]
  if (b == closed) {  // the open block
    T* open = (T*)a.c.open + pair * 2 * B * HD;
    for (int q = tid; q < ns * (HD / 4); q += THREADS) st4<T>(open + q * 4, ld4<T>(K + q * 4));
    for (int q = tid; q < ns * HD; q += THREADS) open[B * HD + q] = VT[q % HD * B + q / HD];
    return;
  }
  uint32_t top = 0;
  float ki, vi;
  if (tid < HD) {
    const KeyThread<HD> kt(tid);
    Raw<T, 16> x, y;
    x.load(K + kt.slot * HD + kt.d0);
    y.load(K + kt.slot * HD + kt.d0 + HD / 2);
    float k0[16], k1[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      k0[e] = x.at(e);
      k1[e] = y.at(e);
      top = magnitude(magnitude(top, k0[e]), k1[e]);
    }
    share_keys<HD>(sh, kt, k0, k1);
    wave_top(sh.top, top);
    __syncthreads();
    block_scales<HD>(sh, a.c, blk, ki, vi);
    write_keys<HD>(kt, k0, k1, ki, a.c, blk);
  } else {  // V: two 16-byte pieces, each slots 8 g .. of channels 32 p + r and 32 p + 16 + r
    Raw<T, 8> v[2][2];
    const int q0 = tid - HD;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int q = q0 + u * HD;
        v[u][h].load(VT + (q / 64 * 32 + 16 * h + q % 16) * B + q / 16 % 4 * 8);
      }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = magnitude(top, v[u][h].at(e));
    wave_top(sh.top, top);
    __syncthreads();
    block_scales<HD>(sh, a.c, blk, ki, vi);
    uint8_t* out = a.c.codes + blk * (2 * B * HD) + B * HD;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = v[u][e / 2].at((4 * e + i) % 8);
        w[e] = code4(f, vi);
      }
      *reinterpret_cast<u4*>(out + (q0 + u * HD) * 16) = w;
    }
    write_bounds<HD>(sh, q0, ki, a.c, blk);
  }
}

// ---------------------------------------------------------------- select
// Upper bound of q . k over the keys of a block, in each channel by the greater of q lo and q hi:
//   sum_d max(q_d lo_d, q_d hi_d) = sum_d (q_d (lo_d + hi_d) + |q_d| (hi_d - lo_d)) / 2,
// the greatest over the kv head's q-heads, times the block's scale.  Products of q (24 bits) and codes (4 bits) and their
// sums are taken in fp64: blocks are compared by these values, and fp32 sums of another order would order near ones
// differently.  HD / 8 lanes to a block, 8 channels each; four heads at a time.
template <int CTRL> __device__ __forceinline__ double dpp64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)u, CTRL, 0xF, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
constexpr int XOR1 = 0xB1, XOR2 = 0x4E, QUAD_REV = 0x1B, HALF_MIRROR = 0x141, ROR8 = 0x128;  // lanes of a row
__device__ __forceinline__ double max_nan(double a, double b) { return (b > a || b != b) ? b : a; }  // NaN stays

template <typename T, int HD>
struct BlockScore {
  double q[4][8];
  int heads;  // of the four
  // heads h0 .. of kv head kvh, this lane's channels
  __device__ __forceinline__ void load(const Kv8SelectArgs& a, int r, int kvh, int h0) {
    constexpr int PL = Act<T>::PL;
    heads = min(4, a.grp - h0);
    Raw<T, 8> raw[4][PL];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const T* p = (const T*)a.q + (size_t)r * PL * a.H * HD + (kvh * a.grp + h0 + min(j, heads - 1)) * HD + threadIdx.x % (HD / 8) * 8;
#pragma unroll
      for (int i = 0; i < PL; ++i) raw[j][i].load(p + i * a.H * HD);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) q[j][e] = (double)(PL == 1 ? raw[j][0].at(e) : raw[j][0].at(e) + raw[j][PL - 1].at(e));
  }
  // twice the greatest bound of the heads, w: the lane's 8 least and 8 greatest codes; the same in every lane of the block
  __device__ __forceinline__ double operator()(u4 w) const {
    double s[4] = {0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const auto lo = p % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(w[p / 2], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[p / 2], false);
      const auto hi = p % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(w[2 + p / 2], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[2 + p / 2], false);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const double sum = (double)(lo[e] + hi[e]), dif = (double)(hi[e] - lo[e]);  // of two codes, exact in fp32
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[j] = fma(q[j][2 * p + e], sum, s[j]);
          s[j] = fma(fabs(q[j][2 * p + e]), dif, s[j]);
        }
      }
    }
    // sums over the block's lanes: each lane of four gives three heads away and keeps one
    const bool odd = threadIdx.x & 1, two = threadIdx.x & 2;
    double a = (odd ? s[2] : s[0]) + dpp64<XOR1>(odd ? s[0] : s[2]);
    double b = (odd ? s[3] : s[1]) + dpp64<XOR1>(odd ? s[1] : s[3]);
    a = (two ? b : a) + dpp64<XOR2>(two ? a : b);
    a += dpp64<QUAD_REV>(dpp64<HALF_MIRROR>(a));  // the lane 4 away
    if constexpr (HD == 128) a += dpp64<ROR8>(a);
    if ((odd ? 2 : 0) + (two ? 1 : 0) >= heads) a = -INFINITY;
    a = max_nan(a, dpp64<XOR1>(a));
    return max_nan(a, dpp64<XOR2>(a));
  }
};
// Bounds of the blocks [b0, b1) of a (row, kv head) for all heads: put(b, twice the bound, first four heads) by one lane of
// each.  A wave takes 64 / LPB blocks at a time, NW of them in turn; the loop is not unrolled (a call fetches its code from
// memory), the next blocks' codes are on their way.
template <typename T, int HD, int NW, typename Put>
__device__ __forceinline__ void score_blocks(const Kv8SelectArgs& a, int r, int kvh, size_t pair, int b0, int b1, Put put) {
  constexpr int LPB = HD / 8, BPW = 64 / LPB;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, sub = lane / LPB, c = lane % LPB;
  const uint8_t* bounds = a.c.bounds + pair * a.c.NB * (2 * HD) + c * 16;
  BlockScore<T, HD> score;
  for (int h0 = 0; h0 < a.grp; h0 += 4) {
    u4 next = zero16();
    if (b0 + w * BPW < b1) next = ld16(bounds + (size_t)min(b0 + w * BPW + sub, b1 - 1) * (2 * HD));
    score.load(a, r, kvh, h0);
#pragma unroll 1
    for (int b = b0 + w * BPW; b < b1; b += NW * BPW) {
      const u4 code = next;
      next = ld16(bounds + (size_t)min(b + NW * BPW + sub, b1 - 1) * (2 * HD));
      const double v = score(code);
      if (c == 0 && b + sub < b1) put(b + sub, v, h0 == 0);
    }
  }
}
// K's scale, or NaN for a block whose K or V holds an infinity or NaN: the block is then among the chosen and is seen
__device__ __forceinline__ float score_scale(const float* scales, size_t blk) {
  const float2 s = *reinterpret_cast<const float2*>(scales + 2 * blk);
  return s.y != s.y ? s.y : s.x;
}
__device__ __forceinline__ float block_score(double twice, float scale) { return (float)(0.5 * twice * (double)scale) + 0.0f; }

// Scores of `per` (at most SCORE_BLOCKS) blocks of a (row, kv head) a workgroup, up to kv_max (blocks that are there, whatever
// the length).  Bound by latency: ~150 instructions of a wave before its first 512 / hd blocks, then ~250, most of them fp64, in
// chains for each of them, with about two waves a SIMD at 4 rows.  4 rows x 1,040 blocks, 8 kv heads of 128: 7.0 us (8.8 MB),
// of which the 1.72 M vector instructions take 2.8 to issue (four cycles each, 1,024 SIMDs).
constexpr int SCORE_NW = 4, SCORE_BLOCKS = 64;
template <typename T, int HD>
__global__ __launch_bounds__(64 * SCORE_NW) void k_kv8_scores(Kv8SelectArgs a, int nb_max, int per) {
  __shared__ double best[SCORE_BLOCKS];
  const int kvh = blockIdx.y, r = blockIdx.z, b0 = blockIdx.x * per, b1 = min(nb_max, b0 + per);
  const size_t pair = (size_t)r * a.Hk + kvh;
  const int i = threadIdx.x;
  const float scale = i < b1 - b0 ? score_scale(a.c.scales, pair * a.c.NB + b0 + i) : 0.f;
  score_blocks<T, HD, SCORE_NW>(a, r, kvh, pair, b0, b1, [&](int b, double v, bool first) {
    best[b - b0] = first ? v : max_nan(best[b - b0], v);
  });
  lds_barrier();
  if (i < b1 - b0) a.scores[pair * nb_max + b0 + i] = block_score(best[i], scale);
}

// The n best blocks of a (row, kv head), in the order of their indices.  Equal scores: the lower index.  A NaN (a block
// with an infinity or NaN in K or V) counts as greatest, so that it is read and seen.  Blocks [f, l) are chosen by score, those before
// and after are always taken.
__device__ __forceinline__ uint32_t score_key(float s) {
  const uint32_t u = __float_as_uint(s);
  return s != s ? 0xFFFFFFFFu : (u & 0x80000000u ? ~u : u | 0x80000000u);
}
struct Choice {
  int closed, take, f, l, need;
  __device__ __forceinline__ Choice(const Kv8SelectArgs& a, int n, int on, int r, int kvh, size_t pair) {
    const bool bad = n < 0 || n > a.kv_max;
    if (bad && kvh == 0 && threadIdx.x == 0) atomicOr(a.err + r, 8);
    closed = bad || !on ? 0 : n / KV8_BLOCK;
    take = min(a.n, closed);
    f = a.first;
    l = closed - a.last;
    need = take - a.first - a.last;  // not negative where closed > a.n
    if (threadIdx.x == 0) a.n_blocks[pair] = take;
  }
};

// Rows of up to PICK_FEW blocks: one launch.  A workgroup scores the blocks of its (row, kv head); for block b thread b and
// three more count the blocks that go before it, a quarter of them each.  32 rows x 80 blocks, 8 kv heads of 128: 6.1 us,
// latency.  PICK_FEW, us here / as two launches at 128, 160 and 192 blocks of 128: 1 row 6.7 / 7.0, 7.8 / 7.2, 8.8 / 7.1;
// 4 rows 7.1 / 7.6, 8.3 / 8.1, 9.2 / 8.4; 32 rows 7.3 / 10.0, 8.5 / 10.8, 9.4 / 11.2; head dim 64 faster here at all of them.
// MOST: the workgroup that just holds the row (32 rows x 80 blocks 6.1 us with 8 waves for 128 blocks, 6.8 with 16 for 256).
constexpr int PICK_FEW = 192;
template <typename T, int HD, int MOST>
__global__ __launch_bounds__(4 * MOST) void k_kv8_pick_few(Kv8SelectArgs a, int nb_max) {
  constexpr int PARTS = 4;
  __shared__ double best[MOST];
  __shared__ __align__(16) uint32_t keys[MOST];
  __shared__ int wsum[MOST / 64], parts[PARTS][MOST];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, kvh = blockIdx.x, r = blockIdx.y, n = a.kv_len[r], on = a.enable[r];
  const size_t pair = (size_t)r * a.Hk + kvh;
  const float scale = tid < nb_max ? score_scale(a.c.scales, pair * a.c.NB + tid) : 0.f;
  score_blocks<T, HD, MOST / 16>(a, r, kvh, pair, 0, nb_max, [&](int b, double v, bool first) {
    best[b] = first ? v : max_nan(best[b], v);
  });
  const Choice ch(a, n, on, r, kvh, pair);
  int* out = a.blocks + pair * a.n;
  for (int i = ch.take + tid; i < a.n; i += 4 * MOST) out[i] = -1;
  lds_barrier();
  // blocks that are not chosen by score have key 0, which no score has
  if (tid < MOST) keys[tid] = tid >= ch.f && tid < ch.l ? score_key(block_score(best[tid], scale)) : 0u;
  lds_barrier();
  const int b = tid % MOST, part = tid / MOST;
  const uint32_t k = keys[b];
  int before = 0;
#pragma unroll 2
  for (int i = (ch.f & ~3) + 4 * part; i < ch.l; i += 4 * PARTS) {
    const u4 v = *reinterpret_cast<const u4*>(&keys[i]);
#pragma unroll
    for (int e = 0; e < 4; ++e) before += v[e] > k || (v[e] == k && i + e < b);
  }
  parts[part][b] = before;
  lds_barrier();
  if (tid >= MOST) return;  // the barrier below counts the waves that are left
#pragma unroll
  for (int i = 1; i < PARTS; ++i) before += parts[i][b];
  const bool taken = tid < ch.closed && (ch.closed <= a.n || tid < ch.f || tid >= ch.l || before < ch.need);
  const unsigned long long m = __ballot(taken);
  if (lane == 0) wsum[w] = __popcll(m);
  lds_barrier();
  if (taken) {
    int at = __popcll(m & ((1ull << lane) - 1));
    for (int i = 0; i < w; ++i) at += wsum[i];
    out[at] = tid;
  }
}

// Longer rows: scores by k_kv8_scores, then one workgroup per (row, kv head) finds the key of the last block to be taken:
// the keys' range in 1,024 bins, the bin in which the count from above reaches the number wanted, and so on within it until
// it holds few enough keys to count for each what lies above it (after one round, unless many are equal), or one value.
// Those above the key and the first of those equal to it are then written in the order of the blocks.  The keys stay in
// registers, UN a thread (at 16 the masks of the ballots overflow the scalar registers: 76 are kept in a vector register); rows
// of more than 16 a thread are read again for each step.  Every step is a few dependent
// instructions and a barrier, and a lone wave issues one instruction in eight to ten cycles: sixteen waves, not four (4 x
// 1,040 blocks 17 -> 13 us with the scores, 12 with the counts shared by the waves, of which this kernel 5).
constexpr int PICK_BINS = 1024, PICK_CAND = 128;  // counting 256 keys takes as long as three rounds of bins
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
template <int UN>
__global__ __launch_bounds__(1024) void k_kv8_pick(Kv8SelectArgs a, int nb_max) {
  constexpr int NW = 16, NT = 64 * NW, STEP = UN * NT, PER = UN * NW > 64 ? UN * NW / 64 : 1;
  __shared__ int hist[PICK_BINS], counts[UN * NW], sums[NW], s_m, s_need, s_want, s_cand;
  __shared__ __align__(16) uint32_t cand[PICK_CAND];
  __shared__ int above[PICK_CAND], upto[PICK_CAND];
  __shared__ uint32_t wlo[NW], whi[NW], s_lo, s_hi;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), kvh = blockIdx.x, r = blockIdx.y;
  const int n = a.kv_len[r], on = a.enable[r];
  const size_t pair = (size_t)r * a.Hk + kvh;
  const float* sc = a.scores + pair * nb_max;
  float v[UN];  // the first scores, before the row's length is known (they are there up to kv_max)
#pragma unroll
  for (int u = 0; u < UN; ++u) v[u] = sc[min(a.first + tid + u * NT, max(nb_max, 1) - 1)];
  static_assert(PICK_BINS == NT, "a bin a thread");
  hist[tid] = 0;
  if (tid < PICK_CAND) {
    cand[tid] = 0;
    above[tid] = 0;
    upto[tid] = 0;
  }
  if (tid == 0) s_cand = 0;
  const Choice ch(a, n, on, r, kvh, pair);
  const int f = ch.f, l = ch.l;
  int need = ch.need;
  int* out = a.blocks + pair * a.n;
  const bool all = ch.closed <= a.n;
  for (int i = tid; i < a.n; i += NT)
    if (i >= ch.take) out[i] = -1;
    else if (all || i < f) out[i] = i;
    else if (i >= ch.take - a.last) out[i] = ch.closed - (ch.take - i);
  if (all || need <= 0) return;
  const bool many = l - f > STEP;
  uint32_t k[UN];  // keys of the blocks c + tid, c + tid + NT, ..: 0 (which no score has) past the last
  const auto keys_of = [&](int c) {
#pragma unroll
    for (int u = 0; u < UN; ++u) k[u] = c + tid + u * NT < l ? score_key(v[u]) : 0;
  };
  const auto fetch = [&](int c) {
#pragma unroll
    for (int u = 0; u < UN; ++u) v[u] = sc[min(c + tid + u * NT, l - 1)];
    keys_of(c);
  };
  keys_of(f);
  uint32_t lo = 0xFFFFFFFFu, hi = 0;
  for (int c = f; c < l; c += STEP) {
    if (c > f) fetch(c);
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      lo = min(lo, k[u] - 1);  // 0 goes last
      hi = max(hi, k[u]);
    }
  }
  lo = ~wave_max(~lo);
  hi = wave_max(hi);
  if (lane == 0) {
    wlo[w] = lo;
    whi[w] = hi;
  }
  lds_barrier();
  lo = ~row_max(~wlo[lane % NW]) + 1;
  hi = row_max(whi[lane % NW]);
  // `need` of the keys in [lo, hi] are taken, all above and none below
  int m = min(l - f, PICK_CAND + 1);
  for (int round = 0; round < 4 && lo < hi && m > PICK_CAND; ++round) {  // 32 -> 22 -> 12 -> 2 -> 0 bits
    const int shift = max(0, 32 - __clz((int)(hi - lo)) - 10);
    for (int c = f; c < l; c += STEP) {
      if (many) fetch(c);
#pragma unroll
      for (int u = 0; u < UN; ++u)
        if (k[u] >= lo && k[u] <= hi) atomicAdd(&hist[(k[u] - lo) >> shift], 1);
    }
    lds_barrier();
    const int bin = PICK_BINS - 1 - tid, here = hist[bin];  // thread t holds bin t from the top
    int before = wave_scan(here);
    if (lane == 63) sums[w] = before;
    lds_barrier();
    before -= here;
    const int waves = row_scan(sums[lane % NW]);
    if (w > 0) before += __builtin_amdgcn_readlane(waves, w - 1);
    if (before < need && need <= before + here) {  // one thread
      s_m = here;
      s_need = need - before;
      s_lo = lo + ((uint32_t)bin << shift);
      s_hi = s_lo + min(hi - s_lo, (1u << shift) - 1);
    }
    hist[bin] = 0;
    lds_barrier();
    lo = s_lo;
    hi = s_hi;
    need = s_need;
    m = s_m;
  }
  const unsigned long long lower = (1ull << lane) - 1;
  if (lo < hi) {  // m (at most PICK_CAND) keys: each counts what lies above it
    for (int c = f; c < l; c += STEP) {
      if (many) fetch(c);
      int hits = 0, at = 0;
#pragma unroll
      for (int u = 0; u < UN; ++u) hits += __popcll(__ballot(k[u] >= lo && k[u] <= hi));
      if (hits == 0) continue;
      if (lane == 0) at = atomicAdd(&s_cand, hits);
      at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const bool in = k[u] >= lo && k[u] <= hi;
        const unsigned long long mask = __ballot(in);
        if (in) cand[min(at + (int)__popcll(mask & lower), PICK_CAND - 1)] = k[u];
        at += __popcll(mask);
      }
    }
    lds_barrier();
    m = min(m, PICK_CAND);
    // 64 keys a group, the waves of a group share what they are compared with
    const int gs = m <= 64 ? 0 : 1, group = w & ((1 << gs) - 1), part = w >> gs, parts = NW >> gs;
    static_assert(PICK_CAND == 128, "at most two groups");
    const uint32_t c = cand[group * 64 + lane];
    int gt = 0, ge = 0;
#pragma unroll 2
    for (int i = 4 * part; i < m; i += 4 * parts) {
      const u4 x = *reinterpret_cast<const u4*>(&cand[i]);  // 0 past the last: above no key
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        gt += x[e] > c;
        ge += x[e] >= c;
      }
    }
    atomicAdd(&above[group * 64 + lane], gt);
    atomicAdd(&upto[group * 64 + lane], ge);
    lds_barrier();
    if (tid < m && above[tid] < need && need <= upto[tid]) {  // equal keys write the same
      s_lo = cand[tid];
      s_want = need - above[tid];
    }
    lds_barrier();
    lo = s_lo;
    need = s_want;
  }
  // keys above lo, and the first `need` of those equal to it: counted for 64 blocks, their places by the sums over those before
  int pg = 0, pe = 0;
  for (int c = f; c < l; c += STEP) {
    if (many) fetch(c);
    int mine = 0;  // lane u: the numbers of u, 16 bits each
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int g = __popcll(__ballot(k[u] > lo)), e = __popcll(__ballot(k[u] == lo));
      if (lane == u) mine = g | e << 16;
    }
    if (c > f) lds_barrier();  // the counts before have been read
    if (lane < UN) counts[lane * NW + w] = mine;
    lds_barrier();
    int x[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      x[i] = lane * PER + i < UN * NW ? counts[lane * PER + i] : 0;
      sum += x[i];
    }
    const int incl = wave_scan(sum);
    int start = incl - sum;  // of this wave's count among a lane's
#pragma unroll
    for (int i = 0; i + 1 < PER; ++i) start += i < w % PER ? x[i] : 0;
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int s0 = __builtin_amdgcn_readlane(start, (u * NW + w) / PER);
      const unsigned long long gt = __ballot(k[u] > lo), eq = __ballot(k[u] == lo);
      const int g = pg + (s0 & 0xFFFF) + (int)__popcll(gt & lower), e = pe + (s0 >> 16) + (int)__popcll(eq & lower), at = f + g + min(e, need);
      if ((k[u] > lo || (k[u] == lo && e < need)) && at < ch.take) out[at] = c + tid + u * NT;
    }
    const int total = __builtin_amdgcn_readlane(incl, 63);
    pg += total & 0xFFFF;
    pe += total >> 16;
  }
}

// ---------------------------------------------------------------- attention
// bf16 planes of an fp32 operand: v = p0 + p1 (+ p2), 16 or 24 significant bits.  Queries have the planes of the model's
// activations, two where those are pairs and three in fp32: nothing of them is lost, as codes are exact in bf16.
template <typename T> struct Planes;
template <> struct Planes<bf16> { static constexpr int N = 2; };
template <> struct Planes<float> { static constexpr int N = 3; };

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

// eight e4m3 codes as bf16 (exact)
__device__ __forceinline__ u4 codes_bf16(uint32_t a, uint32_t b) {
  return u4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true))};
}

// A block in registers: 16 bytes a lane of each 1 KB piece.  Range-checked loads, so that a loop of them has no branches
// (blk < 0: nothing is read, the block is zeros): the compiler then waits for the half that it needs and not for what is
// behind it.  The next block's K is loaded as soon as this one's is used up, its V likewise: half a block is always on its
// way, with one set of registers and one copy of the code (a call's first pass fetches every instruction from memory).
template <int HD>
struct CodeBlock {
  u4 k[2][HD / 64], v[HD / 32];
  float ks, vs;  // by vector loads: a scalar load on its way would be waited for with every read of LDS
  __device__ __forceinline__ void load_k(const uint8_t* codes, const float* scales, int blk) {
    const BufRsrc rs = buf_rsrc(codes + (size_t)max(blk, 0) * (2 * KV8_BLOCK * HD), blk < 0 ? 0 : 2 * KV8_BLOCK * HD);
    ks = buf_f1(buf_rsrc(scales + 2 * (size_t)max(blk, 0), blk < 0 ? 0 : 8), 0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < HD / 64; ++i) k[t][i] = buf_u4_stream(rs, (threadIdx.x & 63) * 16 + (t * (HD / 64) + i) * 1024);
    __builtin_amdgcn_sched_barrier(0);  // the loads stay in this order: the wait for K must not cover V
  }
  __device__ __forceinline__ void load_v(const uint8_t* codes, const float* scales, int blk) {
    const BufRsrc rs = buf_rsrc(codes + (size_t)max(blk, 0) * (2 * KV8_BLOCK * HD), blk < 0 ? 0 : 2 * KV8_BLOCK * HD);
    vs = buf_f1(buf_rsrc(scales + 2 * (size_t)max(blk, 0), blk < 0 ? 0 : 8), 4);
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) v[i] = buf_u4_stream(rs, (threadIdx.x & 63) * 16 + KV8_BLOCK * HD + i * 1024);
    __builtin_amdgcn_sched_barrier(0);
  }
};

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
// Scores of the 16 query rows against the block (lane: row r, slots 8 g ..), the softmax update of (m, l, o) in base 2, and
// P V; then x holds block `next`.  q: fragments in LDS (registers would not do for four waves a SIMD).  `scale` is log2(e) /
// sqrt(hd).  m is that of the row in all four lane groups, l this lane's slots alone.  LIST: a block that is not `there`
// (zeros) counts for nothing.  SPARE > 0: the operand rows from SPARE on repeat the queries of those before, and take the
// third plane of their weights in the first product.
template <int HD, int N, bool LIST, int SPARE>
__device__ __forceinline__ void attend_block(CodeBlock<HD>& x, const u4 (*q)[64], float scale, float& m, float& l, f4* o,
                                             const uint8_t* codes, const float* scales, int next, bool there) {
  float sc[8];
  const float c = LIST && !there ? 0.f : x.ks * scale, none = LIST && !there ? -INFINITY : 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    f4 s = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < HD / 64; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u4 k = codes_bf16(x.k[t][i][2 * h], x.k[t][i][2 * h + 1]);
#pragma unroll
        for (int n = 0; n < N; ++n) Frag<bf16>::mma(s, k, q[(2 * i + h) * N + n][threadIdx.x & 63]);
      }
#pragma unroll
    for (int e = 0; e < 4; ++e) sc[4 * t + e] = s[e];
  }
  x.load_k(codes, scales, next);
  float top = sc[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[e]);
  top = top * c + none;  // c is not negative
  if (__any(top > m)) {  // rarely, once a row has seen many keys
    const float mnew = fmaxf(m, group_max(top));
    const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mnew);
    l *= alpha;
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float ai = __shfl(alpha, 4 * g + i, WAVE);
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d][i] *= ai;
    }
    m = mnew;
  }
  const float mz = none - (m == -INFINITY ? 0.f : m);  // scores of -inf alone: all weights 0
  float p[8];
  const float vs = LIST && !there ? 0.f : x.vs;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], c, mz));
    l += p[e];
    p[e] *= vs;
  }
  u4 pp[3];
  to_planes<3>(p, pp);
  if constexpr (SPARE > 0) {
    const bool third = threadIdx.x & SPARE;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pp[0][i] = third ? pp[2][i] : pp[0][i];
      pp[1][i] = third ? 0u : pp[1][i];
    }
  }
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u4 v = codes_bf16(x.v[i][2 * h], x.v[i][2 * h + 1]);
#pragma unroll
      for (int n = 0; n < (SPARE > 0 ? 2 : 3); ++n) Frag<bf16>::mma(o[2 * i + h], pp[n], v);
    }
  x.load_v(codes, scales, next);
}

// Waves of a workgroup: two a SIMD, and two workgroups a CU (four waves of 128 registers) for a bf16 model with up to 8 q-heads a
// kv head.  At head dim 128 one workgroup a CU with 16 (93 KB of LDS) and in fp32 (140 registers and more).  A SIMD takes its
// waves' blocks one after the other, the oldest wave first (0.6 us a block at head dim 128), so a few blocks want many CUs:
// 4 rows x 64 listed blocks 12.9 us with 16 waves, 10.4 with 8, 1 x 4,096 slots 10.5 and 8.4, 4 x 33,300 45.8 and 45.3.
constexpr int ATT_WAVES = 8;
template <int HD, int GR, int N>
struct AttLds {
  static constexpr int NW = ATT_WAVES;
  u4 qf[HD / 32 * N][64];                      // query fragments, channels in the order of the K codes
  union {
    float o[NW][GR][HD];
    float q[GR][HD];                           // queries for the open block, done with before the main loop ends
  };
  float m[NW][16], l[NW][16];
  float v[KV8_BLOCK][HD], p[GR][KV8_BLOCK];    // values and weights of the open block
  float tm[GR], tl[GR];                        // its maxima and sums; in the end its factors, and the sums of all
  float top[GR];
};

// One workgroup per (split, kv head, row).  Wave w of NW of split s takes the blocks (or list entries) NW s + w, NW
// (s + nsplit) + w, ...: which block is first depends on nothing in memory, so its loads are under way before the row's
// length is known (a cache holds blocks up to kv_max, whatever the length), and rows of any length are shared evenly.  Split
// 0 attends over the open block too, in fp32 on the vector units (at most 31 slots), while its first blocks are on their way.
// A wave's block is 64 conversions and 32 matrix instructions among 290 at head dim 128, for 8.2 KB.  8 kv heads of 128, 4
// q-heads each, bf16: 4 rows x 33,300 slots 45 us and 32 x 2,560 28 (6.0 TB/s; memory); 4 rows x 64 listed blocks 7.8 and
// 1 x 700 slots of 8 heads of 64 7.0 (latency: arguments, length or list, blocks, softmax, the waves' sums).
template <typename T, int HD, int GR, bool LIST>
__global__ __launch_bounds__(64 * ATT_WAVES, Act<T>::SPLIT ? 4 : 2) void k_kv8_attn(Kv8AttnArgs a) {
  constexpr int N = Planes<T>::N, NF = HD / 32, ND = HD / 16, B = KV8_BLOCK, PL = Act<T>::PL;
  // the weights' third plane (24 significant bits; with 16 the outputs were 3 times as far off) shares the first one's product
  // where a bf16 model's queries leave half of the 16 operand rows
  constexpr int SPARE = N == 2 && GR < 16 ? GR : 0;
  constexpr int NW = ATT_WAVES, THREADS = 64 * NW, LPS = THREADS / B, CPL = HD / LPS;  // open block: lanes of a slot, channels a lane
  constexpr int OUT = (GR * HD + THREADS - 1) / THREADS;  // outputs of a thread
  __shared__ AttLds<HD, GR, N> sh;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g = lane >> 4;
  const int split = blockIdx.x, kvh = blockIdx.y, r = blockIdx.z, grp = a.grp;
  const size_t pair = (size_t)r * a.Hk + kvh;
  const int first = split * NW + w, stride = a.nsplit * NW;
  const uint8_t* codes = a.c.codes + pair * a.c.NB * (2 * B * HD);
  const float* scales = a.c.scales + pair * a.c.NB * 2;
  const int* list = LIST ? a.blocks + pair * a.max_blocks : nullptr;
  int blk = -1, before = -1;  // this lane's list entry and the one before it
  if constexpr (LIST) {
    const int e = first + lane * stride;
    if (e < a.max_blocks) {
      blk = list[e];
      if (e > 0) before = list[e - 1];
    }
  }
  int n = a.kv_len[r], cnt = LIST ? a.n_blocks[pair] : 0;
  const int on = a.enable[r];
  // this thread's share of the open block: slot ts, channels tc ..
  const int ts = tid / LPS, tc = tid % LPS * CPL;
  static_assert(GR * HD / 4 <= THREADS, "four query channels a thread");
  static_assert(LPS == 16, "row_sum adds up the lanes of a slot");
  Raw<T, CPL> tk, tv;
  Raw<T, 4> tq[PL];
  const T* qrow = (const T*)a.q + (size_t)r * PL * a.H * HD + kvh * grp * HD;  // hi plane of the kv head's q-heads
  if (split == 0) {
    const T* op = (const T*)a.c.open + pair * 2 * B * HD + ts * HD + tc;
    tk.load(op);
    tv.load(op + B * HD);
    if (tid * 4 < grp * HD) {
#pragma unroll
      for (int i = 0; i < PL; ++i) tq[i].load(qrow + i * a.H * HD + tid * 4);
    }
  }
  // query fragments: fragment f = 2 i + h holds channels 64 i + 16 g + 8 h ..; one or more a wave.  Rows past the q-heads of
  // the kv head are out of the buffer's range, which loads zeros.
  constexpr int QL = (int)sizeof(T) / 2;  // 16-byte loads of 8 channels
  constexpr int FRAGS = Act<T>::SPLIT ? NF * PL : NF;
  static_assert(FRAGS <= NW, "a fragment a wave");
  const int qf = Act<T>::SPLIT ? w / PL : w, plane = Act<T>::SPLIT ? w % PL : 0;
  u4 raw[QL];
  if (w < FRAGS) {
    const BufRsrc qs = buf_rsrc(qrow + (size_t)plane * a.H * HD, grp * HD * (int)sizeof(T));
    const uint32_t qo = ((SPARE > 0 && r16 < 2 * SPARE ? r16 % (SPARE > 0 ? SPARE : 1) : r16) * HD + 64 * (qf / 2) + 16 * g + 8 * (qf % 2)) * (uint32_t)sizeof(T);
#pragma unroll
    for (int j = 0; j < QL; ++j) raw[j] = buf_u4(qs, qo + 16 * j);
  }
  CodeBlock<HD> x;
  if constexpr (!LIST) {
    const int b0 = first < a.kv_max / B ? first : -1;
    x.load_k(codes, scales, b0);
    x.load_v(codes, scales, b0);
  }
  if (n < 0 || n > a.kv_max) {
    if (split == 0 && kvh == 0 && tid == 0) atomicOr(a.err + r, 8);
    n = 0;
  }
  if (!on) n = 0;
  const int closed = n / B, rest = split == 0 ? n % B : 0;
  if (!LIST || n == 0) {
    cnt = closed;
  } else if (cnt < 0 || cnt > a.max_blocks) {
    if (split == 0 && tid == 0) atomicOr(a.err + r, 16);
    cnt = 0;
  }
  int mine = 0;  // list entries among the wave's next 64
  const auto check_entries = [&](int e0) {  // an entry that is not ascending or out of range is left out
    const bool there = e0 + lane * stride < cnt;
    mine = __popcll(__ballot(there));
    if (there && (blk < 0 || blk <= before || blk >= closed)) {
      atomicOr(a.err + r, 16);
      blk = -1;
    }
  };
  if constexpr (LIST) {
    check_entries(first);
    asm volatile("" : "+v"(blk));
    const int b0 = mine > 0 ? __builtin_amdgcn_readlane(blk, 0) : -1;
    x.load_k(codes, scales, b0);
    x.load_v(codes, scales, b0);
  }
  const float scale = 1.4426950408889634f / sqrtf((float)HD);
  if (w < FRAGS) {
    if constexpr (Act<T>::SPLIT) {
      sh.qf[w][lane] = raw[0];
    } else {
      float v[8];
      u4 pl[N];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(raw[e / 4][e % 4]);
      to_planes<N>(v, pl);
#pragma unroll
      for (int i = 0; i < N; ++i) sh.qf[w * N + i][lane] = pl[i];
    }
  }
  if (rest > 0) {
    if (tid * 4 < grp * HD) {
#pragma unroll
      for (int e = 0; e < 4; ++e) (&sh.q[0][0])[tid * 4 + e] = PL == 1 ? tq[0].at(e) : tq[0].at(e) + tq[PL - 1].at(e);
    }
#pragma unroll
    for (int e = 0; e < CPL; ++e) sh.v[ts][tc + e] = ts < rest ? tv.at(e) : 0.f;  // what lies past the row's end may be NaN
  }
  lds_barrier();
  float tx[OUT];  // the open block's part of this thread's outputs
  if (rest > 0) {
    for (int j = 0; j < grp; ++j) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < CPL; ++e) s += sh.q[j][tc + e] * tk.at(e);
      s = row_sum(s);
      if (tid % LPS == 0) sh.p[j][ts] = ts < rest ? s * scale : -INFINITY;
    }
    lds_barrier();
    for (int j = w; j < grp; j += NW) {  // weights, 32 slots twice in a wave
      const float s = sh.p[j][lane % B];
      const float top = group_max(row_max(s)), mz = top == -INFINITY ? 0.f : top;
      const float p = __builtin_amdgcn_exp2f(s - mz);
      const float sum = group_sum(row_sum(p)) * 0.5f;
      if (lane < B) sh.p[j][lane] = p;
      if (lane == 0) {
        sh.tm[j] = top;
        sh.tl[j] = sum;
      }
    }
    lds_barrier();
#pragma unroll
    for (int k = 0; k < OUT; ++k) {
      const int t = tid + k * THREADS, j = t / HD, d = t % HD;
      tx[k] = 0.f;
      if (j >= grp) break;
#pragma unroll 4
      for (int i = 0; i < B; i += 4) {
        const f4 p = *reinterpret_cast<const f4*>(&sh.p[j][i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) tx[k] += p[e] * sh.v[i + e][d];
      }
    }
  }
  f4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  if constexpr (!LIST) {
    for (int e = first; e < cnt; e += stride)
      attend_block<HD, N, false, SPARE>(x, sh.qf, scale, m, l, o, codes, scales, e + stride < cnt ? e + stride : -1, true);
  } else {
    for (int e0 = first; e0 < cnt; e0 += 64 * stride) {  // 64 of the wave's entries at a time: one a lane
      if (e0 > first) {
        const int e = e0 + lane * stride;
        blk = -1;
        if (e < cnt) {
          blk = list[e];
          before = list[e - 1];
        }
        check_entries(e0);
        asm volatile("" : "+v"(blk));  // waited for here, not with blocks under way
        const int b0 = __builtin_amdgcn_readlane(blk, 0);
        x.load_k(codes, scales, b0);
        x.load_v(codes, scales, b0);
      }
      for (int j = 0; j < mine; ++j) {
        const int next = j + 1 < mine ? __builtin_amdgcn_readlane(blk, j + 1) : -1;
        attend_block<HD, N, true, SPARE>(x, sh.qf, scale, m, l, o, codes, scales, next, __builtin_amdgcn_readlane(blk, j) >= 0);
      }
    }
  }
  if constexpr (SPARE > 0) {  // rows r and r + SPARE belong together: lanes 16 apart for 4 rows, 32 for 8
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[d][i] = SPARE == 4 ? pair16_sum(o[d][i]) : pair32_sum(o[d][i]);
  }
  // per wave: maximum, sum and unnormalised outputs
  l = group_sum(l);
  if (g == 0) {
    sh.m[w][r16] = m;
    sh.l[w][r16] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = 4 * g + i;
    if (j < grp) {
#pragma unroll
      for (int d = 0; d < ND; ++d) sh.o[w][j][d * 16 + r16] = o[d][i];
    }
  }
  lds_barrier();
  if (tid < 16 * GR) {  // 16 lanes a head: the waves' factors, once
    const int j = tid / 16, i = tid % 16;
    const float mi = i < NW ? sh.m[i % NW][j] : -INFINITY, li = i < NW ? sh.l[i % NW][j] : 0.f;
    const float tm = rest > 0 ? sh.tm[j] : -INFINITY, tl = rest > 0 ? sh.tl[j] : 0.f;
    const float M = fmaxf(row_max(mi), tm), mz = M == -INFINITY ? 0.f : M;
    // 0 for a wave without slots; one whose scores are all NaN has maximum -inf and sum NaN, which the factor 0 keeps
    const float e = __builtin_amdgcn_exp2f(mi - mz), et = __builtin_amdgcn_exp2f(tm - mz);
    const float L = row_sum(e * li) + et * tl;
    if (i < NW) sh.m[i][j] = e;
    if (i == 0) {
      sh.tm[j] = et;
      sh.tl[j] = L;
      sh.top[j] = M;
    }
  }
  lds_barrier();
#pragma unroll
  for (int k = 0; k < OUT; ++k) {
    const int t = tid + k * THREADS, j = t / HD, d = t % HD;
    if (j >= grp) break;
    const float L = sh.tl[j];
    float out = rest > 0 ? sh.tm[j] * tx[k] : 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) out += sh.m[i][j] * sh.o[i][j][d];
    if (a.nsplit == 1) {
      Act<T>::put(a.out, r, a.H * HD, (kvh * grp + j) * HD + d, L == 0.f ? 0.f : out / L);
    } else {
      const size_t rec = (pair * a.nsplit + split) * grp + j;
      a.part[rec * HD + d] = out;
      if (d == 0) {
        float* ml = a.part + (size_t)a.R * a.H * a.nsplit * HD + 2 * rec;
        ml[0] = sh.top[j];
        ml[1] = L;
      }
    }
  }
}

// Log-sum-exp combine of the splits of one (row, q-head), in split order.  The outputs are on their way while the weights
// are formed: one round trip to memory, which with the launch is most of its time (4 x 32 heads of 128, 6 or 8 splits: 2.0 to
// 4.6 us).
constexpr int COMB_THREADS = 256;
template <typename T, int HD>
__global__ __launch_bounds__(COMB_THREADS) void k_kv8_combine(Kv8AttnArgs a) {
  constexpr int G = COMB_THREADS / HD, UN = 8;
  __shared__ float wts[64];
  __shared__ float acc[COMB_THREADS];
  const int j = blockIdx.x, kvh = blockIdx.y, r = blockIdx.z, tid = threadIdx.x, lane = tid & 63, ns = a.nsplit, grp = a.grp;
  const size_t rec0 = ((size_t)r * a.Hk + kvh) * ns * grp + j;  // record of split s: rec0 + s * grp
  const int d = tid % HD, sg = tid / HD;
  float v[UN];
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    const int s = sg + u * G;
    v[u] = s < ns ? a.part[(rec0 + (size_t)s * grp) * HD + d] : 0.f;
  }
  if (tid < 64) {
    float ms = -INFINITY, ls = 0.f;
    if (lane < ns) {
      const float* ml = a.part + (size_t)a.R * a.H * ns * HD + 2 * (rec0 + (size_t)lane * grp);
      ms = ml[0];
      ls = ml[1];
    }
    const float M = group_max(row_max(ms)), mz = M == -INFINITY ? 0.f : M;
    const float e = __builtin_amdgcn_exp2f(ms - mz);
    const float L = group_sum(row_sum(e * ls));
    wts[lane] = L == 0.f ? 0.f : e / L;
  }
  lds_barrier();
  float o = 0.f;
#pragma unroll
  for (int u = 0; u < UN; ++u)
    if (sg + u * G < ns) o += wts[sg + u * G] * v[u];
  for (int s = sg + UN * G; s < ns; s += G) o += wts[s] * a.part[(rec0 + (size_t)s * grp) * HD + d];
  acc[tid] = o;
  lds_barrier();
  if (tid < HD) {
    float x = acc[tid];
#pragma unroll
    for (int i = 1; i < G; ++i) x += acc[i * HD + tid];
    Act<T>::put(a.out, r, a.H * HD, (kvh * grp + j) * HD + tid, x);
  }
}

template <typename T, int HD>
int append_t(const Kv8AppendArgs& a, Stream s) {
  const int nb = (a.T + 31) / 32;
  const unsigned steps = (unsigned)((((long long)a.R * nb + 7) / 8) * 8);
  launch_k((k_kv8_append<T, HD>), dim3(steps * a.Hk * (a.q ? 2 : 1)), dim3(2 * HD), 0, s, a, nb);
  return 0;
}
template <typename T, int HD>
int pack_t(const Kv8PackArgs& a, Stream s) {
  launch_k((k_kv8_pack<T, HD>), dim3(std::max(1, (a.kv_max + KV8_BLOCK - 1) / KV8_BLOCK), a.Hk, a.R), dim3(2 * HD), 0, s, a);
  return 0;
}
template <typename T, int HD>
int select_t(const Kv8SelectArgs& a, Stream s) {
  const int nb = a.kv_max / KV8_BLOCK;
  if (nb <= PICK_FEW && nb > 0) {
    launch_k(nb <= 128 ? k_kv8_pick_few<T, HD, 128> : k_kv8_pick_few<T, HD, PICK_FEW>, dim3(a.Hk, a.R), dim3(nb <= 128 ? 512 : 768), 0, s, a, nb);
    return 0;
  }
  if (nb > a.n) {
    // one block a lane group while that leaves a SIMD no more than two waves: 1 row x 256 blocks 7.5 us, 8.2 with 64 a workgroup;
    // 8 rows x 1,040 17.7, 14.5 with 64
    const int per = (long long)nb * a.Hk * a.R <= 512 * SCORE_NW * (512 / HD) ? SCORE_NW * (512 / HD) : SCORE_BLOCKS;
    launch_k((k_kv8_scores<T, HD>), dim3((nb + per - 1) / per, a.Hk, a.R), dim3(64 * SCORE_NW), 0, s, a, nb, per);
  }
  // the least that holds the row: 1,040 blocks in 2 keys a thread 11.7 us, in 16 18.8; 4 x 4,096 in 4 20.6, in 8 21.8, in 16 27.0
  launch_k(nb <= 2048 ? k_kv8_pick<2> : nb <= 4096 ? k_kv8_pick<4> : nb <= 8192 ? k_kv8_pick<8> : k_kv8_pick<16>, dim3(a.Hk, a.R), dim3(1024), 0, s, a, nb);
  return 0;
}
template <typename T, int HD>
int attention_t(const Kv8AttnArgs& a, Stream s) {
  const auto kernel = [&](auto list) {
    constexpr bool LIST = decltype(list)::value;
    return a.grp <= 4 ? k_kv8_attn<T, HD, 4, LIST> : a.grp <= 8 ? k_kv8_attn<T, HD, 8, LIST> : k_kv8_attn<T, HD, 16, LIST>;
  };
  launch_k(a.blocks ? kernel(std::true_type{}) : kernel(std::false_type{}), dim3(a.nsplit, a.Hk, a.R), dim3(64 * ATT_WAVES), 0, s, a);
  if (a.nsplit > 1) launch_k((k_kv8_combine<T, HD>), dim3(a.grp, a.Hk, a.R), dim3(COMB_THREADS), 0, s, a);
  return 0;
}

#define KV8_DISPATCH(fn)                                                    \
  do {                                                                      \
    if (hd == 64) return dtype == 1 ? fn<bf16, 64>(a, s) : fn<float, 64>(a, s);    \
    if (hd == 128) return dtype == 1 ? fn<bf16, 128>(a, s) : fn<float, 128>(a, s); \
    return -1;                                                              \
  } while (0)

}  // namespace

int launch_kv8_append(int dtype, int hd, const Kv8AppendArgs& a, Stream s) { KV8_DISPATCH(append_t); }
int launch_kv8_pack(int dtype, int hd, const Kv8PackArgs& a, Stream s) { KV8_DISPATCH(pack_t); }
int launch_kv8_select(int dtype, int hd, const Kv8SelectArgs& a, Stream s) { KV8_DISPATCH(select_t); }
int launch_kv8_attention(int dtype, int hd, const Kv8AttnArgs& a, Stream s) { KV8_DISPATCH(attention_t); }

}  // namespace ham
