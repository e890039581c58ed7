// Operators on a paged KV cache (layout: kernels_paged.h; bf16 prompts: kernels_paged_prompt.hip).
//
// k_paged_append    RoPE of packed projection rows, K and V into the rows' pages, q out.
// k_paged_attn      attention of up to 16 query rows that share a kv head over their row's pages: the q-heads of one new token
//                   of each sequence, or 16 (token, q-head) pairs of packed rows; k_paged_join joins its splits.
// k_paged_take, k_paged_give, k_paged_copy  rows take over other rows' pages, give up theirs, get new ones; pages that two rows
//                   share are copied before one writes to them.
// k_paged_compact   pages in use to the front of the pool (k_paged_copy moves them).
#include <algorithm>

#include "launch_rules.h"
#include "paged_device.h"

namespace ham {

namespace {

// ---------------------------------------------------------------- append
// A step is 32 slots (aligned) of a row that get new tokens.  For each step and kv head one workgroup writes K and V and, if
// q is wanted, another rotates its q-heads (with many rows a workgroup takes several of these in turn, paged_append_groups); those
// of a step run on one XCD, whose L2 then holds the step's RoPE factors.
// Bound by memory.  K: a thread has 8 RoPE pairs of a slot, so that 16 lanes write 256 bytes and 4 read 128.  V: a thread has a
// channel of the E slots that lie together; at the ends of the new tokens, where some of them are others', values one by one.
__device__ __forceinline__ int append_count(const PagedAppendArgs& a, int r) {  // -1: does not fit
  const int c = packed_count(a.offsets, r, a.N), s = a.start[r];
  return s >= 0 && (long long)s + c <= (long long)a.z.row_pages << a.z.lgP ? c : -1;
}
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_append(PagedAppendArgs a) {
  constexpr int HALF = HD / 2, E = 16 / (int)sizeof(T), B = 32;
  const PagedSizes& z = a.z;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, heads = (a.q ? 2 : 1) * z.Hk;
  const uint32_t s8 = blockIdx.x / 8, step = s8 / (uint32_t)a.per_step * 8 + blockIdx.x % 8;
  if (blockIdx.x == 0)
    for (int r = tid; r < z.R; r += 256)
      if (append_count(a, r) < 0) atomicOr(a.err + r, 8);
  __shared__ int scratch[10];
  const Share sh = find_share<256>(z.R, (int)step, scratch, [&](int r) {
    const int c = append_count(a, r), s = a.start[r];
    return c > 0 ? (s + c - 1) / B - s / B + 1 : 0;
  });
  if (sh.r < 0) return;
  const int r = sh.r, o = a.offsets[r], c = a.offsets[r + 1] - o, s0 = a.start[r];
  const int base = (s0 / B + sh.at) * B, lo = max(base, s0), hi = min(base + B, s0 + c);  // slots [lo, hi)
  const size_t ld = (size_t)(z.H + 2 * z.Hk) * HD;
  const size_t tok = (size_t)o - s0;  // packed row of slot 0
  for (int head = (int)(s8 % (uint32_t)a.per_step); head < heads; head += a.per_step) {
    const int kvh = head % z.Hk;
    if (head >= z.Hk) {  // q
      const int items = (hi - lo) * z.grp * (HALF / 8);
      for (int q = tid; q < items; q += 256) {
        const int i = q % (HALF / 8) * 8, hq = q / (HALF / 8), h = kvh * z.grp + hq % z.grp;
        const size_t t = tok + lo + hq / z.grp;
        const float* p = a.qkv + t * ld + h * HD + i;
        f4 x[2], y[2], cs[2], sn[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          x[u] = *reinterpret_cast<const f4*>(p + 4 * u);
          y[u] = *reinterpret_cast<const f4*>(p + HALF + 4 * u);
          cs[u] = *reinterpret_cast<const f4*>(a.cos + t * HALF + i + 4 * u);
          sn[u] = *reinterpret_cast<const f4*>(a.sin + t * HALF + i + 4 * u);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) rotate(x[u], y[u], cs[u], sn[u]);
        put_act8<T>(a.q, t, z.H * HD, h * HD + i, x);
        put_act8<T>(a.q, t, z.H * HD, h * HD + i + HALF, y);
      }
      continue;
    }
    const int* table = a.table + (size_t)r * z.row_pages;
    const int P = 1 << z.lgP;
    const size_t run = (size_t)P * HD;  // K, or V, of a kv head in a page
    // where slot s's page holds the kv head, or null
    const auto place = [&](int s) -> T* {
      const int id = table[s >> z.lgP];
      if ((unsigned)id >= (unsigned)z.n_pages) {
        atomicOr(a.err + r, 32);
        return nullptr;
      }
      return (T*)a.pool + ((size_t)id * z.Hk + kvh) * 2 * run;
    };
    const float* ksrc = a.qkv + (size_t)(z.H + kvh) * HD;
    const float* vsrc = ksrc + (size_t)z.Hk * HD;
    {
      const int s = base + (w & 1) * 16 + (lane & 15), i = ((w >> 1) * 4 + (lane >> 4)) * 8;
      if (i < HALF && s >= lo && s < hi) {
        const size_t t = tok + s;
        f4 x[2], y[2], cs[2], sn[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          x[u] = *reinterpret_cast<const f4*>(ksrc + t * ld + i + 4 * u);
          y[u] = *reinterpret_cast<const f4*>(ksrc + t * ld + HALF + i + 4 * u);
          cs[u] = *reinterpret_cast<const f4*>(a.cos + t * HALF + i + 4 * u);
          sn[u] = *reinterpret_cast<const f4*>(a.sin + t * HALF + i + 4 * u);
        }
        T* out = place(s);
#pragma unroll
        for (int u = 0; u < 2; ++u) rotate(x[u], y[u], cs[u], sn[u]);
        if (out != nullptr) {
          const int at = s & (P - 1);
#pragma unroll
          for (int u = 0; u < 8; u += 4) {  // of 8 channels that lie together (fp32: 4 and 4)
            st4<T>(out + paged_k_index<E>(at, i + u, HD), x[u / 4]);
            st4<T>(out + paged_k_index<E>(at, HALF + i + u, HD), y[u / 4]);
          }
        }
      }
    }
    for (int q = tid; q < B / E * HD; q += 256) {
      const int d = q % HD, s = base + q / HD * E;  // slots s .. s + E - 1, in one page
      if (s + E <= lo || s >= hi) continue;
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = s + e >= lo && s + e < hi ? vsrc[(tok + s + e) * ld + d] : 0.f;
      T* out = place(max(s, lo));
      if (out == nullptr) continue;
      out += run + paged_v_index<E>(s & (P - 1), d, HD);
      if (s >= lo && s + E <= hi) {
        u4 x;
        if constexpr (E == 8) x = pack_frag_bf16(v);
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = __float_as_uint(v[e]);
        *reinterpret_cast<u4*>(out) = x;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (s + e >= lo && s + e < hi) out[e] = from_f<T>(v[e]);
      }
    }
  }
}

// ---------------------------------------------------------------- attention
// A block of B slots (32 in bf16, 16 in fp32) in registers, as operands of 16-row products: K row r of product t (16 slots
// each, hd in pieces of 4 E channels), V^T row d (all B slots).  ka and kb are its first and (bf16) second 16 slots.
template <typename T, int HD> struct KvBlock {
  static constexpr int E = 16 / (int)sizeof(T), B = 4 * E, KT = B / 16, NF = HD / (4 * E), ND = HD / 16;
  u4 k[KT][NF], v[ND];
  // STREAM: read once, past the caches, or the 256 MB of the last one keep what no one reads again (4 x 33,300 slots 89 us without)
  template <bool STREAM> static __device__ __forceinline__ u4 ld(const char* p) {
    if constexpr (STREAM) return ld16_stream(p);
    else return ld16(p);
  }
  // !there: nothing is wanted; the pool's first bytes, which no loop of these loads then needs a branch for
  template <bool STREAM> __device__ __forceinline__ void load_k(const char* ka, const char* kb, bool there, const char* pool) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const char* p;
    if constexpr (KT == 2) p = (r & 8 ? kb : ka) + (g * 16 + (r & 7)) * 16;
    else p = ka + (g * 16 + r) * 16;
    p = there ? p : pool;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int f = 0; f < NF; ++f) k[t][f] = ld<STREAM>(p + (4 * f * 16 + 8 * t) * 16);
  }
  template <bool STREAM> __device__ __forceinline__ void load_v(const char* va, const char* vb, bool there, const char* pool) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const char* p;
    if constexpr (KT == 2) p = (g & 2 ? vb : va) + ((g & 1) * HD + r) * 16;
    else p = va + (((g & 1) << 1 | g >> 1) * HD + r) * 16;
    p = there ? p : pool;
#pragma unroll
    for (int d = 0; d < ND; ++d) v[d] = ld<STREAM>(p + d * 256);
  }
};
// first slot, within a block, of the E that lane group g has
template <typename T> __device__ __forceinline__ int lane_slot(int g) {
  return sizeof(T) == 2 ? 8 * g : 4 * ((g & 1) << 1 | g >> 1);
}

// Waves of a workgroup take blocks in turn; queries and the softmax of a column (16 of them: lane l & 15) are fp32, weights
// three bf16 planes (24 significant bits), queries the two of an activation row, or all fp32.
constexpr int PATT_WAVES = 4;
template <int HD> struct PattLds {
  float o[PATT_WAVES][16][HD + 4];
  float m[PATT_WAVES][16], l[PATT_WAVES][16];
  float top[16], sum[16];
};

// The slots of a row that are attended over; a length out of range is reported by one thread.
__device__ __forceinline__ int slots_of(const PagedAttnArgs& a, int r, bool report) {
  const int n = a.kv_len[r];
  if (n < 0 || n > a.kv_max) {
    if (report) atomicOr(a.err + r, 8);
    return 0;
  }
  return a.enable[r] ? n : 0;
}
// One row per sequence, split: the blocks of all rows in about a.nsplit shares of the same size, so that a long row among short
// ones has many workgroups.  Of row r they are shares `first` .. `first` + `of` - 1, `size` blocks each.
struct RowShare {
  int r, size, first, of;
};
template <typename Pick>
__device__ __forceinline__ RowShare row_share(const PagedAttnArgs& a, int block, const Pick& pick) {
  const int R = a.z.R, lane = threadIdx.x & 63;
  const auto blocks = [&](int r) { return r < R ? (slots_of(a, r, false) + block - 1) / block : 0; };
  long long all = 0;
  int most = 0, n = 0;
  for (int r0 = 0; r0 < R; r0 += 64) {
    n = blocks(r0 + lane);
    all += __builtin_amdgcn_readlane(wave_scan(n), 63);
    most = max(most, (int)group_max(row_max((float)n)));  // below 2^24: exact
  }
  const int size = paged_share_size(all, most, R, a.nsplit);
  int before = 0;
  for (int r0 = 0; r0 < R; r0 += 64) {
    const int r = r0 + lane;
    if (R > 64) n = blocks(r);
    const int of = r < R ? max(1, (n + size - 1) / size) : 0, end = before + wave_scan(of);
    const uint64_t hit = __ballot(r < R && pick(r, end - of, end));
    if (hit) {
      const int l = __builtin_ctzll(hit), first = __builtin_amdgcn_readlane(end - of, l);
      return RowShare{r0 + l, size, first, __builtin_amdgcn_readlane(of, l)};
    }
    before = __builtin_amdgcn_readlane(end, 63);
  }
  return RowShare{-1, 0, 0, 0};
}

// Tiles of a packed row, where they are this kernel's.
__device__ __forceinline__ int few_tiles(const PagedAttnArgs& a, int r) {
  const int n = prompt_count(a, r) * a.z.grp;
  return n > 0 && n <= a.few ? (n + 15) / 16 : 0;
}

// One workgroup per (tile, kv head, split).  PACKED: a tile is 16 (token, q-head) pairs of a row's packed tokens, each of which
// sees the slots up to its token's; else the q-heads of the row's newest token, which see all, and splits are shares.  The waves
// of a workgroup take its blocks in turn; a block's K is loaded as soon as the one before it is used up, its V likewise.
template <typename T, int HD, bool PACKED, bool SPLIT>
__global__ __launch_bounds__(64 * PATT_WAVES, HD == 64 ? 4 : 2) void k_paged_attn(PagedAttnArgs a) {
  using Blk = KvBlock<T, HD>;
  constexpr int NW = PATT_WAVES, E = Blk::E, B = Blk::B, NF = Blk::NF, ND = Blk::ND, KT = Blk::KT, NP = sizeof(T) == 2 ? 3 : 1;
  __shared__ PattLds<HD> sh;
  const PagedSizes& z = a.z;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g = lane >> 4;
  const int tile = (int)(blockIdx.x / (uint32_t)z.Hk), kvh = (int)(blockIdx.x % (uint32_t)z.Hk), split = blockIdx.y;
  int first = split * NW + w, stride = (PACKED ? a.nsplit : 1) * NW, stop = 0x7FFFFFFF;  // this wave's blocks: first, first + stride, ..
  int r = tile, n, end, limit, col = c16;   // slots of the row, slots that any column sees, that this lane's column sees
  size_t q_row;                             // activation row of this lane's column
  int head;
  bool live;
  if constexpr (PACKED) {
    if (blockIdx.x == 0 && split == 0)
      for (int i = tid; i < z.R; i += 64 * NW)
        if (prompt_count(a, i) < 0) atomicOr(a.err + i, 8);
    const Share s = find_share<64 * NW>(z.R, tile, (int*)&sh, [&](int i) { return few_tiles(a, i); });
    if (s.r < 0) return;
    r = s.r;
    const int o = a.offsets[r], c = a.offsets[r + 1] - o;
    n = a.kv_len[r];
    col = s.at * 16 + c16;
    live = col < c * z.grp;
    const int t = live ? col / z.grp : 0;
    limit = live ? n - c + t + 1 : 0;
    end = n - c + min(c, (s.at * 16 + 15) / z.grp + 1);
    q_row = (size_t)o + t;
    head = kvh * z.grp + (live ? col % z.grp : 0);
  } else {
    if constexpr (SPLIT) {
      const RowShare s = row_share(a, B, [&](int, int from, int to) { return from <= tile && tile < to; });
      if (s.r < 0) return;
      r = s.r;
      first = (tile - s.first) * s.size + w;
      stop = (tile - s.first + 1) * s.size;
    }
    q_row = r;
    live = c16 < z.grp;
    head = kvh * z.grp + (live ? c16 : 0);
  }
  const int* table = a.table + (size_t)r * z.row_pages;
  // entries of the wave's first 64 blocks, before the row's length is known
  const auto entry = [&](int slot) { return min(slot >> z.lgP, z.row_pages - 1); };
  int id0 = 0, id1 = 0;
  if constexpr (!PACKED) {
    const int slot = (first + lane * stride) * B;
    id0 = table[entry(slot)];
    if (KT == 2 && z.lgP == 4) id1 = table[entry(slot + 16)];
  }
  // queries: piece f holds channels 4 E f + E g ..
  u4 qh[NF], ql[NF];
  {
    const int W = z.H * HD;
    const T* p = (const T*)a.q + q_row * Act<T>::PL * W + (size_t)head * HD + E * g;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      qh[f] = live ? ld16(p + 4 * E * f) : zero16();
      if constexpr (Act<T>::SPLIT) ql[f] = live ? ld16(p + W + 4 * E * f) : zero16();
    }
  }
  if constexpr (!PACKED) end = limit = n = slots_of(a, r, kvh == 0 && tid == 0);
  const int nb = min((end + B - 1) / B, stop);
  const size_t run = (size_t)(HD * sizeof(T)) << z.lgP, page = 2 * run * z.Hk;
  const char* pool = (const char*)a.pool;
  const char* mine0 = pool + 2 * run * kvh;
  const float scale = 1.4426950408889634f / sqrtf((float)HD);
  f4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  int odd = 0;
  Blk x;
  const int least = __builtin_amdgcn_readfirstlane(limit);  // column 0 sees least
  for (int e0 = first; e0 < nb; e0 += 64 * stride) {
    const int mine = min(64, (nb - e0 + stride - 1) / stride);
    if (PACKED || e0 > first) {
      const int slot = (e0 + min(lane, mine - 1) * stride) * B;
      id0 = table[entry(slot)];
      if (KT == 2 && z.lgP == 4) id1 = table[entry(slot + 16)];
    }
    if (lane < mine) {
      id0 = checked_page(id0, z, a.err + r);
      if (KT == 2 && z.lgP == 4) id1 = (e0 + lane * stride) * B + 16 < end ? checked_page(id1, z, a.err + r) : id0;
    }
    asm volatile("" : "+v"(id0), "+v"(id1));  // waited for here, not with blocks under way
    const char *ka, *kb;
    const auto at = [&](int j) {
      const int slot = (e0 + j * stride) * B;
      ka = mine0 + (size_t)__builtin_amdgcn_readlane(id0, j) * page + (size_t)((slot & ((1 << z.lgP) - 1)) * HD) * sizeof(T);
      kb = ka + 16 * HD * sizeof(T);
      if (KT == 2 && z.lgP == 4) kb = mine0 + (size_t)__builtin_amdgcn_readlane(id1, j) * page;
    };
    at(0);
    x.template load_k<!PACKED>(ka, kb, true, pool);
    x.template load_v<!PACKED>(ka + run, kb + run, true, pool);
    for (int j = 0; j < mine; ++j) {
      const int base = (e0 + j * stride) * B;
      const bool masked = base + B > least, more = j + 1 < mine;
      if (more) at(j + 1);
      float sc[4 * KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        f4 s = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < NF; ++f) mma_act_b<T>(s, x.k[t][f], qh[f], ql[f]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[4 * t + e] = s[e];
      }
      x.template load_k<!PACKED>(ka, kb, more, pool);
      const int mine_slot = base + lane_slot<T>(g);  // this lane's E slots
      if (masked) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (mine_slot + e >= limit) sc[e] = -INFINITY;
      }
      float top = sc[0];
#pragma unroll
      for (int e = 1; e < E; ++e) top = fmaxf(top, sc[e]);
      top *= scale;
      if (__any(top > m)) {  // rarely, once a column has seen many keys
        const float mnew = fmaxf(m, group_max(top));
        const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mnew);
        l *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= alpha;
        m = mnew;
      }
      const float mz = m == -INFINITY ? 0.f : m;  // scores of -infinity alone: all weights 0
      float p[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], scale, -mz));
        l += p[e];
      }
      u4 pp[NP];
      if constexpr (NP == 3) weight_planes(p, pp);
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) pp[0][e] = __float_as_uint(p[e]);
      if (masked) {
        u4 keep;  // what lies past the slots that are seen may be NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int left = end - mine_slot - E / 4 * i;
          keep[i] = left >= E / 4 ? 0xFFFFFFFFu : E == 8 && left == 1 ? 0x0000FFFFu : 0u;
        }
        bool any = false;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          x.v[d] &= keep;
          if constexpr (PACKED) {  // columns see different slots: not finite values are dealt with after the loop
            any |= any_nonfinite<T>(x.v[d]);
            drop_nonfinite<T>(x.v[d]);
          }
        }
        if constexpr (PACKED) odd |= __any(any);
      }
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < NP; ++i) Frag<T>::mma(o[d], x.v[d], pp[i]);
      x.template load_v<!PACKED>(ka + run, kb + run, more, pool);
    }
  }
  if constexpr (PACKED)
    if (odd)  // infinities and NaN in V into the outputs of the columns that see their slots (mark_nonfinite)
      for (int e = first; e < nb; e += stride) {
        const int base = e * B, s0 = base + lane_slot<T>(g);
        if (base + B <= least) continue;
        u4 seen;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (E == 8) seen[i] = (s0 + 2 * i < limit ? 0x3F80u : 0u) | (s0 + 2 * i + 1 < limit ? 0x3F800000u : 0u);
          else seen[i] = s0 + i < limit ? 0x3F800000u : 0u;
        }
        // a lane's slots lie together, in one page; those that no column sees are not looked for
        const int id = s0 < end ? checked_page(table[s0 >> z.lgP], z, a.err + r) : 0;
        const char* v = mine0 + (size_t)id * page + run + ((size_t)(s0 & ((1 << z.lgP) - 1)) / E * HD + c16) * 16;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const u4 x = s0 < end ? ld16(v + d * 256) : zero16();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            f4 n = f4{0.f, 0.f, 0.f, 0.f};
            Frag<T>::mma(n, mark_nonfinite<T>(x, k), seen);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[d][i] += n[i] > 0.f ? (k ? -INFINITY : INFINITY) : 0.f;  // both: NaN
          }
        }
      }
  // per wave: maximum, sum and unnormalised outputs of each column
  l = group_sum(l);
  if (g == 0) {
    sh.m[w][c16] = m;
    sh.l[w][c16] = l;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) *reinterpret_cast<f4*>(&sh.o[w][c16][16 * d + 4 * g]) = o[d];
  __syncthreads();
  if (tid < 16) {
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) M = fmaxf(M, sh.m[i][tid]);
    const float mz = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      // 0 for a wave without slots; one whose scores are all NaN has maximum -infinity and sum NaN, which the factor 0 keeps
      const float e = __builtin_amdgcn_exp2f(sh.m[i][tid] - mz);
      L += e * sh.l[i][tid];
      sh.m[i][tid] = e;
    }
    sh.top[tid] = M;
    sh.sum[tid] = L;
  }
  __syncthreads();
  const int rows = PACKED ? 16 : z.grp;
  for (int t = tid; t < rows * (HD / 8); t += 64 * NW) {
    const int j = t / (HD / 8), d = t % (HD / 8) * 8;
    f4 v[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float e = sh.m[i][j];
#pragma unroll
      for (int u = 0; u < 2; ++u) v[u] += e * *reinterpret_cast<const f4*>(&sh.o[i][j][d + 4 * u]);
    }
    if constexpr (!SPLIT) {
      const float L = sh.sum[j];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][e] = L == 0.f ? 0.f : v[u][e] / L;
      size_t row = q_row;
      int h = kvh * z.grp + j;
      if constexpr (PACKED) {
        const int i = col - c16 + j, o0 = a.offsets[r], c = a.offsets[r + 1] - o0;
        if (i >= c * z.grp) break;
        row = (size_t)o0 + i / z.grp;
        h = kvh * z.grp + i % z.grp;
      }
      put_act8<T>(a.out, row, z.H * HD, h * HD + d, v);
    } else {
      const size_t rec = ((size_t)blockIdx.x * gridDim.y + split) * rows + j;
#pragma unroll
      for (int u = 0; u < 2; ++u) *reinterpret_cast<f4*>(a.part + rec * HD + d + 4 * u) = v[u];
      if (d == 0) {
        float* ml = a.part + (size_t)gridDim.x * gridDim.y * rows * HD + 2 * rec;
        ml[0] = sh.top[j];
        ml[1] = sh.sum[j];
      }
    }
  }
}

// The splits of a tile's (PACKED), or of a row's, query rows joined, a wave each.  `tiles`: of the attention's launch.
template <typename T, int HD, bool PACKED>
__global__ __launch_bounds__(256) void k_paged_join(PagedAttnArgs a, int tiles) {
  constexpr int V = HD / 64;
  const PagedSizes& z = a.z;
  const int lane = threadIdx.x & 63, rows = PACKED ? 16 : z.grp, j = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int x = (int)(blockIdx.x / (uint32_t)z.Hk), kvh = (int)(blockIdx.x % (uint32_t)z.Hk);
  if (!PACKED && j >= rows) return;
  size_t row = x, rec, step;
  int h = kvh * z.grp + j, ns = a.nsplit;
  if constexpr (PACKED) {
    __shared__ int scratch[10];
    const Share s = find_share<256>(z.R, x, scratch, [&](int i) { return few_tiles(a, i); });
    if (s.r < 0 || j >= rows) return;
    const int o = a.offsets[s.r], c = a.offsets[s.r + 1] - o, i = s.at * 16 + j;
    if (i >= c * z.grp) return;
    row = (size_t)o + i / z.grp;
    h = kvh * z.grp + i % z.grp;
    rec = (size_t)blockIdx.x * ns * rows + j;
    step = rows;
  } else {
    const RowShare s = row_share(a, KvBlock<T, HD>::B, [&](int r, int, int) { return r == x; });
    ns = s.of;
    rec = ((size_t)s.first * z.Hk + kvh) * rows + j;
    step = (size_t)z.Hk * rows;
  }
  float v[V];
  join_row<HD>(a.part, a.part + (size_t)tiles * z.Hk * (PACKED ? ns : 1) * rows * HD, rec, step, ns, v);
#pragma unroll
  for (int i = 0; i < V; ++i) Act<T>::put(a.out, row, z.H * HD, h * HD + lane * V + i, v[i]);
}

// ---------------------------------------------------------------- pages
__device__ __forceinline__ int pages_of(int slots, int lgP) { return (int)(((long long)slots + (1 << lgP) - 1) >> lgP); }
__device__ __forceinline__ bool fits(long long slots, const PagedSizes& z) { return slots >= 0 && slots <= (long long)z.row_pages << z.lgP; }
__device__ __forceinline__ bool in_pool(int id, const PagedSizes& z) { return (unsigned)id < (unsigned)z.n_pages; }

// With `parent`: a row takes over the entries of another as they were, -1 for what it had beyond them; pages count the rows
// that hold them.  The tables are written back at the end (k_paged_copy), when every row has been read.
struct Taken {
  int from, now, old;  // the row whose entries are taken over (or -1), their number, that of the row's own
};
__device__ __forceinline__ Taken take_length(const PagedAdvanceArgs& a, int r, bool first) {  // `first`: the thread that reports
  const PagedSizes& z = a.z;
  const int had = a.kv_len[r];
  int from = a.parent[r], len = 0, old = 0;
  bool bad = false;
  if (!fits(had, z)) {            // nothing is known of the row's pages: it stays as it is
    bad = true;
    from = r;
    len = had;
  } else {
    old = pages_of(had, z.lgP);
    if (from >= 0) {
      bad = from >= z.R || !fits(a.kv_len[from], z);
      if (bad) from = r;
      len = a.kv_len[from];
    } else if (from < -1) {
      bad = true;
      from = r;
      len = had;
    }
  }
  const int now = fits(len, z) ? pages_of(len, z.lgP) : 0;
  if (first) {
    if (bad) atomicOr(a.err + r, 8);
    a.taken_len[r] = len;
    a.span[r] = max(old, now);
  }
  return Taken{from, now, old};
}
__device__ __forceinline__ void take_entry(const PagedAdvanceArgs& a, int r, const Taken& t, int e) {  // e < max(old, now)
  const PagedSizes& z = a.z;
  const int id = e < t.now ? a.table[(size_t)max(t.from, 0) * z.row_pages + e] : -1;
  a.taken[(size_t)r * z.row_pages + e] = id;
  if (t.from == r) return;
  if (e < t.old) {
    const int was = a.table[(size_t)r * z.row_pages + e];
    if (in_pool(was, z)) atomicSub(a.refs + was, 1);
    else atomicOr(a.err + r, 32);
  }
  if (e < t.now) {
    if (in_pool(id, z)) atomicAdd(a.refs + id, 1);
    else atomicOr(a.err + r, 32);
  }
}
__global__ __launch_bounds__(256) void k_paged_take(PagedAdvanceArgs a) {  // a workgroup a row
  const int r = blockIdx.x, tid = threadIdx.x;
  const Taken t = take_length(a, r, tid == 0);
  for (int e = tid; e < max(t.old, t.now); e += 256) take_entry(a, r, t, e);
}

constexpr int GIVE_THREADS = 1024;
constexpr int PAGED_MAX_ROWS = 4096;

// inclusive sums over the workgroup's threads; `total` of all
__device__ __forceinline__ int block_scan(int v, int* waves, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan(v);
  __syncthreads();
  if (lane == 63) waves[w] = v;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < GIVE_THREADS / 64; ++i) {
    const int x = waves[i];
    before += i < w ? x : 0;
    all += x;
  }
  total = all;
  return before + v;
}
// Global memory that atomics of this workgroup have changed before a barrier.  Atomics are done in the L2, and these loads go there
// past the CU's cache, which may hold the value as it was.  The barrier orders the two for threads of one workgroup; it does not wait
// for the atomics.  It need not: the workgroup's waves are on one CU, whose requests for an address reach the L2 in the order in which
// they were issued.  (Compiled for threadgroup split, where waves of a workgroup may be on two CUs, the barrier does come with a wait
// for vector memory.)  Work of several workgroups would need fences for the whole GPU, 2 to 4 us each here.
__device__ __forceinline__ int changed(const int* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// The pages from p0 on, CHUNKS times 64 to a wave: chunk k is pages page_at(p0, k) of its lanes.  All loads are under way at once.
// CHUNKS is 16 in pools of more than FEW_PAGES, where tiles follow one another, else 4, which leaves less to do for each wave (give /
// compact, us, by 4 and by 16: 4,096 pages 6.7 / 6.6 and 7.5 / 9.9, 131,072 all held 48 / 107 and 16 / 51).
constexpr int FEW_PAGES = 4096;
template <int CHUNKS> __device__ __forceinline__ int page_at(int p0, int k) {
  return p0 + (int)(threadIdx.x >> 6) * CHUNKS * 64 + k * 64 + (int)(threadIdx.x & 63);
}
template <int CHUNKS, bool ATOMIC>
__device__ __forceinline__ void page_refs(const int* refs, int p0, int n, int absent, int* out) {
  const int base = __builtin_amdgcn_readfirstlane(page_at<CHUNKS>(p0, 0)), lane = threadIdx.x & 63;
  const int* at = refs + base;
  if (base + CHUNKS * 64 <= n) {
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) out[k] = ATOMIC ? changed(at + k * 64 + lane) : at[k * 64 + lane];
  } else {
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      out[k] = absent;
      if (base + k * 64 + lane < n) out[k] = ATOMIC ? changed(at + k * 64 + lane) : at[k * 64 + lane];
    }
  }
}
// What the waves before this one have of `mine`, a value of the wave; `total` of all.  `waves` is another half in every second call,
// so that one barrier does.
__device__ __forceinline__ int waves_before(int mine, int (*waves)[GIVE_THREADS / 64], int turn, int& total) {
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) waves[turn & 1][w] = mine;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < GIVE_THREADS / 64; ++i) {
    const int x = waves[turn & 1][i];
    before += i < w ? x : 0;
    all += x;
  }
  total = all;
  return before;
}
__device__ __forceinline__ int lanes_before(uint64_t mask) {  // of the mask's
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// One workgroup: gives up the pages of slots that rows drop, finds out which shared pages have to be copied and how many
// pages each row needs, and hands out the lowest free ones in the order of the rows.  A row whose page has other holders gets
// a copy, except, where all holders write to it in this call, the lowest of them.  Bound by latency: lengths, the rows' last
// entries, their references, and the writes, one round trip to memory each, and the scans between them.
constexpr int GIVE_PAGES = 2048;            // of the pages to give out, in LDS; those behind them in the workspace
// TAKE: up to TAKE_ENTRIES table entries are taken over here, a launch less (32 rows of beams, 16 layers, 20 us for 22).
constexpr int TAKE_ENTRIES = 4 * GIVE_THREADS;
template <int CHUNKS, bool TAKE>
__global__ __launch_bounds__(GIVE_THREADS) void k_paged_give(PagedAdvanceArgs a) {
  __shared__ int ends[PAGED_MAX_ROWS];      // pages wanted by the rows up to this one
  __shared__ unsigned char copied[PAGED_MAX_ROWS];
  __shared__ int waves[GIVE_THREADS / 64], halves[2][GIVE_THREADS / 64];
  __shared__ int given[GIVE_PAGES];
  const PagedSizes& z = a.z;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, P = 1 << z.lgP;
  constexpr int PER = PAGED_MAX_ROWS / GIVE_THREADS;  // rows of a thread: tid, tid + GIVE_THREADS, ..
  int* table = a.parent ? a.taken : a.table;
  const int* lengths = a.parent ? a.taken_len : a.kv_len;
  if constexpr (TAKE) {
    __shared__ Taken taken[GIVE_THREADS];
    if (tid < z.R) taken[tid] = take_length(a, tid, true);
    __syncthreads();
    const int entries = z.R * z.row_pages;
#pragma unroll
    for (int i = 0; i < TAKE_ENTRIES / GIVE_THREADS; ++i) {
      const int at = tid + i * GIVE_THREADS, r = at / z.row_pages, e = at - r * z.row_pages;
      if (at < entries && e < max(taken[r].old, taken[r].now)) take_entry(a, r, taken[r], e);
    }
    __syncthreads();
  }
  // references of the first pages, for the search for free ones
  const auto load_refs = [&](int p0, int* refs) {
    page_refs<CHUNKS, true>(a.refs, p0, z.n_pages, 1, refs);
  };
  int refs[CHUNKS];
  load_refs(0, refs);
  // a row's length, and by how many slots it changes: 0 where it cannot
  int len[PER], c[PER];
  bool drops = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = tid + i * GIVE_THREADS;
    len[i] = c[i] = 0;
    if (r >= z.R) continue;
    len[i] = lengths[r];
    const int want = a.count[r];
    const bool ok = fits(len[i], z) && fits((long long)len[i] + want, z);
    c[i] = ok ? want : 0;
    if (!fits(len[i], z) || (!ok && want != 0)) atomicOr(a.err + r, 8);
    drops |= c[i] < 0;
  }
  if (__syncthreads_or(drops)) {  // dropped slots: a wave a row
    for (int r = w; r < z.R; r += GIVE_THREADS / 64) {
      const int n = lengths[r], less = a.count[r];
      if (less >= 0 || !fits(n, z) || !fits((long long)n + less, z)) continue;
      for (int e = pages_of(n + less, z.lgP) + lane; e < pages_of(n, z.lgP); e += 64) {
        int& entry = table[(size_t)r * z.row_pages + e];
        if (in_pool(entry, z)) atomicSub(a.refs + entry, 1);
        else atomicOr(a.err + r, 32);
        entry = -1;
      }
    }
    __syncthreads();
    load_refs(0, refs);
  }
  // rows whose last page is written to and has other holders
  int page[PER], holders[PER];
  bool any = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = tid + i * GIVE_THREADS;
    page[i] = holders[i] = 0;
    if (c[i] <= 0 || len[i] % P == 0) continue;
    page[i] = table[(size_t)r * z.row_pages + len[i] / P];
    if (in_pool(page[i], z)) holders[i] = changed(a.refs + page[i]);
    else atomicOr(a.err + r, 32);
    if (holders[i] > 1) {
      a.owner[2 * page[i]] = 0;
      a.owner[2 * page[i] + 1] = z.R;
      any = true;
    }
  }
  bool copy[PER] = {};
  int ncopy = 0;
  if (__syncthreads_or(any)) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (holders[i] > 1) {
        atomicAdd(a.owner + 2 * page[i], 1);
        atomicMin(a.owner + 2 * page[i] + 1, tid + i * GIVE_THREADS);
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (holders[i] > 1) {
        copy[i] = changed(a.owner + 2 * page[i]) != holders[i] || changed(a.owner + 2 * page[i] + 1) != tid + i * GIVE_THREADS;
        ncopy += copy[i];
      }
  }
  // pages wanted by the rows before: GIVE_THREADS rows at a time
  int need[PER], total = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = tid + i * GIVE_THREADS;
    need[i] = c[i] > 0 ? pages_of(len[i] + c[i], z.lgP) - pages_of(len[i], z.lgP) + copy[i] : 0;
    if (i * GIVE_THREADS >= z.R) break;
    int here;
    const int end = total + block_scan(need[i], waves, here);
    total += here;
    if (r < z.R) {
      ends[r] = end;
      copied[r] = copy[i];
    }
  }
  int copies;
  int my_copy = block_scan(ncopy, waves, copies) - ncopy;
  // the lowest free pages, until there are enough
  int found = 0;
  for (int p0 = 0, turn = 0; p0 < z.n_pages && found < total; p0 += CHUNKS * GIVE_THREADS, ++turn) {
    if (p0 > 0) load_refs(p0, refs);
    int mine = 0, here;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) mine += __builtin_popcountll(__ballot(refs[k] <= 0));
    int at = found + waves_before(mine, halves, turn, here);
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      const uint64_t free = __ballot(refs[k] <= 0);
      if (free == 0) continue;
      const int to = at + lanes_before(free);
      if (refs[k] <= 0) {
        if (to < min(total, GIVE_PAGES)) given[to] = page_at<CHUNKS>(p0, k);
        else if (to < total) a.pages[to] = page_at<CHUNKS>(p0, k);
      }
      at += __builtin_popcountll(free);
    }
    found += here;
  }
  const bool enough = found >= total;
  __syncthreads();
  const auto given_page = [&](int k) { return k < GIVE_PAGES ? given[k] : a.pages[k]; };
  if (enough) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (copy[i]) {
        a.copies[2 + 2 * my_copy] = page[i];
        a.copies[3 + 2 * my_copy] = given_page(ends[tid + i * GIVE_THREADS] - need[i]);
        atomicSub(a.refs + page[i], 1);
        ++my_copy;
      }
    for (int k = tid; k < total; k += GIVE_THREADS) {
      int lo = 0, hi = z.R - 1;  // the first row with ends > k
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (ends[mid] > k) hi = mid;
        else lo = mid + 1;
      }
      const int r = lo, i = k - (r ? ends[r - 1] : 0), id = given_page(k);
      table[(size_t)r * z.row_pages + pages_of(lengths[r], z.lgP) + i - copied[r]] = id;
      a.refs[id] = 1;
    }
  }
  if (tid == 0) a.copies[0] = enough ? copies : 0;
  __syncthreads();  // lengths are read above
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = tid + i * GIVE_THREADS;
    if (r >= z.R) continue;
    if (c[i] > 0 && !enough) {
      atomicOr(a.err + r, 64);
      c[i] = 0;
    }
    a.kv_len[r] = len[i] + c[i];
    a.start[r] = len[i] + min(c[i], 0);
    if (a.parent && fits(len[i], z)) a.span[r] = max(a.span[r], pages_of(len[i] + c[i], z.lgP));
  }
}

// Pages `copies` of every layer, in pieces of 16 KB, by a grid of fixed size that goes round; beside them the tables: what rows
// have taken over is written back (`span` entries of a row), or entries go by the map of the compaction.
constexpr int COPY_THREADS = 256, COPY_PIECE = 16 * 1024;  // bytes of a workgroup at a time
struct PagedTables {
  PagedSizes z;
  int* table;
  const int* taken; const int* span;
  const int* map; const int* kv_len; int* err;
};
__global__ __launch_bounds__(COPY_THREADS) void k_paged_copy(PagedCopyArgs c, PagedTables t) {
  const int tid = threadIdx.x;
  const int n = c.copies[0], pieces = (c.page_bytes + COPY_PIECE - 1) / COPY_PIECE;
  if (t.span)
    for (int r = blockIdx.x; r < t.z.R; r += gridDim.x)
      for (int e = tid; e < t.span[r]; e += COPY_THREADS) t.table[(size_t)r * t.z.row_pages + e] = t.taken[(size_t)r * t.z.row_pages + e];
  if (t.map)
    for (int r = blockIdx.x; r < t.z.R; r += gridDim.x) {
      const int len = t.kv_len[r];
      if (!fits(len, t.z)) {
        if (tid == 0) atomicOr(t.err + r, 8);
        continue;
      }
      int* table = t.table + (size_t)r * t.z.row_pages;
      for (int e = tid; e < pages_of(len, t.z.lgP); e += COPY_THREADS) {
        const int id = table[e], to = in_pool(id, t.z) ? t.map[id] : -1;
        if (to < 0) atomicOr(t.err + r, 32);
        else table[e] = to;
      }
    }
  const uint32_t items = (uint32_t)n * c.layers * pieces;  // below 2^31
  for (uint32_t i = blockIdx.x; i < items; i += gridDim.x) {
    const int piece = (int)(i % pieces), layer = (int)(i / pieces % c.layers), k = (int)(i / pieces / c.layers);
    const size_t from = (size_t)c.copies[2 + 2 * k] * c.page_bytes, to = (size_t)c.copies[3 + 2 * k] * c.page_bytes;
    char* base = c.pool + (size_t)layer * c.layer_bytes + (size_t)piece * COPY_PIECE;
    const int left = c.page_bytes - piece * COPY_PIECE;
    u4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int b = (u * COPY_THREADS + tid) * 16;
      if (b < left) v[u] = ld16_stream(base + from + b);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int b = (u * COPY_THREADS + tid) * 16;
      if (b < left) *reinterpret_cast<u4*>(base + to + b) = v[u];
    }
  }
}

// Pages with holders move to the free places below their number, the lowest first.  One workgroup finds them; map and counts
// follow.  (Pools of one tile are read once.)
template <int CHUNKS>
__global__ __launch_bounds__(GIVE_THREADS) void k_paged_compact(PagedCompactArgs a) {
  __shared__ int halves[2][GIVE_THREADS / 64];
  const int tid = threadIdx.x, n = a.z.n_pages;
  const auto load = [&](int p0, int* refs) {
    page_refs<CHUNKS, false>(a.refs, p0, n, 0, refs);
  };
  int refs[CHUNKS], mine = 0, used, turn = 0;
  for (int p0 = 0; p0 < n; p0 += CHUNKS * GIVE_THREADS) {
    load(p0, refs);
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) mine += __builtin_popcountll(__ballot(refs[k] > 0));
  }
  waves_before(mine, halves, turn++, used);
  int holes = 0, moves = 0;  // so far
  for (int p0 = 0; p0 < n; p0 += CHUNKS * GIVE_THREADS) {
    if (n > CHUNKS * GIVE_THREADS) load(p0, refs);
    // free places below `used`, pages that move
    const auto hole = [&](int k) { return refs[k] <= 0 && page_at<CHUNKS>(p0, k) < used; };
    const auto move = [&](int k) { return refs[k] > 0 && page_at<CHUNKS>(p0, k) >= used; };
    int both = 0, here;  // 16 bits each: a tile has 2^14 at most
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) both += __builtin_popcountll(__ballot(hole(k))) | __builtin_popcountll(__ballot(move(k))) << 16;
    const int at = waves_before(both, halves, turn++, here);
    int ah = holes + (at & 0xFFFF), am = moves + (at >> 16);
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      const int p = page_at<CHUNKS>(p0, k);
      const uint64_t h = __ballot(hole(k)), m = __ballot(move(k));
      if (p < n) a.map[p] = refs[k] > 0 && p < used ? p : -1;
      if (h != 0 && hole(k)) a.copies[3 + 2 * (ah + lanes_before(h))] = p;
      if (m != 0 && move(k)) a.copies[2 + 2 * (am + lanes_before(m))] = p;
      ah += __builtin_popcountll(h);
      am += __builtin_popcountll(m);
    }
    holes += here & 0xFFFF;
    moves += here >> 16;
  }
  if (tid == 0) {
    a.copies[0] = moves;
    a.used[0] = used;
  }
  __syncthreads();
  for (int k = tid; k < moves; k += GIVE_THREADS) {
    const int from = changed(a.copies + 2 + 2 * k), to = changed(a.copies + 3 + 2 * k);
    a.map[from] = to;
    a.refs[to] = a.refs[from];
    a.refs[from] = 0;
  }
}

template <typename T, int HD>
int append_t(const PagedAppendArgs& a, Stream s) {
  const unsigned blocks = (unsigned)paged_append_workgroups(a.N, a.z.R, a.z.Hk * (a.q ? 2 : 1));
  launch_k((k_paged_append<T, HD>), dim3(blocks), dim3(256), 0, s, a);
  return 0;
}
template <typename T, int HD>
int attention_t(const PagedAttnArgs& a, long long packed_tiles, Stream s) {
  const PagedSizes& z = a.z;
  const dim3 block(64 * PATT_WAVES);
  if (a.offsets) {
    const int tiles = (int)packed_tiles;
    launch_k(a.nsplit > 1 ? k_paged_attn<T, HD, true, true> : k_paged_attn<T, HD, true, false>, dim3(tiles * z.Hk, a.nsplit), block, 0, s, a);
    if (a.nsplit > 1) launch_k((k_paged_join<T, HD, true>), dim3(tiles * z.Hk, 4), dim3(256), 0, s, a, tiles);
    return 0;
  }
  const int tiles = z.R + a.nsplit;  // a share more for the end of each row
  launch_k(a.nsplit > 0 ? k_paged_attn<T, HD, false, true> : k_paged_attn<T, HD, false, false>, dim3(tiles * z.Hk), block, 0, s, a);
  if (a.nsplit > 0) launch_k((k_paged_join<T, HD, false>), dim3(z.R * z.Hk, (z.grp + 3) / 4), dim3(256), 0, s, a, tiles);
  return 0;
}

#define PAGED_DISPATCH(fn, ...)                                             \
  do {                                                                      \
    if (hd == 64) return dtype == 1 ? fn<bf16, 64>(__VA_ARGS__) : fn<float, 64>(__VA_ARGS__);    \
    if (hd == 128) return dtype == 1 ? fn<bf16, 128>(__VA_ARGS__) : fn<float, 128>(__VA_ARGS__); \
    return -1;                                                              \
  } while (0)

}  // namespace

int launch_paged_append(int dtype, int hd, const PagedAppendArgs& a, Stream s) { PAGED_DISPATCH(append_t, a, s); }
int launch_paged_attention(int dtype, int hd, const PagedAttnArgs& a, long long tiles, Stream s) { PAGED_DISPATCH(attention_t, a, tiles, s); }

int launch_paged_advance(const PagedAdvanceArgs& a, const PagedCopyArgs& c, Stream s) {
  const bool many = a.z.n_pages > FEW_PAGES, take = a.parent && a.z.R <= GIVE_THREADS && (long long)a.z.R * a.z.row_pages <= TAKE_ENTRIES;
  if (a.parent && !take) launch_k(k_paged_take, dim3(a.z.R), dim3(256), 0, s, a);
  launch_k(many ? take ? k_paged_give<16, true> : k_paged_give<16, false> : take ? k_paged_give<4, true> : k_paged_give<4, false>, dim3(1),
           dim3(GIVE_THREADS), 0, s, a);
  const PagedTables t{a.z, a.table, a.taken, a.parent ? a.span : nullptr, nullptr, nullptr, nullptr};
  launch_k(k_paged_copy, dim3(1024), dim3(COPY_THREADS), 0, s, c, t);
  return 0;
}
int launch_paged_compact(const PagedCompactArgs& a, const PagedCopyArgs& c, Stream s) {
  launch_k(a.z.n_pages > FEW_PAGES ? k_paged_compact<16> : k_paged_compact<4>, dim3(1), dim3(GIVE_THREADS), 0, s, a);
  const PagedTables t{a.z, a.table, nullptr, nullptr, a.map, a.kv_len, a.err};
  launch_k(k_paged_copy, dim3(2048), dim3(COPY_THREADS), 0, s, c, t);
  return 0;
}

}  // namespace ham
