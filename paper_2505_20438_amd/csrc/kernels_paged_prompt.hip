// Causal attention of packed bf16 prompts over their pages (layout: kernels_paged.h).
//
// A row's c tokens times the grp q-heads of a kv head are c * grp query rows in the order of the tokens; 32 of them, whatever
// the group, are one wave's operand.  A workgroup of NW waves has QR = 32 NW / KS of them, its waves' keys in KS shares; 8 NW slots
// at a time (a stage) land in LDS straight from the pages, in the order of the pool, which is that of the operands.  Both products are
// 32x32x16 matrix instructions with the query row in the lane index:
//   S^T = K Q^T (A = K rows, B = Q rows)  and  O^T = V^T P^T (A = V^T rows, B = P rows),
// so a lane (row l & 31, half l >> 5) holds scores, weights, softmax state and output columns of one row and only the other half
// shares it.  The running maximum moves, and with it the outputs, only when a score exceeds it by more than 8 powers of two.
// Masks, and values past the slots that a wave sees, are dealt with only in blocks that reach past the wave's first row.
//
// Bound by the matrix cores at the card's power limit: 2,048 tokens of 32 heads of 128 behind 30,720 slots 1,890 to 1,950 us, 1.4 PFLOP/s
// of the products that are executed (K Q^T for two planes of the queries, P V for three of the weights), as a library's 8,192^3
// product; 7 prompts of 500 to 4,001 tokens 704 to 740 us, 1.1 to 1.2 (softmax, and planes, on the vector units are the rest).
// Without softmax the first took 1,612 us, without products 767; two planes of the weights, 16 bits, 1,590.
#include "gemm_epilogue.h"
#include "launch_rules.h"
#include "paged_device.h"

namespace ham {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

template <int HD> struct PP {
  static constexpr int KB = 32, NS = 4;                            // slots of a block; stages in the ring
  static constexpr int RUN = 2 * HD;                               // 16-byte units of 16 slots of K or V: a stage is NW / 2 of each
  static constexpr int LPW = RUN / 64;                             // a wave's loads of a stage: one run
  static constexpr int NF = HD / 16, ND = HD / 32;
};

// Scores of this wave's 32 rows against a block of 32 slots.
template <int HD>
__device__ __forceinline__ f16v block_scores(const u4* kblk, const u4* qh, const u4* ql) {
  using P = PP<HD>;
  const int lane = lane_anew(), h = lane >> 5, r = lane & 31;
  f16v s;
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = 0.f;
  const u4* kr = kblk + (r >> 4) * P::RUN + h * 16 + (r & 15);
#pragma unroll
  for (int f = 0; f < P::NF; ++f) {
    const bf16x8 k = __builtin_bit_cast(bf16x8, kr[f * 32]);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, __builtin_bit_cast(bf16x8, qh[f]), s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, __builtin_bit_cast(bf16x8, ql[f]), s, 0, 0, 0);
  }
  return s;
}

// The softmax update of (m, l, o) by a block's scores, whose weights are left in three bf16 planes, all 24 bits of them.  `keep`:
// how many of the block's slots the lane's row sees (32 or more: all); score e is slot 16 (e / 8) + 8 h + e % 8.
template <int HD>
__device__ __forceinline__ void block_weights(f16v s, bool masked, int keep, float sc, float& mrun, float& lrun, f16v* o, u4 (*pp)[3]) {
  using P = PP<HD>;
  const int h = (threadIdx.x & 63) >> 5;
  if (masked) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (16 * (e >> 3) + 8 * h + (e & 7) >= keep) s[e] = -INFINITY;
  }
  float bm = s[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) bm = fmaxf(bm, s[e]);
  bm *= sc;  // sc > 0
  if (__any(bm > mrun + 8.f)) {  // each row by its own scores, whatever the others of the wave do
    bm = fmaxf(bm, __shfl_xor(bm, 32, WAVE));
    const float mnew = bm > mrun + 8.f ? bm : mrun;
    const float alpha = mnew == mrun ? 1.f : __builtin_amdgcn_exp2f(mrun - mnew);  // 0 from the initial -infinity
    lrun *= alpha;
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
    mrun = mnew;
  }
  const float mref = mrun == -INFINITY ? 0.f : mrun;  // no score above -infinity yet: weights 0
  float p[16], ps = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[e], sc, -mref));
#pragma unroll
  for (int e = 0; e < 16; ++e) ps += p[e];
  lrun += ps;
  weight_planes(p, pp[0]);
  weight_planes(p + 8, pp[1]);
}

// Outputs += weights of a block times its V, whose first operands `v` are there already (first_values).
constexpr int VFIRST = 4;
template <int HD>
__device__ __forceinline__ const u4* lane_values(const u4* vblk) {  // channels 32 d + r of slots 16 t + 8 h ..: [t * RUN + 32 d]
  return vblk + ((threadIdx.x & 63) >> 5) * HD + (threadIdx.x & 31);
}
template <int HD>
__device__ __forceinline__ void first_values(const u4* vblk, u4* v) {
  const u4* vr = lane_values<HD>(vblk);
#pragma unroll
  for (int i = 0; i < VFIRST; ++i) v[i] = vr[i % 2 * PP<HD>::RUN + i / 2 * 32];
}
template <int HD>
__device__ __forceinline__ void block_values(const u4* vblk, const u4* v, const u4 (*pp)[3], f16v* o) {
  using P = PP<HD>;
  const u4* vr = lane_values<HD>(vblk);
#pragma unroll
  for (int d = 0; d < P::ND; ++d)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 x = __builtin_bit_cast(bf16x8, 2 * d + t < VFIRST ? v[(2 * d + t) % VFIRST] : vr[t * P::RUN + d * 32]);
#pragma unroll
      for (int i = 0; i < 3; ++i) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, pp[t][i]), o[d], 0, 0, 0);
    }
}
// The order of a phase's products and LDS reads: an operand is read four before its turn.
template <int HD>
__device__ __forceinline__ void order_products() {
  using P = PP<HD>;
  constexpr int NV = 2 * P::ND, NK = P::NF;
  static_assert(NK >= VFIRST, "the reads of the last of them go with V's products");
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
    __builtin_amdgcn_sched_group_barrier(0x008, 3, 0);  // matrix products
  }
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    if (i < NK - VFIRST) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
  }
}
// ... of a block of which the wave sees `vkeep` slots: values past them count as 0, whatever they hold, and so do infinities and
// NaN, since a row that does not see their slot has weight 0 for it, and 0 times them is NaN.  Whether there are any: see_nonfinite
// deals with them when all blocks are done and the registers are free for it.
template <int HD>
__device__ __forceinline__ bool block_values_masked(const u4* vblk, int vkeep, const u4 (*pp)[3], f16v* o) {
  using P = PP<HD>;
  const int h = (threadIdx.x & 63) >> 5;
  const u4* vr = lane_values<HD>(vblk);
  bool odd = false;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int k = vkeep - (16 * t + 8 * h);  // of this lane's eight slots
    u4 keep;
#pragma unroll
    for (int i = 0; i < 4; ++i) keep[i] = k >= 2 * i + 2 ? 0xFFFFFFFFu : k == 2 * i + 1 ? 0x0000FFFFu : 0u;
#pragma unroll
    for (int d = 0; d < P::ND; ++d) {
      u4 v = vr[t * P::RUN + d * 32] & keep;
      odd |= any_nonfinite<bf16>(v);
      drop_nonfinite<bf16>(v);
#pragma unroll
      for (int i = 0; i < 3; ++i)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pp[t][i]), o[d], 0, 0, 0);
    }
  }
  return __any(odd);
}
// Infinities and NaN among 16 values of each channel, `v` (pool) of slots from `base` on, into the outputs of the rows that see
// their slots: products of 1 for such a value (infinity and NaN, then -infinity and NaN) and 1 for a slot that is seen.
template <int HD>
__device__ __forceinline__ void see_nonfinite(const u4* v, int base, int limit, f16v* o) {
  const int l = threadIdx.x & 63, h = l >> 5, r = l & 31;
  u4 seen;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s0 = base + 8 * h + 2 * i;
    seen[i] = (s0 < limit ? 0x3F80u : 0u) | (s0 + 1 < limit ? 0x3F800000u : 0u);
  }
#pragma unroll
  for (int d = 0; d < PP<HD>::ND; ++d) {
    const u4 x = v[h * HD + 32 * d + r];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f16v n;
#pragma unroll
      for (int e = 0; e < 16; ++e) n[e] = 0.f;
      n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, mark_nonfinite<bf16>(x, k)), __builtin_bit_cast(bf16x8, seen), n, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] += n[e] > 0.f ? (k ? -INFINITY : INFINITY) : 0.f;  // both: NaN
    }
  }
}

// The rows' shares of QR query rows: those of the row with the most slots first, and of a row the last first (its keys are the
// most), so that the workgroups that take longest start first.  Rows past the 64th in the order they have.
struct PromptShare {
  int r, at, offset, count, slots;  // row (< 0: none left), share of it; its packed tokens and slots
};
template <int QR, int NT>
__device__ __forceinline__ PromptShare prompt_share(const PagedAttnArgs& a, int i, int* scratch) {
  const int R = a.z.R, lane = threadIdx.x & 63;
  const auto shares = [&](int c) { return c * a.z.grp > a.few ? (c * a.z.grp + QR - 1) / QR : 0; };
  if (R > 64) {
    const Share s = find_share<NT>(R, i, scratch, [&](int r) { return shares(prompt_count(a, r)); });
    if (s.r < 0) return PromptShare{-1, 0, 0, 0, 0};
    const int o = scalar_at(a.offsets, s.r), c = scalar_at(a.offsets + 1, s.r) - o;
    return PromptShare{s.r, shares(c) - 1 - s.at, o, c, scalar_at(a.kv_len, s.r)};
  }
  int o = 0, c = -1, len = -1;  // of row `lane`: one round trip for all that is asked of it
  if (lane < R) {
    o = a.offsets[lane];
    const int e = a.offsets[lane + 1];
    len = a.kv_len[lane];
    c = o >= 0 && e >= o && e <= a.N && len <= a.kv_max && e - o <= len ? e - o : -1;
  }
  const int n = shares(c);
  int before = 0;
  for (int j = 0; j < R; ++j) {
    const int kj = __builtin_amdgcn_readlane(len, j), nj = __builtin_amdgcn_readlane(n, j);
    before += kj > len || (kj == len && j < lane) ? nj : 0;
  }
  const uint64_t hit = __ballot(i >= before && i < before + n);
  if (hit == 0) return PromptShare{-1, 0, 0, 0, 0};
  const int r = __builtin_ctzll(hit);
  return PromptShare{r, __builtin_amdgcn_readlane(n, r) - 1 - (i - __builtin_amdgcn_readlane(before, r)), __builtin_amdgcn_readlane(o, r),
                     __builtin_amdgcn_readlane(c, r), __builtin_amdgcn_readlane(len, r)};
}

template <int HD, int KS, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_paged_prompt(PagedAttnArgs a) {
  using P = PP<HD>;
  constexpr int NS = P::NS, LPW = P::LPW, QT = NW / KS, QR = 32 * QT;
  constexpr int SR = NW / 2, ST = 16 * SR;  // a stage: runs of K, slots
  __shared__ u4 lds[NS][NW * P::RUN];
  const PagedSizes& z = a.z;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int job = (int)(blockIdx.x / (uint32_t)z.Hk), kvh = (int)(blockIdx.x % (uint32_t)z.Hk), split = blockIdx.y;
  if (blockIdx.x == 0 && split == 0)
    for (int i = threadIdx.x; i < z.R; i += 64 * NW)
      if (prompt_count(a, i) < 0) atomicOr(a.err + i, 8);
  const PromptShare sh = prompt_share<QR, 64 * NW>(a, job, (int*)lds);
  if (sh.r < 0) return;
  const int r = sh.r, o0 = sh.offset, c = sh.count, held = sh.slots - c;
  const int qt = w % QT, ks = w / QT;
  const int i0 = sh.at * QR + qt * 32, i1 = min(i0 + 32, c * z.grp);  // this wave's rows [i0, i1), of c * grp
  const bool rows_ok = i0 < c * z.grp;
  const int wave_least = rows_ok ? held + i0 / z.grp + 1 : 0, wave_end = rows_ok ? held + (i1 - 1) / z.grp + 1 : 0;
  const int wg_end = held + (min(sh.at * QR + QR, c * z.grp) - 1) / z.grp + 1;
  const int W = z.H * HD;
  struct Row {      // of a lane: its token, q-head, and how many slots it sees; past the rows none
    bool there;
    int token, head, limit;
  };
  const auto row_of = [&](int l) {
    const int i = i0 + (l & 31), t = i / z.grp;
    const bool there = i < c * z.grp;
    return Row{there, there ? t : 0, kvh * z.grp + (there ? i - t * z.grp : 0), there ? held + t + 1 : 0};
  };
  u4 qh[P::NF], ql[P::NF];
  {
    const Row row = row_of(lane);
    const bf16* qp = (const bf16*)a.q + (size_t)(o0 + row.token) * 2 * W + (size_t)row.head * HD + (lane >> 5) * 8;
#pragma unroll
    for (int f = 0; f < P::NF; ++f) {
      qh[f] = row.there ? ld16(qp + f * 16) : zero16();
      ql[f] = row.there ? ld16(qp + W + f * 16) : zero16();
    }
  }
  const int* table = a.table + (size_t)r * z.row_pages;
  const int ngrp = (wg_end + 15) / 16, nall = (wg_end + ST - 1) / ST;
  const int per = (nall + a.nsplit - 1) / a.nsplit, st0 = split * per, nst = min(nall, st0 + per);  // stages [st0, nst)
  const size_t run = (size_t)(HD * 2) << z.lgP, page = 2 * run * z.Hk;
  const char* mine0 = (const char*)a.pool + 2 * run * kvh + (w & 1 ? run : 0);
  // wave w loads 16 slots of K (w even) or V of a stage; groups past the end read the last one again, and are never used, so
  // that every wave has the same number of loads under way
  const auto group = [&](int st) { return min(st * SR + (w >> 1), ngrp - 1); };
  const auto page_of = [&](int st) { return st0 < nst ? scalar_at(table, group(min(st, nst - 1)) * 16 >> z.lgP) : 0; };
  int id0 = page_of(st0), id1 = page_of(st0 + 1);
  const auto issue = [&](int u) {  // the loads of stage st0 + u, whose page id is there, and the id of the one after the next
    const int st = st0 + u, slot = group(st) * 16, id = checked_page(id0, z, a.err + r);
    id0 = id1;
    id1 = page_of(st + 2);
    const BufRsrc src = buf_rsrc(mine0 + (size_t)id * page + (size_t)(slot & ((1 << z.lgP) - 1)) * (HD * 2), P::RUN * 16);
    const uint32_t at = lane_anew() * 16;
    auto* dst = (__attribute__((address_space(3))) void*)(lds[u % NS] + ((w & 1) * SR + (w >> 1)) * P::RUN);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, dst, 16, at, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, dst, 16, at, 0, 1024, 0);
    if constexpr (LPW == 4) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, dst, 16, at, 0, 2048, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, dst, 16, at, 0, 3 * 1024, 0);
    }
  };

  f16v o[P::ND];
#pragma unroll
  for (int d = 0; d < P::ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float mrun = -INFINITY, lrun = 0.f;
  const float sc = 1.44269504088896341f / sqrtf((float)HD);  // scores in powers of two
  // A wave's block j: the products of the weights of block j - 1 with its V and of K with the queries, then the softmax.  So the
  // place of stage u - 1 is free again, and is loaded with stage u + 3, only in stage u + 1: two stages are on their way.
  constexpr int NBS = SR / 2 / KS;                     // blocks of a wave in a stage
  const int cnt = max(nst - st0, 0);
  const auto keys_of = [&](int u, int b) { return lds[u % NS] + 2 * (KS == 2 ? ks : b) * P::RUN; };
  const auto values_of = [&](int u, int b) { return keys_of(u, b) + SR * P::RUN; };
  const auto base_of = [&](int u, int b) { return (st0 + u) * ST + (KS == 2 ? ks : b) * P::KB; };
  const auto landed = [&](int u) {                // stage u, of which all waves' loads have arrived after this
    if (u + 1 < cnt) wait_vm_lgkm0<LPW>();
    else wait_vm_lgkm0<0>();
    asm volatile("s_barrier" ::: "memory");
  };
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (u < cnt) issue(u);
  landed(0);
  f16v s;
  u4 pp[2][3], vf[VFIRST];
  // stages whose slots every row of the wave sees, then the others (each wave by itself: the barriers are one a stage in both)
  const int full = max(0, min(cnt, wave_least / ST - st0));
  for (int j = 0; j < full * NBS; ++j) {
    const int u = j / NBS, b = j % NBS;
    if (j > 0) {
      block_values<HD>(values_of((j - 1) / NBS, (j - 1) % NBS), vf, pp, o);
      s = block_scores<HD>(keys_of(u, b), qh, ql);
      order_products<HD>();
    } else {
      s = block_scores<HD>(keys_of(u, b), qh, ql);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (b == 0 && u + 2 < cnt) issue(u + 2);  // with the products under way: before them they hold back their LDS reads
    block_weights<HD>(s, false, 0, sc, mrun, lrun, o, pp);
    first_values<HD>(values_of(u, b), vf);
    __builtin_amdgcn_sched_barrier(0);
    if (b == NBS - 1) landed(u + 1);
  }
  if (full > 0) block_values<HD>(values_of(full - 1, NBS - 1), vf, pp, o);
  // At head dim 128 the forms of four waves and of two key shares have six registers too few.  None is stored or loaded in the loop
  // above; of four waves one is loaded again in each stage below, with a wait for the stages on their way: one to five stages of a
  // workgroup, by the group.
  const int l = lane_anew(), limit = row_of(l).limit;
  int odd = 0;
  for (int u = full; u < cnt; ++u) {
    if (u + 2 < cnt) issue(u + 2);
#pragma unroll 1
    for (int b = 0; b < NBS; ++b) {
      const int base = base_of(u, b);
      if (base >= wave_end) break;
      const bool masked = base + P::KB > wave_least;
      s = block_scores<HD>(keys_of(u, b), qh, ql);
      block_weights<HD>(s, masked, limit - base, sc, mrun, lrun, o, pp);
      if (masked) {
        odd |= block_values_masked<HD>(values_of(u, b), wave_end - base, pp, o);
      } else {
        first_values<HD>(values_of(u, b), vf);
        block_values<HD>(values_of(u, b), vf, pp, o);
      }
    }
    landed(u + 1);
  }
  if (odd)  // the blocks that were masked, again: slots from the first that not all of the wave's rows see
#pragma unroll 1
    for (int st = st0 + full; st < nst; ++st)
#pragma unroll 1
      for (int b = 0; b < SR; ++b) {
        const int base = st * ST + b * 16;
        if (base / P::KB * P::KB + P::KB <= wave_least || base >= wave_end || (KS == 2 && b / 2 != ks)) continue;
        const int id = checked_page(scalar_at(table, base >> z.lgP), z, a.err + r);
        const char* v = (const char*)a.pool + (size_t)id * page + 2 * run * kvh + run + (size_t)(base & ((1 << z.lgP) - 1)) * (HD * 2);
        see_nonfinite<HD>((const u4*)v, base, limit, o);
      }
  lrun += __shfl_xor(lrun, 32, WAVE);
  if constexpr (KS == 2) {  // merge the two waves of 32 rows: the second leaves its state in LDS
    constexpr int OV = P::ND * 16;  // output values per lane
    static_assert((size_t)QT * (OV + 2) * 64 * 4 <= sizeof(lds), "merge records");
    __syncthreads();  // every wave is past its last block
    float* rec = reinterpret_cast<float*>(&lds[0][0]) + (size_t)qt * (OV + 2) * 64 + l;
    if (ks == 1) {
      rec[0] = mrun;
      rec[64] = lrun;
#pragma unroll
      for (int d = 0; d < P::ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) rec[(2 + d * 16 + e) * 64] = o[d][e];
    }
    __syncthreads();
    if (ks == 1) return;
    const float m1 = rec[0], mnew = fmaxf(mrun, m1), mz = mnew == -INFINITY ? 0.f : mnew;
    // 0 for a wave without slots; a sum that is NaN stays
    const float a0 = __builtin_amdgcn_exp2f(mrun - mz), a1 = __builtin_amdgcn_exp2f(m1 - mz);
    lrun = lrun * a0 + rec[64] * a1;
    mrun = mnew;
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = o[d][e] * a0 + rec[(2 + d * 16 + e) * 64] * a1;
  }
  const Row row = row_of(l);
  if (!row.there) return;
  if (a.nsplit > 1) {
    const size_t rec = ((size_t)blockIdx.x * a.nsplit + split) * QR + qt * 32 + (l & 31);
    float* out = a.part + rec * HD + 4 * (l >> 5);
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4)
        *reinterpret_cast<f4*>(out + d * 32 + e4 * 8) = f4{o[d][4 * e4], o[d][4 * e4 + 1], o[d][4 * e4 + 2], o[d][4 * e4 + 3]};
    if (l < 32) {
      float* ml = a.part + (size_t)gridDim.x * a.nsplit * QR * HD + 2 * rec;
      ml[0] = mrun;
      ml[1] = lrun;
    }
    return;
  }
  const float inv = lrun == 0.f ? 0.f : 1.0f / lrun;
  bf16* op = (bf16*)a.out + (size_t)(o0 + row.token) * 2 * W + (size_t)row.head * HD + 4 * (l >> 5);
#pragma unroll
  for (int d = 0; d < P::ND; ++d)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {  // columns 32 d + 8 e4 + 4 (lane >> 5) + 0..3
      float v[4], l[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = o[d][4 * e4 + e] * inv;
      const uint2 hw = uint2{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
      l[0] = v[0] - __uint_as_float(hw.x << 16);
      l[1] = v[1] - __uint_as_float(hw.x & 0xFFFF0000u);
      l[2] = v[2] - __uint_as_float(hw.y << 16);
      l[3] = v[3] - __uint_as_float(hw.y & 0xFFFF0000u);
      *reinterpret_cast<uint2*>(op + d * 32 + e4 * 8) = hw;
      *reinterpret_cast<uint2*>(op + W + d * 32 + e4 * 8) = uint2{f2bf2(l[0], l[1]), f2bf2(l[2], l[3])};
    }
}

// The splits of a share's query rows joined, a wave a row.
template <int HD, int QR>
__global__ __launch_bounds__(256) void k_paged_prompt_join(PagedAttnArgs a) {
  constexpr int V = HD / 64;
  const PagedSizes& z = a.z;
  const int lane = threadIdx.x & 63, j = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int job = (int)(blockIdx.x / (uint32_t)z.Hk), kvh = (int)(blockIdx.x % (uint32_t)z.Hk);
  __shared__ int scratch[10];
  const PromptShare s = prompt_share<QR, 256>(a, job, scratch);
  const int o = s.offset, c = s.count, i = s.at * QR + j;
  if (s.r < 0 || i >= c * z.grp) return;
  float v[V];
  join_row<HD>(a.part, a.part + (size_t)gridDim.x * a.nsplit * QR * HD, (size_t)blockIdx.x * a.nsplit * QR + j, QR, a.nsplit, v);
#pragma unroll
  for (int k = 0; k < V; ++k) Act<bf16>::put(a.out, (size_t)o + i / z.grp, z.H * HD, (kvh * z.grp + i % z.grp) * HD + lane * V + k, v[k]);
}

template <int HD, int KS, int NW>
void prompt_t(const PagedAttnArgs& a, Stream s) {
  constexpr int QR = 32 * NW / KS;
  const unsigned x = (unsigned)(paged_tiles(a.N, a.z.R, a.z.grp, QR) * a.z.Hk);
  launch_k((k_paged_prompt<HD, KS, NW>), dim3(x, a.nsplit), dim3(64 * NW), 0, s, a);
  if (a.nsplit > 1) launch_k((k_paged_prompt_join<HD, QR>), dim3(x, QR / 4), dim3(256), 0, s, a);
}

}  // namespace

int launch_paged_prompt(int hd, const PagedAttnArgs& a, int ks, int nw, Stream s) {
  if (hd == 64) ks == 2 ? prompt_t<64, 2, 8>(a, s) : nw == 8 ? prompt_t<64, 1, 8>(a, s) : prompt_t<64, 1, 4>(a, s);
  else if (hd == 128) ks == 2 ? prompt_t<128, 2, 8>(a, s) : nw == 8 ? prompt_t<128, 1, 8>(a, s) : prompt_t<128, 1, 4>(a, s);
  else return -1;
  return 0;
}

}  // namespace ham
