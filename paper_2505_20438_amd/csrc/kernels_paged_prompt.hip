// Causal attention of packed bf16 prompts over their pages (layout: kernels_paged.h).
//
// A row's c tokens times the grp q-heads of a kv head are c * grp query rows in the order of the tokens; 32 of them, whatever
// the group, are one wave's operand.  A workgroup of eight waves has QR = 256 / KS of them, its waves' keys in KS shares; 64 slots
// at a time land in LDS straight from the pages, in the order of the pool, which is that of the operands.  Both products are
// 32x32x16 matrix instructions with the query row in the lane index:
//   S^T = K Q^T (A = K rows, B = Q rows)  and  O^T = V^T P^T (A = V^T rows, B = P rows),
// so a lane (row l & 31, half l >> 5) holds scores, weights, softmax state and output columns of one row and only the other half
// shares it.  The running maximum moves, and with it the outputs, only when a score exceeds it by more than 8 powers of two.
// Masks, and values past the slots that a wave sees, are dealt with only in blocks that reach past the wave's first row.
#include "gemm_epilogue.h"
#include "launch_rules.h"
#include "paged_device.h"

namespace ham {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

template <int HD> struct PP {
  static constexpr int NW = 8, KB = 32, ST = 64, NS = 4;           // waves; slots of a block, of a stage; stages in the ring
  static constexpr int RUN = 2 * HD, STAGE = 8 * RUN;              // 16-byte units of 16 slots of K or V; of a stage: 4 K, 4 V
  static constexpr int LPW = RUN / 64;                             // a wave's loads of a stage: one run
  static constexpr int NF = HD / 16, ND = HD / 32;
};

// One block of 32 slots from `base` for this wave's 32 rows.  MASK: slots at or past `limit` (the lane's row) count as
// -infinity, and values at or past `vlimit` as 0, whatever they hold.  `load(j)`, j < NLD, issues this wave's loads of a later
// stage, spread among the products.
template <int HD, bool MASK, int NLD, typename Load>
__device__ __forceinline__ void prompt_block(const u4* kblk, const u4* vblk, int base, int limit, int vlimit, const u4* qh, const u4* ql,
                                             float sc, float& mrun, float& lrun, f16v* o, const Load& load) {
  using P = PP<HD>;
  const int lane = threadIdx.x & 63, h = lane >> 5, r = lane & 31;
  f16v s;
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = 0.f;
  __builtin_amdgcn_s_setprio(1);  // products before the other wave's softmax
  const u4* kr = kblk + (r >> 4) * P::RUN + h * 16 + (r & 15);
#pragma unroll
  for (int f = 0; f < P::NF; ++f) {
    const bf16x8 k = __builtin_bit_cast(bf16x8, kr[f * 32]);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, __builtin_bit_cast(bf16x8, qh[f]), s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, __builtin_bit_cast(bf16x8, ql[f]), s, 0, 0, 0);
    if (NLD > 0 && f % (P::NF / (NLD > 0 ? NLD : 1)) == 0) {
      __builtin_amdgcn_sched_barrier(0);
      load(f / (P::NF / (NLD > 0 ? NLD : 1)));
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_setprio(0);
  if constexpr (MASK) {
#pragma unroll
    for (int e = 0; e < 16; ++e)  // score e: slot 16 (e / 8) + 8 h + e % 8
      if (base + 16 * (e >> 3) + 8 * h + (e & 7) >= limit) s[e] = -INFINITY;
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
  u4 pp[2][3];
  to_planes<3>(p, pp[0]);
  to_planes<3>(p + 8, pp[1]);
  const u4* vr = vblk + h * HD + r;  // channels 32 d + r of slots 16 t + 8 h ..
  if constexpr (MASK) {
    u4 seen[2];
    bool odd = false;
    const auto value = [&](int d, int t) {
      u4 v = vr[t * P::RUN + d * 32];
      const int keep = vlimit - (base + 16 * t + 8 * h);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= keep) v[e >> 1] &= (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
      return v;
    };
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        odd |= any_nonfinite<bf16>(value(d, t));
    const bool fix = __any(odd);
    if (fix)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int s0 = base + 16 * t + 8 * h + 2 * i;
          seen[t][i] = (s0 < limit ? 0x3F80u : 0u) | (s0 + 1 < limit ? 0x3F800000u : 0u);
        }
#pragma unroll
    for (int d = 0; d < P::ND; ++d) {
      u4 v[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) v[t] = value(d, t);
      if (fix) {
        f16v cu, cd;
#pragma unroll
        for (int e = 0; e < 16; ++e) cu[e] = cd[e] = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          u4 up, down;
          split_nonfinite<bf16>(v[t], up, down);
          cu = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, up), __builtin_bit_cast(bf16x8, seen[t]), cu, 0, 0, 0);
          cd = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, down), __builtin_bit_cast(bf16x8, seen[t]), cd, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] += seen_nonfinite(cu[e], cd[e]);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 3; ++i)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[t]), __builtin_bit_cast(bf16x8, pp[t][i]), o[d], 0, 0, 0);
    }
  } else {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8 v = __builtin_bit_cast(bf16x8, vr[t * P::RUN + d * 32]);
#pragma unroll
        for (int i = 0; i < 3; ++i)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, pp[t][i]), o[d], 0, 0, 0);
      }
    __builtin_amdgcn_s_setprio(0);
  }
}

// The rows' shares of QR query rows: those of the row with the most slots first, and of a row the last first (its keys are the
// most), so that the workgroups that take longest start first.  Rows past the 64th in the order they have.
template <int QR>
__device__ __forceinline__ Share prompt_share(const PagedAttnArgs& a, int i) {
  const int R = a.z.R, lane = threadIdx.x & 63;
  const auto need = [&](int r) { return max(0, (prompt_count(a, r) * a.z.grp + QR - 1) / QR); };
  Share s{-1, 0};
  int n = 0;
  if (R <= 64) {
    n = lane < R ? need(lane) : 0;
    const int key = lane < R ? a.kv_len[lane] : -1;
    int before = 0;
    for (int j = 0; j < R; ++j) {
      const int kj = __builtin_amdgcn_readlane(key, j), nj = __builtin_amdgcn_readlane(n, j);
      before += kj > key || (kj == key && j < lane) ? nj : 0;
    }
    const uint64_t hit = __ballot(i >= before && i < before + n);
    if (hit == 0) return s;
    s.r = __builtin_ctzll(hit);
    n = __builtin_amdgcn_readlane(n, s.r);
    s.at = n - 1 - (i - __builtin_amdgcn_readlane(before, s.r));
    return s;
  }
  s = find_share(R, i, need);
  if (s.r >= 0) s.at = need(s.r) - 1 - s.at;
  return s;
}

template <int HD, int KS>
__global__ __launch_bounds__(512, 2) void k_paged_prompt(PagedAttnArgs a) {
  using P = PP<HD>;
  constexpr int NS = P::NS, LPW = P::LPW, QT = P::NW / KS, QR = 32 * QT;
  __shared__ u4 lds[NS][P::STAGE];
  const PagedSizes& z = a.z;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int job = (int)(blockIdx.x / (uint32_t)z.Hk), kvh = (int)(blockIdx.x % (uint32_t)z.Hk), split = blockIdx.y;
  if (blockIdx.x == 0 && split == 0)
    for (int i = threadIdx.x; i < z.R; i += 512)
      if (prompt_count(a, i) < 0) atomicOr(a.err + i, 8);
  const Share sh = prompt_share<QR>(a, job);
  if (sh.r < 0) return;
  const int r = sh.r, o0 = a.offsets[r], c = a.offsets[r + 1] - o0, n = a.kv_len[r], held = n - c;
  const int qt = w % QT, ks = w / QT;
  const int i0 = sh.at * QR + qt * 32, i1 = min(i0 + 32, c * z.grp);  // this wave's rows [i0, i1), of c * grp
  const bool rows_ok = i0 < c * z.grp;
  const int wave_least = rows_ok ? held + i0 / z.grp + 1 : 0, wave_end = rows_ok ? held + (i1 - 1) / z.grp + 1 : 0;
  const int wg_end = held + (min(sh.at * QR + QR, c * z.grp) - 1) / z.grp + 1;
  const int i = i0 + (lane & 31);
  const bool qok = i < c * z.grp;
  const int tok = qok ? i / z.grp : 0, head = kvh * z.grp + (qok ? i % z.grp : 0), limit = qok ? held + tok + 1 : 0;
  const int W = z.H * HD;
  const size_t q_row = (size_t)o0 + tok;
  u4 qh[P::NF], ql[P::NF];
  {
    const bf16* qp = (const bf16*)a.q + q_row * 2 * W + (size_t)head * HD + (lane >> 5) * 8;
#pragma unroll
    for (int f = 0; f < P::NF; ++f) {
      qh[f] = qok ? ld16(qp + f * 16) : zero16();
      ql[f] = qok ? ld16(qp + W + f * 16) : zero16();
    }
  }
  const int* table = a.table + (size_t)r * z.row_pages;
  const int ngrp = (wg_end + 15) / 16, nall = (wg_end + P::ST - 1) / P::ST;
  const int per = (nall + a.nsplit - 1) / a.nsplit, st0 = split * per, nst = min(nall, st0 + per);  // stages [st0, nst)
  const size_t run = (size_t)(HD * 2) << z.lgP, page = 2 * run * z.Hk;
  const char* mine0 = (const char*)a.pool + 2 * run * kvh + (w & 1 ? run : 0) + lane * 16;
  // wave w loads 16 slots of K (w even) or V of a stage; groups past the end read the last one again, and are never used, so
  // that every wave has the same number of loads under way
  const auto group = [&](int st) { return min(st * 4 + (w >> 1), ngrp - 1); };
  int next_id = st0 < nst ? table[group(st0) * 16 >> z.lgP] : 0;
  const char* src = mine0;
  const auto locate = [&](int st) {  // the page of stage st, whose id is there, and the id of the stage after it
    const int slot = group(st) * 16, id = checked_page(__builtin_amdgcn_readfirstlane(next_id), z, a.err + r);
    src = mine0 + (size_t)id * page + (size_t)(slot & ((1 << z.lgP) - 1)) * (HD * 2);
    next_id = table[group(min(st + 1, nst - 1)) * 16 >> z.lgP];
  };
  const auto issue1 = [&](int st, int j) {
    __builtin_amdgcn_global_load_lds((const void*)(src + j * 1024),
                                     (__attribute__((address_space(3))) void*)(lds[st % NS] + ((w & 1) * 4 + (w >> 1)) * P::RUN + j * 64), 16, 0, 0);
  };

  f16v o[P::ND];
#pragma unroll
  for (int d = 0; d < P::ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float mrun = -INFINITY, lrun = 0.f;
  const float sc = 1.44269504088896341f / sqrtf((float)HD);  // scores in powers of two
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (st0 + s < nst) {
      locate(st0 + s);
#pragma unroll
      for (int j = 0; j < LPW; ++j) issue1(st0 + s, j);
    }
  for (int st = st0; st < nst; ++st) {
    // stage st has landed once at most the loads of the stages issued after it are pending
    if (st + NS - 2 < nst) wait_vm_lgkm0<(NS - 2) * LPW>();
    else wait_vm_lgkm0<0>();
    asm volatile("s_barrier" ::: "memory");
    // every wave is past stage st - 1: its place takes stage st + NS - 1
    constexpr int NB = 2 / KS, NLD = LPW / NB;  // blocks of this wave, loads issued in each
    const bool more = st + NS - 1 < nst;
    if (more) locate(st + NS - 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int bi = KS == 2 ? ks : b, base = st * P::ST + bi * P::KB;
      const u4 *kb = lds[st % NS] + 2 * bi * P::RUN, *vb = kb + 4 * P::RUN;
      const auto load = [&](int j) {
        if (more) issue1(st + NS - 1, b * NLD + j);
      };
      if (rows_ok && base + P::KB <= wave_least) {  // every slot visible to every row
        prompt_block<HD, false, NLD>(kb, vb, base, limit, wave_end, qh, ql, sc, mrun, lrun, o, load);
      } else if (base < wave_end) {
        prompt_block<HD, true, NLD>(kb, vb, base, limit, wave_end, qh, ql, sc, mrun, lrun, o, load);
      } else {  // blocks past this wave's last row hold nothing it sees
#pragma unroll
        for (int j = 0; j < NLD; ++j) load(j);
      }
    }
  }
  lrun += __shfl_xor(lrun, 32, WAVE);
  if constexpr (KS == 2) {  // merge the two waves of 32 rows: the second leaves its state in LDS
    constexpr int OV = P::ND * 16;  // output values per lane
    static_assert((size_t)QT * (OV + 2) * 64 * 4 <= sizeof(lds), "merge records");
    __syncthreads();  // every wave is past its last block
    float* rec = reinterpret_cast<float*>(&lds[0][0]) + (size_t)qt * (OV + 2) * 64 + lane;
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
  if (!qok) return;
  if (a.nsplit > 1) {
    const size_t rec = ((size_t)blockIdx.x * a.nsplit + split) * QR + qt * 32 + (lane & 31);
    float* out = a.part + rec * HD + 4 * (lane >> 5);
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4)
        *reinterpret_cast<f4*>(out + d * 32 + e4 * 8) = f4{o[d][4 * e4], o[d][4 * e4 + 1], o[d][4 * e4 + 2], o[d][4 * e4 + 3]};
    if (lane < 32) {
      float* ml = a.part + (size_t)gridDim.x * a.nsplit * QR * HD + 2 * rec;
      ml[0] = mrun;
      ml[1] = lrun;
    }
    return;
  }
  const float inv = lrun == 0.f ? 0.f : 1.0f / lrun;
  bf16* op = (bf16*)a.out + q_row * 2 * W + (size_t)head * HD + 4 * (lane >> 5);
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
  const Share s = prompt_share<QR>(a, job);
  if (s.r < 0) return;
  const int o = a.offsets[s.r], c = a.offsets[s.r + 1] - o, i = s.at * QR + j;
  if (i >= c * z.grp) return;
  float v[V];
  join_row<HD>(a.part, a.part + (size_t)gridDim.x * a.nsplit * QR * HD, (size_t)blockIdx.x * a.nsplit * QR + j, QR, a.nsplit, v);
#pragma unroll
  for (int k = 0; k < V; ++k) Act<bf16>::put(a.out, (size_t)o + i / z.grp, z.H * HD, (kvh * z.grp + i % z.grp) * HD + lane * V + k, v[k]);
}

template <int HD, int KS>
void prompt_t(const PagedAttnArgs& a, Stream s) {
  constexpr int QR = 256 / KS;
  const unsigned x = (unsigned)(paged_tiles(a.N, a.z.R, a.z.grp, QR) * a.z.Hk);
  launch_k((k_paged_prompt<HD, KS>), dim3(x, a.nsplit), dim3(512), 0, s, a);
  if (a.nsplit > 1) launch_k((k_paged_prompt_join<HD, QR>), dim3(x, QR / 4), dim3(256), 0, s, a);
}

}  // namespace

int launch_paged_prompt(int hd, const PagedAttnArgs& a, int ks, Stream s) {
  if (hd == 64) ks == 2 ? prompt_t<64, 2>(a, s) : prompt_t<64, 1>(a, s);
  else if (hd == 128) ks == 2 ? prompt_t<128, 2>(a, s) : prompt_t<128, 1>(a, s);
  else return -1;
  return 0;
}

}  // namespace ham
