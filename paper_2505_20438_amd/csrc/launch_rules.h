// Launch rules that depend on sizes alone, without a GPU or a HIP header, so that they can be checked by themselves.
#pragma once
#include <algorithm>

namespace ham {

constexpr int MAX_ATTN_SPLIT = 64;

// Slot splits of the filled-cache attention for R rows of Hk kv heads of which the longest has kv_max slots: none while
// the keys of a (row, kv head) are under 128 KB (one workgroup then reads them about as fast as the extra combine
// launch, 4 us, takes), else the count with the least estimated time for rows of equal length, two key blocks or more
// each.  One workgroup runs per CU, so R * Hk * splits workgroups take ceil(... / 256) rounds; a workgroup needs 3.4 us
// and, per 32 slots of head dim 128 in bf16 (16 KB), 0.42 us alone and 0.59 with all 256 at work.  That takes splits whose
// last round is full.  8 kv heads of 128 in bf16, us at 256 / (R * Hk) splits rounded down and at the splits here: 12 rows x
// 4,096 slots 44.3 / 42.8, 17 x 8,192 131 / 105, 20 x 4,096 72 / 64, 24 x 32K 540 / 476, 40 x 4,096 150 / 124, 48 x 8,192
// 287 / 257; the same where 256 workgroups come out even (1 x 2,048 10.4, 8 x 4,096 29, 32 x 4,096 87, 4 x 32K 89).
// A row's slots are shared by its own splits alone, so a long row among short ones is a serial chain.  From 2 MB of keys
// (8,192 such slots: 111 us unsplit) a row gets at least two rounds' share, up to 8 splits.  One row of 32K slots and the
// rest of 500: 8 rows 126 -> 75 us, 20 rows 444 -> 75, 40 rows 445 -> 129; where all are long this costs up to a tenth (10 x
// 8,192 61 -> 67 us, 5 x 8,192 35 -> 37, 16 x 8,192 89 -> 97, 32 x 8,192 165 -> 174, 8 x 32K 169 -> 177).
inline int attn_decode_splits(int dtype, int R, int Hk, int hd, int kv_max) {
  const int es = dtype == 1 ? 2 : 4, kb = dtype == 1 ? 32 : 16;
  const long long keys = (long long)kv_max * hd * es, pairs = (long long)R * Hk;
  if (keys < 128 * 1024) return 1;
  const int blocks = (kv_max + kb - 1) / kb, most = std::max(1, std::min((blocks + 1) / 2, MAX_ATTN_SPLIT));
  int least = 1;
  if (keys >= 2 * 1024 * 1024) least = (int)std::min({(512 + pairs - 1) / pairs, 8ll, (long long)most});
  int best = least;
  double best_t = 1e30;
  for (int s = least; s <= most; ++s) {
    const double rounds = (double)((pairs * s + 255) / 256), last = (double)(pairs * s) / 256 - (rounds - 1);
    const double units = (double)((blocks + s - 1) / s) * hd / 128;  // of 16 KB
    const double t = rounds * 3.4 + units * (0.59 * (rounds - 1) + 0.42 + 0.17 * last) + (s > 1 ? 4 : 0);
    if (t < best_t) {
      best_t = t;
      best = s;
    }
  }
  return best;
}

// Whether k_gemm_rows takes a bf16 projection of M rows and N columns (k range a multiple of 128).  It runs one workgroup
// of 128 columns per CU, so its time grows by rounds of 256 where k_gemm_wide's grows with the columns: a second round
// has to be an eighth full at up to 16 rows and a quarter full at 32, and at 32 rows a fourth does not pay.  Gate/up, us,
// k_gemm_wide with the reduction of its splits / k_gemm_rows: k 4,096, 32 rows: 224 groups of columns 51 / 45, 260 73 / 79,
// 288 76 / 80, 320 85 / 81, 520 131 / 125, 768 170 / 145, 780 173 / 174; 16 rows: 260 71 / 69, 288 76 / 71, 780 166 / 153;
// k 8,192, 32 rows: 260 130 / 150, 288 139 / 153, 320 152 / 154, 448 201 / 175, 780 316 / 334; 16 rows: 260 126 / 134,
// 288 140 / 134.
constexpr int ROWS_MAX_M = 32;
inline bool gemm_rows_takes(int M, int N) {
  if (M <= 8 || M > ROWS_MAX_M) return false;
  const int groups = (N + 127) / 128;
  if (groups > 256 && groups < 512) return groups >= (M <= 16 ? 288 : 320);
  return M <= 16 || groups <= 768;
}

// Grid of the bf16 prompt attention (kernels_attn_prompt.hip): `blocks` x kv heads x `seqs` workgroups of eight waves, for
// R rows from input s0 of a sequence on, through sequences of T inputs.  Tiles of 32 rows; `blocks` covers the longest share
// of a sequence.  The keys form while the rows form would give no more than every other CU a workgroup (one sequence,
// rows / keys form: 512 rows of the 1B shape 20.2 / 17.0 us, 1,024 rows 35.5 / 28.7 and of the 8B shape 54.7 / 46.1; above
// that the rows form wins: 2,048 rows 68.9 / 96.0 and 99.4 / 142.5).
constexpr int PROMPT_ATTN_WAVES = 8, PROMPT_ATTN_KEYS_MAX_WGS = 128;
struct PromptAttnGrid {
  int blocks, seqs;
  bool keys;
};
inline PromptAttnGrid prompt_attn_grid(int R, int s0, int T, int H, int Hkv) {
  const int seqs = (s0 + R - 1) / T + 1, tiles = (std::min(R, T) + 31) / 32;
  const int half = PROMPT_ATTN_WAVES / (H / Hkv) / 2;  // row tiles of a workgroup: 2 * half (rows form) or half
  const int rows_blocks = ((tiles + 1) / 2 + half - 1) / half;
  const bool keys = (long)rows_blocks * Hkv * seqs <= PROMPT_ATTN_KEYS_MAX_WGS;
  return PromptAttnGrid{keys ? (tiles + half - 1) / half : rows_blocks, seqs, keys};
}

// Splits of the attention over the 8-bit cache for R rows of Hk kv heads of which the longest reads `blocks` blocks of 32
// slots.  Workgroups of 8 waves, two a CU (as a bf16 model's with up to 8 q-heads a kv head at head dim 128; with 9 to 16, or in
// fp32, registers or LDS leave one there, and at head dim 64 three fit: for those the rule is the same and was not fitted).
// Their 8 blocks (one a wave) take 1.14 us at head dim 128 and 0.75 at 64 alone
// and half as much again with all 256 CUs at work, as long again for the second workgroup of a CU, but no less than their
// share of memory: a block of every CU's takes 0.30 us (7 TB/s; 5% less at three CUs of four) at 128, half at 64.  R * Hk *
// splits workgroups take ceil(... / 512) rounds, the first 5.4 us (4 at head dim 64) and the others 2 beside that, and a split
// launch 2.5 us more for the combine.  The count with the least estimate, the lowest of equal ones.
// 8 kv heads of 128, us at the splits here / at 256 / (R * Hk) rounded up: 4 rows x 33,300 slots 45.1 / 46.6, 5 x 33,300
// 54 / 71, 12 x 4,096 21 / 27, 20 x 4,096 28 / 37, 40 x 4,096 58 / 62 (and unsplit: 1 x 1,000 9.0 / 10.0, 4 x 64 listed blocks
// 10.5 / 15.3).  At 23 shapes the best of 1 .. 48 splits was at most 3% below it.
// A row's blocks are shared by its own splits alone, so a long row among short ones is a serial chain (1,040 blocks 153 us
// unsplit, 46 in four): from 512 blocks on a row gets one split for every 256, up to four; where all rows are long that
// costs up to a twentieth (32 x 33,300 314 -> 326).
constexpr int KV8_MOST_WGS = 1024;  // workgroups of a split launch, unless four splits of every pair are more
inline int kv8_attn_splits(int R, int Hk, int hd, int blocks) {
  const long long pairs = (long long)R * Hk;
  const int least = std::max(1, std::min(4, blocks / 256));
  const int most = (int)std::max<long long>(least, std::min<long long>({(blocks + 7) / 8, KV8_MOST_WGS / pairs, MAX_ATTN_SPLIT}));
  const double wave = hd == 128 ? 1.14 : 0.75, share = hd == 128 ? 0.30 : 0.15, rest = hd == 128 ? 5.4 : 4.0;
  int best = least;
  double best_t = 1e30;
  for (int s = least; s <= most; ++s) {
    const int u = (blocks + s - 1) / s;
    const long long rounds = (pairs * s + 511) / 512;
    const auto time = [&](long long wgs) {
      const double fill = (double)wgs / 256, busy = std::min(fill, 1.0);
      return std::max(wave * (1 + 0.55 * busy) * ((wgs + 255) / 256) * ((u + 7) / 8), share * (0.85 + 0.15 * busy) * u * fill);
    };
    const double t = rest + (rounds - 1) * (2 + time(512)) + time(pairs * s - (rounds - 1) * 512) + (s > 1 ? 2.5 : 0);
    if (t < best_t - 1e-9) {
      best_t = t;
      best = s;
    }
  }
  return best;
}

// Append of N packed tokens of R rows: steps of 32 aligned slots at most, and workgroups a step, whose heads (kv heads, and with q
// as many more for their q-heads) they take in turn.  Up to 64 rows one a head; with more of them, finding a step's row costs a
// workgroup as much as a head's values do, so that their number is kept to APPEND_MANY.  Rows of a token, 8 kv heads of 128, us, at
// most 8,192 / 4,096 / 2,048 of them: 256 rows 15 / 15 / 12, 512 28 / 19 / 16, 1,024 35 / 27 / 25, 4,096 134 / 119 / 119.
inline long long paged_append_steps(long long N, long long R) { return std::min(N, (N + 62 * R) / 32); }
constexpr int APPEND_MANY = 2048;
inline int paged_append_groups(int N, int R, int heads) {
  return R <= 64 ? heads : (int)std::max<long long>(1, std::min<long long>(heads, APPEND_MANY / paged_append_steps(N, R)));
}
// Workgroups of a launch: steps in eights, one for each XCD.  A launch has fewer than 2^24 workgroups of 256 threads; a call of up to
// 2^27 (token, kv head) pairs stays below: up to 64 rows N / 32 + 132 steps at most, of 2 Hk heads, and with more rows a step has
// one workgroup as soon as there are many.
inline long long paged_append_workgroups(int N, int R, int heads) { return (paged_append_steps(N, R) + 7) / 8 * 8 * paged_append_groups(N, R, heads); }
inline bool paged_append_fits(long long N, int Hk) { return N * Hk <= 1 << 27; }

// Shares of `width` (token, q-head) pairs, at most, of N packed tokens of R rows with grp <= width q-heads a kv head: a row's
// last share may be partly filled, and a share has a token at least.
inline long long paged_tiles(long long N, long long R, long long grp, long long width) {
  return std::min(N, (N * grp + (width - 1) * R) / width);
}

// Attention of one token over pages (kernels_paged.hip): whether its slots are split over workgroups, which a second launch then
// joins, for R rows of which the longest has kv_max slots, in blocks of 16 KB (head dim 128) of K and V.  A workgroup of four
// waves takes about 5 us and 0.6 us for each four blocks, a join 3 to 5.  Split / not, us: 1 row of 2,000 slots of 8 heads of 128
// 9.7 / 14.8, 8 x 1,000 10.8 / 10.4, 8 x 500 9.5 / 6.9, 1 x 700 of 64 8.1 / 6.4.  With more workgroups memory is busy without
// splits while all rows are long, and they pay for rows of different lengths: (row, kv head) pairs of 80 blocks each / of 80 down
// to 20: bf16 96 27.7 / 29.7 and 19.5 / 28.4, 128 35.2 / 34.6 and 23.2 / 29.2, 160 46.0 / 38.1 and 28.1 / 30.4; of 48 blocks 128
// 25.1 / 22.7 and 17.3 / 19.1; fp32 of head dim 64, of 80 blocks, 160 44.4 / 45.7 and 28.6 / 40.3, 192 52.3 / 47.0 and 32.5 /
// 40.2. Past 128 blocks a long row among short ones would hold its workgroup for more than 25 us.  With hundreds of rows, finding
// a share's row costs every workgroup more and short rows hide a longer one: 512 rows of 300 slots and one of 8,000 183 / 153, one
// of 33,000 193 / 365; 512 of 5,000 1,615 / 1,570.  The records of a split launch have room for PAGED_SPLIT_MAX_HEADS (row,
// q-head) pairs.
constexpr int PAGED_SPLIT_MAX_HEADS = 16384;
inline bool paged_attn_split(int R, int H, int Hk, int hd, int kv_max, int block) {
  const int blocks = (kv_max + block - 1) / block * hd / 128, pairs = R * Hk;
  if (R * H > PAGED_SPLIT_MAX_HEADS) return false;
  const int few = block == 16 ? 160 : blocks > 60 ? 128 : 95;  // blocks of 16 slots: fp32
  return blocks > 28 && (pairs <= few || blocks > (R > 256 ? 512 : 128));
}
// Shares that the slots of all rows are cut into, for each kv head: workgroups for one, or with more rows up to four, whole rounds
// over the CUs (at 8 kv heads a round is 32; rows of so many slots down to 0.8 times as many, us: 4 x 33,300 24 shares 78, 32 77, 40 93,
// 48 85, 64 77, 72 89; 16 x 8,300 32 shares 92, 64 79, 96 84; 48 x 8,300 32 257, 64 237, 96 225, 128 228).  No share is less than
// PAGED_LEAST_BLOCKS, two for each of the four waves.
constexpr int PAGED_LEAST_BLOCKS = 8;
inline int paged_attn_shares(int R, int Hk) { return std::max(1, 256 * std::min(4, 1 + R * Hk / 128) / Hk); }
// Blocks of a share, where R rows have `all` together and the longest `most`: R + shares workgroups do for all rows, and no row has
// more than PAGED_MAX_SPLIT of them.  4,096 rows of 2^24 slots are 2^32 blocks of 16: the sum has 64 bits, the division 32, for which
// 2^32 counts as one less (that gives no share more: with shares of ceil((2^32 - 1) / n) blocks, 2^32 hold n whole ones at most).
constexpr int PAGED_MAX_SPLIT = 64;  // splits of a row's slots (the join holds one a lane)
constexpr int paged_share_size(long long all, int most, int R, int shares) {
  const unsigned whole = (unsigned)(shares - (R < shares / 2 ? R : shares / 2));  // the rows' ends are shares too
  const unsigned n = all < 0xFFFFFFFFll ? (unsigned)all : 0xFFFFFFFFu;
  const int size = (int)(n / whole + (n % whole != 0)), least = (most + PAGED_MAX_SPLIT - 1) / PAGED_MAX_SPLIT;
  return size < least ? (least < PAGED_LEAST_BLOCKS ? PAGED_LEAST_BLOCKS : least) : size < PAGED_LEAST_BLOCKS ? PAGED_LEAST_BLOCKS : size;
}

// Packed rows, two kernels.  k_paged_attn takes (token, q-head) pairs 16 at a time, each tile's keys shared by four waves that
// read them for themselves; k_paged_prompt (bf16) takes 256 or 128, whose keys go through LDS once.  The first fills the card with
// few tokens, the second does with a sixteenth of the reads.  8 kv heads of 128, 4 q-heads each, us, first / second: 1 row of 64 tokens
// 7 / 15, of 512 21 / 28, of 1,024 45 / 44, of 1,500 77 / 60; 4 x 300 41 / 31, 4 of 300 down to 38 21 / 22, 32 of 77 down to 10 34 / 23;
// behind 8,000 slots 8 tokens 16 / 26, 128 51 / 52, 256 90 / 84; behind 33,000 32 tokens 56 / 66, 64 96 / 76; 64 rows of a token behind
// 0 to 2,000 slots 43 / 79, behind 2,000 each 93 / 108.
inline bool paged_prompt_tiles(int N, int R, int Hk, int grp, int kv_max) {
  const long long wgs = paged_tiles(N, R, grp, 16) * Hk;
  return (long long)N * grp <= 32ll * R || (wgs <= 2048 && wgs * kv_max <= 1600 * 2048);
}
// ... and where the second takes a call of several rows, those of up to so many pairs are the first's all the same: a new token among
// prompts would hold a workgroup of the second for all its slots (7 rows of one token behind 8,000 slots and a prompt of 2,000: 275 us
// in the second alone, 181 in both, the prompt by itself 95; 31 such rows 384 and 333).
constexpr int PAGED_FEW = 32;
// Splits of a tile's slots: two workgroups a CU, eight blocks of `block` slots at least each.
inline int paged_tile_splits(long long tiles, int Hk, int kv_max, int block) {
  const long long pairs = tiles * Hk;
  const int blocks = (kv_max + block - 1) / block;
  const long long most = std::max<long long>(1, std::min<long long>({(blocks + 7) / 8, 1024 / pairs, 64}));
  return (int)std::min<long long>(most, std::max<long long>(1, 512 / pairs));
}
// k_paged_prompt: shares of the keys among a workgroup's waves (2: twice the workgroups, half the rows each), splits of them over
// workgroups, waves of a workgroup: 8, or (1 share) 4, of which two are on a CU and begin and end at times of their own, but load the
// keys twice.  Splits (2 shares), us: 512 tokens behind 8,000 slots 241 unsplit, 156 in two, 163 in four; 128 227, 52 in eight, 64 in
// 16; 64 behind 33,000 730, 76 in 16, 91 in 32.  2 shares / 1 of 4 waves, up to one round of workgroups of 256 rows: 1,500 tokens from the
// first 68 / 78, 2,048 100 / 104, 2 x 700 47 / 48, 1,000 behind 4,000 slots 180 / 207; but 4 x 400 49 / 42, 5 x 300 45 / 37, 1,500 behind
// 4,000 300 / 270, 6 x 250 276 / 247.  8 waves / 4, `rounds` of the 8's: 2,048 behind 30,720 (1) 1,895 / 1,960, 1,500 behind 16,000 (0.7)
// 835 / 900 (but of head dim 64 1,184 / 1,148 and 571 / 506), 32 x 60 (0.9) 34 / 31; from the first 2,500 (1.2) 161 / 141, 3,000 (1.5)
// 190 / 178, 3,500 (1.7) 229 / 239, 4,000 (2) 302 / 309, 5,000 (2.4) 452 / 428, 6,000 (2.9) 621 / 597, 16,000 (7.8) 3,939 / 3,959,
// 16 x 1,000 (7.8) 417 / 400, 8 x 600 (2.3) 105 / 94; 4,000 of head dim 64 (2) 179 / 167.
struct PagedPromptGrid {
  int shares, splits;
};
inline PagedPromptGrid paged_prompt_grid(int N, int R, int Hk, int grp, int kv_max) {
  const long long wide = paged_tiles(N, R, grp, 256) * Hk, narrow = paged_tiles(N, R, grp, 128) * Hk;
  const bool alike = N < kv_max / 2 || N / 2 > kv_max;  // most slots are held already, or several rows: no long rows to pair with short
  if (wide > 256 || (wide > 128 && (kv_max > 8192 || alike))) return PagedPromptGrid{1, 1};
  const long long stages = (kv_max + 63) / 64;
  return PagedPromptGrid{2, (int)std::max<long long>(1, std::min<long long>({256 / narrow, stages / 4, 32}))};
}
inline int paged_prompt_waves(int N, int Hk, int grp, int hd, int kv_max) {  // of 1 share
  const double rounds = (double)N * grp * Hk / (256 * 256);
  return (rounds <= 1 && kv_max > 8192) || (hd == 128 && rounds > 1.5 && rounds <= 2) ? 8 : 4;
}

}  // namespace ham
