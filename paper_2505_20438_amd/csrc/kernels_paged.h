// Argument blocks, layout and launchers of the operators on a paged KV cache (kernels_paged.hip, kernels_paged_prompt.hip; host
// side paged.cpp).
#pragma once
#include "ham_internal.h"

namespace ham {

constexpr int PAGED_MAX_GROUP = 16;   // q-heads of a kv head: the columns of a 16-wide matrix product
constexpr int PAGED_MAX_RECORDS = 1 << 15;  // query rows times splits of a split launch (launch_rules.h keeps below it)

// A layer's pool is [n_pages][n_kv_heads][2: K, V][P * hd] values of the storage type.  With E = 16 bytes of values:
//   K: 16 slots after 16, of each E channels after E, of each the slots in the order of the matrix cores' operand rows (bits
//      2 and 3 of the slot swapped): the scores of K Q^T then lie in the registers from which P V takes its probabilities, and
//      a wave's operand loads are runs of 128 bytes (16-row products) or 256 (32-row);
//   V: E slots after E, each channel's E slots together.
// 16 slots of K, or of V, are one run of 16 * hd values, so a page may have any multiple of 16 slots.
__host__ __device__ __forceinline__ int paged_k_place(int s) { return (s & 3) | (s & 4) << 1 | (s & 8) >> 1; }  // of slot s < 16
template <int E> __host__ __device__ __forceinline__ int paged_k_index(int s, int d, int hd) {
  return ((s / 16 * (hd / E) + d / E) * 16 + paged_k_place(s % 16)) * E + d % E;
}
template <int E> __host__ __device__ __forceinline__ int paged_v_index(int s, int d, int hd) { return (s / E * hd + d) * E + s % E; }

struct PagedSizes {
  int R, H, Hk, grp;                 // grp = H / Hk
  int lgP, n_pages, row_pages;       // slots of a page, 2^lgP
};
struct PagedAppendArgs {
  PagedSizes z;
  int N;                             // packed tokens
  const float* qkv; const float* cos; const float* sin;
  const int* offsets; const int* start; const int* table;
  void* pool; void* q;               // q: act rows, or null
  int per_step;                      // workgroups of 32 slots
  int* err;
};
struct PagedAttnArgs {
  PagedSizes z;
  int N, kv_max, nsplit;             // N: packed query rows; nsplit: splits of a tile, or (one row per sequence) 0 or the
                                     // shares of all rows
  int few;                           // packed rows of up to so many (token, q-head) pairs are k_paged_attn's, those of more
                                     // k_paged_prompt's
  const void* q; void* out;          // act rows
  const void* pool;
  const int* offsets;                // of the packed rows, or null: one query row per sequence
  const int* table; const int* kv_len; const int* enable;
  int* err;
  float* part;                       // records of the splits: outputs [tile][nsplit][rows of a tile][hd], then (max, sum)
};
struct PagedAdvanceArgs {
  PagedSizes z;
  const int* parent;                 // or null
  const int* count;
  int* kv_len; int* start; int* table; int* refs;
  int* err;
  // workspace, int32: what the rows take over (with parent), lengths and table entries to write back, page lists
  int* taken; int* taken_len; int* span;
  int* owner;                        // [n_pages][2]: writers of a shared page, the lowest of them
  int* pages;                        // [n_pages]: pages to give out
  int* copies;                       // [0]: how many; [2 + 2 i]: from, to
};
struct PagedCompactArgs {
  PagedSizes z;
  const int* kv_len; int* table; int* refs;
  int* map; int* used;
  int* err;
  int* copies;                       // as above; [n_pages] pairs
};
struct PagedCopyArgs {               // pages of `copies` in each layer
  char* pool;
  size_t layer_bytes;
  int layers, page_bytes;
  const int* copies;
};

int launch_paged_append(int dtype, int hd, const PagedAppendArgs& a, Stream s);
int launch_paged_attention(int dtype, int hd, const PagedAttnArgs& a, long long tiles, Stream s);  // tiles: of packed rows, at most
int launch_paged_prompt(int hd, const PagedAttnArgs& a, int key_shares, int waves, Stream s);  // bf16
int launch_paged_advance(const PagedAdvanceArgs& a, const PagedCopyArgs& c, Stream s);
int launch_paged_compact(const PagedCompactArgs& a, const PagedCopyArgs& c, Stream s);

}  // namespace ham
