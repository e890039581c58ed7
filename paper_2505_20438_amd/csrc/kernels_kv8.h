// Argument blocks and launchers of the operators on a KV cache in 8 bits (kernels_kv8.hip; host side kv8.cpp).
#pragma once
#include "ham_internal.h"

namespace ham {

constexpr int KV8_BLOCK = 32;        // slots of a block
constexpr float KV8_MAX = 448.0f;    // greatest e4m3 value
constexpr int KV8_MAX_GROUP = 16;    // q-heads of a kv head: the 16 rows of a matrix product
constexpr int KV8_MAX_SPLIT = 64;    // splits of a row's blocks (the combine holds one a lane)

// Regions of a cache buffer of NB blocks per (row, kv head) pair = row * Hk + kv head:
//   codes  [pair][NB][2][32 * hd] bytes: K then V of a block, in the order in which a wave's lanes read them (kv8_k_index,
//          kv8_v_index)
//   scales [pair][NB][2]: K, V
//   bounds [pair][NB][hd / 8][2][8] bytes: least and greatest code of K in each channel over the block's slots
//   open   [pair][2][32][hd], storage type: K and V of the slots past the last full block
struct Kv8Cache {
  uint8_t* codes;
  float* scales;
  uint8_t* bounds;
  void* open;
  int NB;
};

// Byte of (slot s, channel d) within the K codes and the V codes of a block.  A 1 KB piece is what the 64 lanes of a wave
// take with one 16-byte load each.  K: piece (t, d / 64), lane 16 g + r holds slot 8 (r / 4) + 4 t + r % 4, channels 64 i +
// 16 g ..: the scores of K Q^T then lie in the lanes and registers that P V takes its probabilities from.  V: piece d / 32,
// lane 16 g + r holds slots 8 g .. 8 g + 7 of channels 32 p + r and 32 p + 16 + r.
__host__ __device__ __forceinline__ int kv8_k_index(int s, int d, int hd) {
  return ((s / 4 % 2 * (hd / 64) + d / 64) * 64 + d / 16 % 4 * 16 + s / 8 * 4 + s % 4) * 16 + d % 16;
}
__host__ __device__ __forceinline__ int kv8_v_index(int s, int d) {
  return ((d / 32 * 4 + s / 8) * 16 + d % 16) * 16 + d / 16 % 2 * 8 + s % 8;
}

struct Kv8AppendArgs {
  Kv8Cache c;
  int R, T, H, Hk, grp;              // grp = H / Hk
  long long slots;                   // capacity of a row
  const float* qkv; const float* cos; const float* sin;
  const int* start; const int* count;
  void* q;                           // act rows, or null
  int* err;
};
struct Kv8PackArgs {
  Kv8Cache c;
  int R, Hk, S, kv_max;              // S: slots of the source caches
  const void* K; const void* VT;     // storage type, as AttnArgs
  const int* kv_len;
  int* err;
};
struct Kv8SelectArgs {
  Kv8Cache c;
  int R, H, Hk, grp, kv_max, n, first, last;  // grp = H / Hk
  const void* q;                     // act rows
  const int* kv_len; const int* enable;
  int* blocks; int* n_blocks;
  int* err;
  float* scores;                     // [pair][nb_max]
};
struct Kv8AttnArgs {
  Kv8Cache c;
  int R, H, Hk, grp, kv_max, nsplit; // grp = H / Hk
  const void* q; void* out;          // act rows
  const int* kv_len; const int* enable;
  const int* blocks; const int* n_blocks; int max_blocks;  // listed blocks, or null: all
  int* err;
  float* part;                       // records: outputs [pair][nsplit][grp][hd], then (max, sum) [pair][nsplit][grp][2]
};

int launch_kv8_append(int dtype, int hd, const Kv8AppendArgs& a, Stream s);
int launch_kv8_pack(int dtype, int hd, const Kv8PackArgs& a, Stream s);
int launch_kv8_select(int dtype, int hd, const Kv8SelectArgs& a, Stream s);
int launch_kv8_attention(int dtype, int hd, const Kv8AttnArgs& a, Stream s);

}  // namespace ham
