/*
 * libham single-operator entry points, on caller-provided buffers.
 *
 * The first ones run one kernel of the decode loop, for parity tests and
 * diagnostics: a test can check one step at shapes where running the whole model
 * through a CPU reference is too slow (e.g. attention over a 32K-slot cache):
 *  - ham_op_attention_step runs the fused decode-attention step that every
 *    base layer of ham_macro_step launches, with the same split choice for the
 *    same batch and slot bound;
 *  - ham_op_decode_attention runs the attention over an already filled cache
 *    that a prompt batch's last base layer and the micro decoder's first step
 *    use (a different kernel).
 * The ham_op_kv8_* operators are for a decode loop of the caller's own: they keep
 * a KV cache in 8 bits, which ham_prefill and ham_macro_step neither write nor
 * read (ham_op_kv8_pack takes what a prefill left).
 * Same conventions as include/ham.h: C functions, HAM_OK or a negative
 * HAM_E* code, ham_last_error() for the message, "d_" = device pointers, work
 * enqueued on `hip_stream` and valid after it is synchronised.
 *
 * Activation layout ("act rows") of width W: fp32 models store fp32 [W] per row;
 * bf16 models store each value v as the bf16 pair hi = bf16(v), lo = bf16(v - hi)
 * in two planes per row, [hi 0..W) [lo 0..W) (4 bytes per value either way).
 */
#ifndef HAM_OPS_H
#define HAM_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Workspace bytes that ham_op_decode_attention needs for `rows` query rows. */
size_t ham_op_attention_workspace_bytes(int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);

/* GQA decode attention of one query row per sequence over that sequence's
 * cache (the base-layer attention of a macro-step over the smashed KV cache,
 * Sec. 3.1): out[r, h] = softmax_j(q[r, h] . K[r, h/(H/Hkv), j] / sqrt(hd)) V[...]
 * over slots j < kv_len[r]; rows with enable[r] == 0 (or kv_len 0) get zeros.
 *  dtype        HAM_F32 or HAM_BF16 (cache element type)
 *  d_q          act rows [rows][n_heads*head_dim], RoPE already applied
 *  d_k          [rows][n_kv_heads][slots_cap][head_dim]   (slot-major)
 *  d_vt         [rows][n_kv_heads][slots_cap/32][head_dim][32]   (V in 32-slot
 *               tiles, d-major inside a tile: element (d, slot) at
 *               ((slot/32)*head_dim + d)*32 + slot%32 of its (row, kv head))
 *  d_kv_len     int32 [rows], each <= slots_cap; d_enable int32 [rows]
 *  kv_max       host upper bound of kv_len (with rows, n_kv_heads, head_dim and
 *               dtype it chooses the slot split; rows may be of any lengths)
 *  d_out        act rows [rows][n_heads*head_dim]
 * head_dim 64 or 128, n_heads/n_kv_heads in 1..4, slots_cap a multiple of 64.
 * HAM_EINVAL on a bad shape, HAM_ENOMEM if the workspace is too small. */
int ham_op_decode_attention(int32_t dtype, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                            int32_t slots_cap, const void* d_q, const void* d_k, const void* d_vt,
                            const int32_t* d_kv_len, const int32_t* d_enable, int32_t kv_max, void* d_out,
                            void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* The fused decode-attention step of one base layer of a macro-step (Sec. 3.1:
 * the fused group's single new KV entry is appended, then attention runs over
 * the smashed cache), for one row per sequence:
 *   q = RoPE(q part of qkv[r]), k = RoPE(k part), v = v part, rotate-half RoPE
 *   with the row's factors (pair (i, i + hd/2) rotated by cos[r][i], sin[r][i]);
 *   k and v are rounded to the cache type and written at slot new_slot[r];
 *   out[r, h] = sum_j softmax_j(q_h . K[r, h/(H/Hkv), j] / sqrt(hd)) V[..., j]
 *   over slots j < kv_len[r] (the new slot included; its score uses the
 *   rounded k).
 *  d_qkv        fp32 [rows][(n_heads + 2*n_kv_heads)*head_dim]: all q heads,
 *               then the k heads, then the v heads (before RoPE)
 *  d_cos, d_sin fp32 [rows][head_dim/2]
 *  d_k, d_vt    caches laid out as for ham_op_decode_attention; slot new_slot[r]
 *               is written, slots below it are read
 *  d_kv_len     int32 [rows]: slots after the append; d_new_slot int32 [rows]
 *               must equal kv_len - 1 and be <= kv_cap, else the row writes
 *               nothing, gets zeros and d_err[r] is OR-ed with 8
 *  d_enable     int32 [rows]: 0 = the row writes nothing and gets zeros
 *  kv_cap       host bound on new_slot for every row, < slots_cap; it and `rows`
 *               choose the slot split exactly as a macro-step over `rows`
 *               sequences does (ham_op_attention_step_splits tells how many)
 *  d_err        int32 [rows], in/out (bits are only set)
 *  d_out        act rows [rows][n_heads*head_dim]
 *  d_workspace  at least ham_op_attention_workspace_bytes(rows, ...) bytes
 * rows in 1..64, head_dim 64 or 128, n_heads/n_kv_heads in 1..4, slots_cap a
 * multiple of 64.  HAM_EINVAL on a bad shape or null pointer, HAM_ENOMEM if
 * the workspace is too small. */
int ham_op_attention_step(int32_t dtype, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                          int32_t slots_cap, const float* d_qkv, const float* d_cos, const float* d_sin, void* d_k,
                          void* d_vt, const int32_t* d_kv_len, const int32_t* d_new_slot, const int32_t* d_enable,
                          int32_t kv_cap, int32_t* d_err, void* d_out, void* d_workspace, size_t workspace_bytes,
                          void* hip_stream);

/* ham_op_attention_step without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc): the split records live in a library-owned device
 * array of ham_op_attention_step_noalloc_max_bytes() bytes (4 MiB), one per
 * GPU, kept until the process ends.  The call allocates nothing (no hipMalloc,
 * hipFree or allocating library routine); on its first use on a device it
 * looks up that device's copy of the array (the current device).  Arguments,
 * results and errors as for ham_op_attention_step, plus HAM_ENOMEM when the
 * launch's split records (rows * n_kv_heads * splits * (n_heads/n_kv_heads) *
 * (head_dim + 2) * 4 bytes, none when unsplit) exceed the array.  Every split
 * writes its whole record before the merge reads it, so nothing needs
 * clearing between calls; calls that overlap on one GPU (other streams or
 * host threads) share the array and race. */
int ham_op_attention_step_noalloc(int32_t dtype, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                  int32_t slots_cap, const float* d_qkv, const float* d_cos, const float* d_sin,
                                  void* d_k, void* d_vt, const int32_t* d_kv_len, const int32_t* d_new_slot,
                                  const int32_t* d_enable, int32_t kv_cap, int32_t* d_err, void* d_out,
                                  void* hip_stream);
size_t ham_op_attention_step_noalloc_max_bytes(void);

/* Slot splits (workgroups per row and kv head) that ham_op_attention_step and
 * a macro-step over `rows` sequences use for this slot bound; 0 if invalid. */
int ham_op_attention_step_splits(int32_t dtype, int32_t rows, int32_t n_kv_heads, int32_t head_dim, int32_t kv_cap);

/* ---------------------------------------------------------------- KV cache in 8 bits
 * One layer's K and V of `rows` sequences in e4m3 codes with a scale for each
 * block of 32 slots and kv head (half the bytes of a bf16 cache), its writers
 * and the attention of one query row per sequence over it, over every block or
 * over the blocks that ham_op_kv8_select chooses.
 *
 * A closed block (32 slots of a kv head) holds K and V apart as
 *   a = max |x| over its 32 x head_dim values, each first rounded to the storage
 *   type; scale = a / 448; code = e4m3(x * (1 / scale)), nearest even, at most 448;
 *   a value stands for code * scale.
 * All codes are 0 where the scale is below the least normal fp32 value.  A block
 * with an infinity or NaN has scale NaN: every row that reads it becomes NaN.
 * The slots past the last full block (kv_len % 32) are in the open block, in the
 * storage type.  A block is coded once, when its 32nd slot arrives, so the cache
 * is the same, bit for bit, whether its slots came one by one or together.  A
 * row may be shortened by slots of its open block, or to a multiple of 32; at any
 * other lower kv_len the open block holds other slots than those past the last
 * full block, and what is read of it is wrong.  So each query row attends over the
 * slots its cache holds at the time: there is no causal attention of a prompt's
 * rows over this cache.  The caller attends over such a prompt by other means
 * (ham_op_kv8_append gives its rotated q), or appends it token by token.
 *
 * The cache is one caller-owned buffer of ham_op_kv8_cache_bytes bytes, 256-byte
 * aligned; it needs no clearing.  Regions (ham_op_kv8_info), pair = row *
 * n_kv_heads + kv head, NB = slots_cap / 32 blocks each:
 *   codes  [pair][NB][2][32*head_dim]: K, then V; (slot s, channel d) at
 *     K ((s/4%2*(head_dim/64) + d/64)*64 + d/16%4*16 + s/8*4 + s%4)*16 + d%16
 *     V ((d/32*4 + s/8)*16 + d%16)*16 + d/16%2*8 + s%8
 *   scales fp32 [pair][NB][2]: K, V
 *   bounds [pair][NB][head_dim/8][2][8]: least and greatest K code of each
 *     channel (for 8 channels: 8 least, then 8 greatest)
 *   open   [pair][2][32][head_dim], storage type: K, V
 *
 * Rows and lengths: a length outside 0..kv_max (append: start and count that do
 * not fit n_tokens or slots_cap) makes the row one without slots and ORs 8 into
 * d_err[r] (int32 [rows], in/out, bits are only set).  d_enable[r] = 0: the row
 * is one without slots.  Other streams or host threads may read one cache at
 * the same time, with workspaces and outputs of their own; a call that writes
 * it is ordered against them by the caller.  Nothing is allocated and no call
 * waits for the GPU: all of them can be captured into a graph.  A workspace needs
 * no clearing and keeps nothing between calls.  kv_max is a bound that a captured
 * graph keeps: ham_op_kv8_select scores blocks up to it whatever the lengths, and
 * ham_op_kv8_attention splits its work, and so orders its sums, by it. */
#define HAM_KV8_BLOCK 32

typedef struct ham_kv8_shape {
  int32_t dtype;      /* storage type of the open block and of activations: HAM_F32 or HAM_BF16 */
  int32_t rows;       /* sequences, 1..4096 */
  int32_t n_heads, n_kv_heads;  /* n_heads <= 1024, a multiple (1..16) of n_kv_heads */
  int32_t head_dim;   /* 64 or 128 */
  int32_t slots_cap;  /* slots of a row, a multiple of 32, at most 2^24 */
} ham_kv8_shape;

/* Bytes of the cache, and of the workspace that any ham_op_kv8_select or
 * ham_op_kv8_attention of this shape needs; 0 for an invalid shape. */
size_t ham_op_kv8_cache_bytes(const ham_kv8_shape* shape);
size_t ham_op_kv8_workspace_bytes(const ham_kv8_shape* shape);
/* Byte offsets of the regions in the cache buffer. */
int ham_op_kv8_info(const ham_kv8_shape* shape, size_t* codes, size_t* scales, size_t* bounds, size_t* open);

/* RoPE and append: count[r] new slots of row r after the start[r] it holds.
 *  d_qkv         fp32 [rows][n_tokens][(n_heads + 2*n_kv_heads)*head_dim]: all q
 *                heads, then k, then v, before RoPE (as ham_op_attention_step)
 *  d_cos, d_sin  fp32 [rows][n_tokens][head_dim/2]; rotate-half RoPE, each
 *                product and each sum rounded to fp32
 *  d_start, d_count  int32 [rows]; 0 <= count <= n_tokens, start + count <= slots_cap
 *  d_q           act rows [rows][n_tokens][n_heads*head_dim]: the rotated q of
 *                the new slots (the rest is left as it is), or NULL
 * Codes, scales and bounds of the blocks that fill up, and the open block's new
 * slots, are written, nothing else.  HAM_EINVAL on a bad shape, null or
 * misaligned (16 bytes) pointer, n_tokens outside 1..2^24, or rows * n_tokens
 * past one launch (rows * (n_tokens + 31) / 32 * n_kv_heads * head_dim about
 * 2^30); HAM_ENOMEM if the cache buffer is too small. */
int ham_op_kv8_append(const ham_kv8_shape* shape, int32_t n_tokens, const float* d_qkv, const float* d_cos,
                      const float* d_sin, const int32_t* d_start, const int32_t* d_count, void* d_cache,
                      size_t cache_bytes, void* d_q, int32_t* d_err, void* hip_stream);

/* A filled cache of the storage type (as a prefill leaves a layer's in the state
 * buffer, ham_state_info) into the 8-bit cache: slots [0, kv_len[r]) of each row.
 *  d_k, d_vt  as for ham_op_decode_attention, of src_slots slots a row
 *  kv_max     host upper bound of kv_len, at most slots_cap and src_slots */
int ham_op_kv8_pack(const ham_kv8_shape* shape, const void* d_k, const void* d_vt, int32_t src_slots,
                    const int32_t* d_kv_len, int32_t kv_max, void* d_cache, size_t cache_bytes, int32_t* d_err,
                    void* hip_stream);

/* For one query row per sequence: the n_blocks closed blocks of each kv head
 * whose keys may score highest (all of them where a row has no more).  A block's
 * score is the greatest over the kv head's q-heads of
 *   scale_K * sum_d max(q_d least_d, q_d greatest_d),
 * an upper bound of q . k over its keys, summed in fp64 and rounded to fp32:
 * no key of a block that is left out scores above the least score chosen.
 * Equal scores: the lower block first.  A block whose K or V holds an infinity
 * or NaN scores NaN, which counts as greatest.  The first keep_first and the last
 * keep_last closed blocks are always chosen.
 *  d_q         act rows [rows][n_heads*head_dim], RoPE applied
 *  kv_max      host upper bound of kv_len
 *  d_blocks    int32 [rows][n_kv_heads][n_blocks], ascending, then -1
 *  d_n_blocks  int32 [rows][n_kv_heads]
 * n_blocks in 1..slots_cap/32, keep_first + keep_last <= n_blocks. */
int ham_op_kv8_select(const ham_kv8_shape* shape, const void* d_q, const void* d_cache, size_t cache_bytes,
                      const int32_t* d_kv_len, const int32_t* d_enable, int32_t kv_max, int32_t n_blocks,
                      int32_t keep_first, int32_t keep_last, int32_t* d_blocks, int32_t* d_n_blocks, int32_t* d_err,
                      void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* GQA attention of one query row per sequence:
 *   out[r, h] = softmax_j(q[r, h] . K[r, h/(H/Hkv), j] / sqrt(hd)) V[...]
 * over the slots j < kv_len[r] of every closed block, or with d_blocks of the
 * listed ones, and of the open block.  A row without slots, or whose scores are all
 * -infinity, gets zeros.  Weights times V's scale are sums of three bf16 values, 24
 * bits while V's magnitudes are above 1e-31 and fewer below.
 *  d_blocks, d_n_blocks  lists as ham_op_kv8_select writes them, max_blocks
 *              entries apart, or both NULL: an entry that is not above the one
 *              before it or not a closed block of the row is left out, a count
 *              outside 0..max_blocks counts as 0; both OR 16 into d_err[r]
 *  kv_max      host upper bound of kv_len (with rows, n_kv_heads and max_blocks
 *              it chooses the split of the blocks over workgroups)
 *  d_q, d_out  act rows [rows][n_heads*head_dim] */
int ham_op_kv8_attention(const ham_kv8_shape* shape, const void* d_q, const void* d_cache, size_t cache_bytes,
                         const int32_t* d_kv_len, const int32_t* d_enable, int32_t kv_max, const int32_t* d_blocks,
                         const int32_t* d_n_blocks, int32_t max_blocks, void* d_out, int32_t* d_err,
                         void* d_workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* HAM_OPS_H */
