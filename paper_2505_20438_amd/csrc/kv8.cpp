// Host side of the operators on a KV cache in 8 bits (ham_op_kv8_*): argument checks, the cache's regions, launches.
#include "../../include/ham.h"
#include "../../include/ham_ops.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "ham_internal.h"
#include "host_common.h"
#include "kernels_kv8.h"
#include "launch_rules.h"

using namespace ham;

namespace {

const char* check_shape(const ham_kv8_shape* p) {
  if (!p) return "null shape";
  if (p->dtype != HAM_F32 && p->dtype != HAM_BF16) return "dtype must be HAM_F32 or HAM_BF16";
  if (p->rows < 1 || p->rows > 4096) return "rows must be in 1..4096";
  if (p->n_heads < 1 || p->n_kv_heads < 1 || p->n_heads % p->n_kv_heads || p->n_heads / p->n_kv_heads > KV8_MAX_GROUP)
    return "n_heads must be a multiple (<= 16x) of n_kv_heads";
  if (p->n_heads > 1024) return "n_heads must be <= 1024";
  if (p->head_dim != 64 && p->head_dim != 128) return "head_dim must be 64 or 128";
  if (p->slots_cap < KV8_BLOCK || p->slots_cap % KV8_BLOCK || p->slots_cap > (1 << 24))
    return "slots_cap must be a multiple of 32 in 32..2^24";
  return nullptr;
}

struct Regions {
  size_t codes, scales, bounds, open, bytes;
};

Regions regions(const ham_kv8_shape* p) {
  const size_t pairs = (size_t)p->rows * p->n_kv_heads, blocks = pairs * (p->slots_cap / KV8_BLOCK), hd = p->head_dim;
  Regions y;
  size_t o = 0;
  auto take = [&](size_t bytes) { size_t r = o; o += al(bytes); return r; };
  y.codes = take(blocks * 2 * KV8_BLOCK * hd);
  y.scales = take(blocks * 2 * 4);
  y.bounds = take(blocks * 2 * hd);
  y.open = take(pairs * 2 * KV8_BLOCK * hd * (p->dtype == HAM_BF16 ? 2 : 4));
  y.bytes = o;
  return y;
}

Kv8Cache cache_of(const ham_kv8_shape* p, const void* d_cache) {
  const Regions y = regions(p);
  char* base = (char*)const_cast<void*>(d_cache);
  return Kv8Cache{(uint8_t*)(base + y.codes), (float*)(base + y.scales), (uint8_t*)(base + y.bounds), base + y.open,
                  p->slots_cap / KV8_BLOCK};
}

// records of the split launch with the most workgroups (kv8_attn_splits)
size_t attn_record_bytes(const ham_kv8_shape* p) {
  const size_t pairs = (size_t)p->rows * p->n_kv_heads;
  return std::min(std::max<size_t>(KV8_MOST_WGS, 4 * pairs), KV8_MAX_SPLIT * pairs) * (p->n_heads / p->n_kv_heads) * (p->head_dim + 2) * 4;
}

// what every call checks: the shape, the cache buffer, alignment of the 16-byte accesses
int check_call(const ham_kv8_shape* p, const void* d_cache, size_t cache_bytes) {
  if (const char* e = check_shape(p)) return fail(HAM_EINVAL, "%s", e);
  if (!d_cache) return fail(HAM_EINVAL, "null cache");
  if ((uintptr_t)d_cache & 255) return fail(HAM_EINVAL, "the cache must be 256-byte aligned");
  const size_t need = regions(p).bytes;
  if (cache_bytes < need) return fail(HAM_ENOMEM, "the cache needs %zu bytes", need);
  return HAM_OK;
}
bool misaligned(std::initializer_list<const void*> ptrs) {
  for (const void* q : ptrs)
    if ((uintptr_t)q & 15) return true;
  return false;
}

int launched(int rc) {
  if (rc) return fail(HAM_EINVAL, "kv8 shape");
  HIP_TRY(hipGetLastError());
  return HAM_OK;
}

}  // namespace

extern "C" {

size_t ham_op_kv8_cache_bytes(const ham_kv8_shape* p) { return check_shape(p) ? 0 : regions(p).bytes; }

size_t ham_op_kv8_workspace_bytes(const ham_kv8_shape* p) {
  if (check_shape(p)) return 0;
  const size_t pairs = (size_t)p->rows * p->n_kv_heads, blocks = p->slots_cap / KV8_BLOCK;
  return al(std::max(attn_record_bytes(p), pairs * blocks * 4));
}

int ham_op_kv8_info(const ham_kv8_shape* p, size_t* codes, size_t* scales, size_t* bounds, size_t* open) {
  if (const char* e = check_shape(p)) return fail(HAM_EINVAL, "%s", e);
  if (!codes || !scales || !bounds || !open) return fail(HAM_EINVAL, "null output");
  const Regions y = regions(p);
  *codes = y.codes;
  *scales = y.scales;
  *bounds = y.bounds;
  *open = y.open;
  return HAM_OK;
}

int ham_op_kv8_append(const ham_kv8_shape* p, int32_t n_tokens, const float* d_qkv, const float* d_cos, const float* d_sin,
                      const int32_t* d_start, const int32_t* d_count, void* d_cache, size_t cache_bytes, void* d_q,
                      int32_t* d_err, void* hip_stream) {
  if (int rc = check_call(p, d_cache, cache_bytes)) return rc;
  if (n_tokens < 1 || n_tokens > (1 << 24)) return fail(HAM_EINVAL, "n_tokens must be in 1..2^24");
  if (!d_qkv || !d_cos || !d_sin || !d_start || !d_count || !d_err) return fail(HAM_EINVAL, "null pointer");
  if (misaligned({d_qkv, d_cos, d_sin, d_q})) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  if (((long long)p->rows * ((n_tokens + 31) / 32) + 8) * p->n_kv_heads * 4 * p->head_dim > UINT32_MAX)
    return fail(HAM_EINVAL, "rows * n_tokens * n_kv_heads * head_dim too large for one call");
  Kv8AppendArgs a{};
  a.c = cache_of(p, d_cache);
  a.R = p->rows; a.T = n_tokens; a.H = p->n_heads; a.Hk = p->n_kv_heads; a.grp = p->n_heads / p->n_kv_heads; a.slots = p->slots_cap;
  a.qkv = d_qkv; a.cos = d_cos; a.sin = d_sin; a.start = d_start; a.count = d_count; a.q = d_q; a.err = d_err;
  return launched(launch_kv8_append(p->dtype, p->head_dim, a, (hipStream_t)hip_stream));
}

int ham_op_kv8_pack(const ham_kv8_shape* p, const void* d_k, const void* d_vt, int32_t src_slots, const int32_t* d_kv_len,
                    int32_t kv_max, void* d_cache, size_t cache_bytes, int32_t* d_err, void* hip_stream) {
  if (int rc = check_call(p, d_cache, cache_bytes)) return rc;
  if (src_slots < KV8_BLOCK || src_slots % KV8_BLOCK) return fail(HAM_EINVAL, "src_slots must be a multiple of 32");
  if (kv_max < 0 || kv_max > p->slots_cap || kv_max > src_slots) return fail(HAM_EINVAL, "kv_max out of range");
  if (!d_k || !d_vt || !d_kv_len || !d_err) return fail(HAM_EINVAL, "null pointer");
  if (misaligned({d_k, d_vt})) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  Kv8PackArgs a{};
  a.c = cache_of(p, d_cache);
  a.R = p->rows; a.Hk = p->n_kv_heads; a.S = src_slots; a.kv_max = kv_max;
  a.K = d_k; a.VT = d_vt; a.kv_len = d_kv_len; a.err = d_err;
  return launched(launch_kv8_pack(p->dtype, p->head_dim, a, (hipStream_t)hip_stream));
}

int ham_op_kv8_select(const ham_kv8_shape* p, const void* d_q, const void* d_cache, size_t cache_bytes,
                      const int32_t* d_kv_len, const int32_t* d_enable, int32_t kv_max, int32_t n_blocks,
                      int32_t keep_first, int32_t keep_last, int32_t* d_blocks, int32_t* d_n_blocks, int32_t* d_err,
                      void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_call(p, d_cache, cache_bytes)) return rc;
  if (kv_max < 0 || kv_max > p->slots_cap) return fail(HAM_EINVAL, "kv_max out of range");
  if (n_blocks < 1 || n_blocks > p->slots_cap / KV8_BLOCK) return fail(HAM_EINVAL, "n_blocks must be in 1..slots_cap/32");
  if (keep_first < 0 || keep_last < 0 || (long long)keep_first + keep_last > n_blocks)
    return fail(HAM_EINVAL, "keep_first and keep_last must not be negative, nor more than n_blocks together");
  if (!d_q || !d_kv_len || !d_enable || !d_blocks || !d_n_blocks || !d_err || !d_workspace)
    return fail(HAM_EINVAL, "null pointer");
  if (misaligned({d_q, d_workspace})) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  const size_t need = ham_op_kv8_workspace_bytes(p);
  if (workspace_bytes < need) return fail(HAM_ENOMEM, "the workspace needs %zu bytes", need);
  Kv8SelectArgs a{};
  a.c = cache_of(p, d_cache);
  a.R = p->rows; a.H = p->n_heads; a.Hk = p->n_kv_heads; a.grp = p->n_heads / p->n_kv_heads; a.kv_max = kv_max; a.n = n_blocks; a.first = keep_first;
  a.last = keep_last; a.q = d_q; a.kv_len = d_kv_len; a.enable = d_enable; a.blocks = d_blocks; a.n_blocks = d_n_blocks;
  a.err = d_err; a.scores = (float*)d_workspace;
  return launched(launch_kv8_select(p->dtype, p->head_dim, a, (hipStream_t)hip_stream));
}

int ham_op_kv8_attention(const ham_kv8_shape* p, const void* d_q, const void* d_cache, size_t cache_bytes,
                         const int32_t* d_kv_len, const int32_t* d_enable, int32_t kv_max, const int32_t* d_blocks,
                         const int32_t* d_n_blocks, int32_t max_blocks, void* d_out, int32_t* d_err, void* d_workspace,
                         size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_call(p, d_cache, cache_bytes)) return rc;
  if (kv_max < 0 || kv_max > p->slots_cap) return fail(HAM_EINVAL, "kv_max out of range");
  if (!d_q || !d_kv_len || !d_enable || !d_out || !d_err || !d_workspace) return fail(HAM_EINVAL, "null pointer");
  if ((d_blocks == nullptr) != (d_n_blocks == nullptr)) return fail(HAM_EINVAL, "d_blocks and d_n_blocks go together");
  if (d_blocks && (max_blocks < 1 || max_blocks > p->slots_cap / KV8_BLOCK))
    return fail(HAM_EINVAL, "max_blocks must be in 1..slots_cap/32");
  if (misaligned({d_q, d_out, d_workspace})) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  const size_t need = ham_op_kv8_workspace_bytes(p);
  if (workspace_bytes < need) return fail(HAM_ENOMEM, "the workspace needs %zu bytes", need);
  Kv8AttnArgs a{};
  a.c = cache_of(p, d_cache);
  a.R = p->rows; a.H = p->n_heads; a.Hk = p->n_kv_heads; a.grp = p->n_heads / p->n_kv_heads; a.kv_max = kv_max;
  a.q = d_q; a.out = d_out; a.kv_len = d_kv_len; a.enable = d_enable;
  a.blocks = d_blocks; a.n_blocks = d_n_blocks; a.max_blocks = d_blocks ? max_blocks : 0; a.err = d_err;
  a.part = (float*)d_workspace;
  const int blocks = d_blocks ? std::min(max_blocks, kv_max / KV8_BLOCK) : kv_max / KV8_BLOCK;
  a.nsplit = kv8_attn_splits(p->rows, p->n_kv_heads, p->head_dim, blocks);
  return launched(launch_kv8_attention(p->dtype, p->head_dim, a, (hipStream_t)hip_stream));
}

}  // extern "C"
