// Host side of the operators on a paged KV cache (ham_op_paged_*): argument checks, workspace, launches.
#include "../../include/ham.h"
#include "../../include/ham_ops.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "ham_internal.h"
#include "host_common.h"
#include "kernels_paged.h"
#include "launch_rules.h"

using namespace ham;

namespace {

const char* check_shape(const ham_paged_shape* p) {
  if (!p) return "null shape";
  if (p->dtype != HAM_F32 && p->dtype != HAM_BF16) return "dtype must be HAM_F32 or HAM_BF16";
  if (p->rows < 1 || p->rows > 4096) return "rows must be in 1..4096";
  if (p->n_heads < 1 || p->n_kv_heads < 1 || p->n_heads % p->n_kv_heads || p->n_heads / p->n_kv_heads > PAGED_MAX_GROUP)
    return "n_heads must be a multiple (<= 16x) of n_kv_heads";
  if (p->n_heads > 1024) return "n_heads must be <= 1024";
  if (p->head_dim != 64 && p->head_dim != 128) return "head_dim must be 64 or 128";
  if (p->page_slots < 16 || p->page_slots > 256 || (p->page_slots & (p->page_slots - 1)))
    return "page_slots must be 16, 32, 64, 128 or 256";
  if (p->n_pages < 1 || p->n_pages > (1 << 22)) return "n_pages must be in 1..2^22";
  if (p->row_pages < 1 || (long long)p->row_pages * p->page_slots > (1 << 24)) return "row_pages * page_slots must be in 16..2^24";
  if ((long long)p->rows * p->row_pages > (1 << 28)) return "rows * row_pages must be at most 2^28";
  return nullptr;
}

size_t page_bytes(const ham_paged_shape* p) {
  return (size_t)p->n_kv_heads * 2 * p->page_slots * p->head_dim * (p->dtype == HAM_BF16 ? 2 : 4);
}
size_t pool_bytes(const ham_paged_shape* p) { return al(page_bytes(p) * p->n_pages); }
long long capacity(const ham_paged_shape* p) { return (long long)p->row_pages * p->page_slots; }

PagedSizes sizes_of(const ham_paged_shape* p) {
  return PagedSizes{p->rows, p->n_heads, p->n_kv_heads, p->n_heads / p->n_kv_heads, __builtin_ctz(p->page_slots), p->n_pages, p->row_pages};
}

// int32 of the workspace that the calls on tables need
size_t table_ints(const ham_paged_shape* p) {
  return (size_t)p->rows * p->row_pages + 4 * (size_t)p->rows + 3 * (size_t)p->n_pages + 64;
}

int check_pool(const ham_paged_shape* p, const void* d_pool, size_t bytes, int layers) {
  if (const char* e = check_shape(p)) return fail(HAM_EINVAL, "%s", e);
  if (layers < 1 || layers > 1024) return fail(HAM_EINVAL, "n_layers must be in 1..1024");
  if (!d_pool) return fail(HAM_EINVAL, "null pool");
  if ((uintptr_t)d_pool & 255) return fail(HAM_EINVAL, "the pool must be 256-byte aligned");
  const size_t need = pool_bytes(p) * layers;
  if (bytes < need) return fail(HAM_ENOMEM, "the pool needs %zu bytes", need);
  return HAM_OK;
}
int check_workspace(const ham_paged_shape* p, const void* d_workspace, size_t bytes) {
  if (!d_workspace) return fail(HAM_EINVAL, "null pointer");
  if ((uintptr_t)d_workspace & 15) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  const size_t need = ham_op_paged_workspace_bytes(p);
  if (bytes < need) return fail(HAM_ENOMEM, "the workspace needs %zu bytes", need);
  return HAM_OK;
}
bool misaligned(std::initializer_list<const void*> ptrs) {
  for (const void* q : ptrs)
    if ((uintptr_t)q & 15) return true;
  return false;
}
int launched(int rc) {
  if (rc) return fail(HAM_EINVAL, "paged shape");
  HIP_TRY(hipGetLastError());
  return HAM_OK;
}

}  // namespace

extern "C" {

size_t ham_op_paged_pool_bytes(const ham_paged_shape* p) { return check_shape(p) ? 0 : pool_bytes(p); }

size_t ham_op_paged_workspace_bytes(const ham_paged_shape* p) {
  if (check_shape(p)) return 0;
  return al(std::max((size_t)PAGED_MAX_RECORDS * (p->head_dim + 2) * 4, table_ints(p) * 4));
}

int ham_op_paged_append(const ham_paged_shape* p, int32_t n_tokens, const float* d_qkv, const float* d_cos, const float* d_sin,
                        const int32_t* d_offsets, const int32_t* d_start, const int32_t* d_table, void* d_pool, size_t pool_bytes_,
                        void* d_q, int32_t* d_err, void* hip_stream) {
  if (int rc = check_pool(p, d_pool, pool_bytes_, 1)) return rc;
  if (n_tokens < 1 || n_tokens > (1 << 24)) return fail(HAM_EINVAL, "n_tokens must be in 1..2^24");
  if (!d_qkv || !d_cos || !d_sin || !d_offsets || !d_start || !d_table || !d_err) return fail(HAM_EINVAL, "null pointer");
  if (misaligned({d_qkv, d_cos, d_sin, d_q})) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  if (!paged_append_fits(n_tokens, p->n_kv_heads))
    return fail(HAM_EINVAL, "n_tokens * n_kv_heads too large for one call");
  PagedAppendArgs a{};
  a.z = sizes_of(p);
  a.N = n_tokens; a.qkv = d_qkv; a.cos = d_cos; a.sin = d_sin; a.offsets = d_offsets; a.start = d_start; a.table = d_table;
  a.pool = d_pool; a.q = d_q; a.err = d_err;
  a.per_step = paged_append_groups(n_tokens, p->rows, p->n_kv_heads * (d_q ? 2 : 1));
  return launched(launch_paged_append(p->dtype, p->head_dim, a, (hipStream_t)hip_stream));
}

int ham_op_paged_attention(const ham_paged_shape* p, const void* d_q, const void* d_pool, size_t pool_bytes_, const int32_t* d_table,
                           const int32_t* d_kv_len, const int32_t* d_enable, int32_t kv_max, void* d_out, int32_t* d_err,
                           void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_pool(p, d_pool, pool_bytes_, 1)) return rc;
  if (kv_max < 0 || kv_max > capacity(p)) return fail(HAM_EINVAL, "kv_max out of range");
  if (!d_q || !d_table || !d_kv_len || !d_enable || !d_out || !d_err) return fail(HAM_EINVAL, "null pointer");
  if (misaligned({d_q, d_out})) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  if (int rc = check_workspace(p, d_workspace, workspace_bytes)) return rc;
  PagedAttnArgs a{};
  a.z = sizes_of(p);
  a.kv_max = kv_max; a.q = d_q; a.out = d_out; a.pool = d_pool; a.table = d_table; a.kv_len = d_kv_len; a.enable = d_enable;
  a.err = d_err; a.part = (float*)d_workspace;
  a.nsplit = paged_attn_split(p->rows, p->n_heads, p->n_kv_heads, p->head_dim, kv_max, p->dtype == HAM_BF16 ? 32 : 16)
                 ? paged_attn_shares(p->rows, p->n_kv_heads) : 0;
  return launched(launch_paged_attention(p->dtype, p->head_dim, a, 0, (hipStream_t)hip_stream));
}

int ham_op_paged_prompt(const ham_paged_shape* p, int32_t n_tokens, const void* d_q, const int32_t* d_offsets, const void* d_pool,
                        size_t pool_bytes_, const int32_t* d_table, const int32_t* d_kv_len, int32_t kv_max, void* d_out,
                        int32_t* d_err, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_pool(p, d_pool, pool_bytes_, 1)) return rc;
  if (n_tokens < 1 || n_tokens > (1 << 24)) return fail(HAM_EINVAL, "n_tokens must be in 1..2^24");
  if (kv_max < 0 || kv_max > capacity(p)) return fail(HAM_EINVAL, "kv_max out of range");
  if (!d_q || !d_offsets || !d_table || !d_kv_len || !d_out || !d_err) return fail(HAM_EINVAL, "null pointer");
  if (misaligned({d_q, d_out})) return fail(HAM_EINVAL, "buffers must be 16-byte aligned");
  if (int rc = check_workspace(p, d_workspace, workspace_bytes)) return rc;
  const int grp = p->n_heads / p->n_kv_heads;
  if (paged_tiles(n_tokens, p->rows, grp, 16) * p->n_kv_heads > (1 << 22))
    return fail(HAM_EINVAL, "n_tokens * n_heads too large for one call");
  PagedAttnArgs a{};
  a.z = sizes_of(p);
  a.N = n_tokens; a.kv_max = kv_max; a.q = d_q; a.out = d_out; a.pool = d_pool; a.offsets = d_offsets; a.table = d_table;
  a.kv_len = d_kv_len; a.err = d_err; a.part = (float*)d_workspace;
  const bool all = p->dtype == HAM_F32 || paged_prompt_tiles(n_tokens, p->rows, p->n_kv_heads, grp, kv_max);
  a.few = all ? INT32_MAX : p->rows > 1 ? PAGED_FEW : 0;
  if (a.few > 0) {
    const long long most = paged_tiles(n_tokens, p->rows, grp, 16), tiles = all ? most : std::min(most, PAGED_FEW / 16 * (long long)p->rows);
    a.nsplit = paged_tile_splits(tiles, p->n_kv_heads, kv_max, p->dtype == HAM_F32 ? 16 : 32);
    if (int rc = launched(launch_paged_attention(p->dtype, p->head_dim, a, tiles, (hipStream_t)hip_stream))) return rc;
    if (all) return HAM_OK;
  }
  const PagedPromptGrid g = paged_prompt_grid(n_tokens, p->rows, p->n_kv_heads, grp, kv_max);
  a.nsplit = g.splits;
  return launched(launch_paged_prompt(p->head_dim, a, g.shares, paged_prompt_waves(n_tokens, p->n_kv_heads, grp, p->head_dim, kv_max),
                                      (hipStream_t)hip_stream));
}

int ham_op_paged_advance(const ham_paged_shape* p, int32_t n_layers, const int32_t* d_parent, const int32_t* d_count,
                         int32_t* d_kv_len, int32_t* d_start, int32_t* d_table, int32_t* d_refs, void* d_pool, size_t pool_bytes_,
                         int32_t* d_err, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_pool(p, d_pool, pool_bytes_, n_layers)) return rc;
  if (!d_count || !d_kv_len || !d_start || !d_table || !d_refs || !d_err) return fail(HAM_EINVAL, "null pointer");
  if (d_start == d_kv_len) return fail(HAM_EINVAL, "d_start must be another buffer than d_kv_len");
  if ((long long)p->rows * n_layers * ((page_bytes(p) + 16383) / 16384) > INT32_MAX)
    return fail(HAM_EINVAL, "rows * n_layers * page bytes too large for one call");
  if (int rc = check_workspace(p, d_workspace, workspace_bytes)) return rc;
  PagedAdvanceArgs a{};
  a.z = sizes_of(p);
  a.parent = d_parent; a.count = d_count; a.kv_len = d_kv_len; a.start = d_start; a.table = d_table; a.refs = d_refs; a.err = d_err;
  int* ws = (int*)d_workspace;
  a.copies = ws; ws += 2 + 2 * p->rows;
  a.taken_len = ws; ws += p->rows;
  a.span = ws; ws += p->rows;
  a.owner = ws; ws += 2 * (size_t)p->n_pages;
  a.pages = ws; ws += p->n_pages;
  a.taken = ws;
  const PagedCopyArgs c{(char*)d_pool, pool_bytes(p), n_layers, (int)page_bytes(p), a.copies};
  return launched(launch_paged_advance(a, c, (hipStream_t)hip_stream));
}

int ham_op_paged_compact(const ham_paged_shape* p, int32_t n_layers, const int32_t* d_kv_len, int32_t* d_table, int32_t* d_refs,
                         void* d_pool, size_t pool_bytes_, int32_t* d_map, int32_t* d_n_used, int32_t* d_err, void* d_workspace,
                         size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_pool(p, d_pool, pool_bytes_, n_layers)) return rc;
  if (!d_kv_len || !d_table || !d_refs || !d_map || !d_n_used || !d_err) return fail(HAM_EINVAL, "null pointer");
  if ((long long)p->n_pages * n_layers * ((page_bytes(p) + 16383) / 16384) > INT32_MAX)
    return fail(HAM_EINVAL, "n_pages * n_layers * page bytes too large for one call");
  if (int rc = check_workspace(p, d_workspace, workspace_bytes)) return rc;
  PagedCompactArgs a{};
  a.z = sizes_of(p);
  a.kv_len = d_kv_len; a.table = d_table; a.refs = d_refs; a.map = d_map; a.used = d_n_used; a.err = d_err;
  a.copies = (int*)d_workspace;
  const PagedCopyArgs c{(char*)d_pool, pool_bytes(p), n_layers, (int)page_bytes(p), a.copies};
  return launched(launch_paged_compact(a, c, (hipStream_t)hip_stream));
}

}  // extern "C"
