// C-ABI entry points: argument validation, error reporting, dispatch to the kernel launchers.
// The operation and its conventions are documented in include/shiftattn.h.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <exception>
#include <vector>

#include "sp_common.h"
#include "fresh_plan.h"

namespace sp {

static thread_local char g_err[512] = "";

int fail(int status, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return status;
}

static int check_cache(const sp_cache_desc *c) {
  if (!c) return fail(SP_ERR_NULL, "cache descriptor is NULL");
  if (!c->k_pages || !c->v_pages) return fail(SP_ERR_NULL, "cache pools are NULL");
  if (c->num_pages <= 0 || c->num_kv_heads <= 0)
    return fail(SP_ERR_BAD_SHAPE, "num_pages=%d num_kv_heads=%d must be positive", c->num_pages,
                c->num_kv_heads);
  if (c->page_size != kPage) return fail(SP_ERR_UNSUPPORTED, "page_size=%d (only 16)", c->page_size);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(SP_ERR_UNSUPPORTED, "head_dim=%d (only 64 or 128)", c->head_dim);
  return SP_OK;
}

static int check_heads(const sp_cache_desc *c, int num_q_heads) {
  if (num_q_heads <= 0 || num_q_heads % c->num_kv_heads != 0)
    return fail(SP_ERR_BAD_SHAPE, "num_q_heads=%d is not a positive multiple of num_kv_heads=%d",
                num_q_heads, c->num_kv_heads);
  return SP_OK;
}

static int check_scale(float scale) {
  if (!(scale > 0.0f) || !std::isfinite(scale))
    return fail(SP_ERR_UNSUPPORTED, "scale=%g must be positive and finite", (double)scale);
  return SP_OK;
}

// What the checks of device arrays do on the host.  No exception crosses the ABI: host memory may not hold arrays of the sizes asked for.
template <typename Check>
static int checked(const char *name, Check check) {
  try {
    return check();
  } catch (const std::exception &) {
    return fail(SP_ERR_UNSUPPORTED, "%s: no host memory for arrays of these sizes", name);
  }
}

}  // namespace sp

using namespace sp;

extern "C" {

int sp_kv_append(const sp_cache_desc *cache, const void *k_new, const void *v_new,
                 const int32_t *cu_seqlens_new, const int32_t *ctx_lens,
                 const int32_t *block_table, int32_t batch, int32_t max_pages_per_seq,
                 int32_t total_new_tokens, void *stream) {
  if (int rc = check_cache(cache)) return rc;
  if (batch < 0 || total_new_tokens < 0 || max_pages_per_seq < 0)
    return fail(SP_ERR_BAD_SHAPE, "negative count (batch=%d total_new_tokens=%d max_pages=%d)", batch,
                total_new_tokens, max_pages_per_seq);
  if (batch == 0 || total_new_tokens == 0) return SP_OK;
  if (!k_new || !v_new || !cu_seqlens_new || !ctx_lens || !block_table)
    return fail(SP_ERR_NULL, "sp_kv_append: NULL argument");
  if (max_pages_per_seq == 0) return fail(SP_ERR_BAD_SHAPE, "max_pages_per_seq=0 with tokens to append");
  return launch_kv_append(*cache, k_new, v_new, cu_seqlens_new, ctx_lens, block_table, batch,
                          max_pages_per_seq, total_new_tokens, (hipStream_t)stream);
}

int sp_attn_prefill(const sp_cache_desc *cache, const void *q, void *out,
                    const int32_t *cu_seqlens_q, const int32_t *ctx_lens,
                    const int32_t *block_table, int32_t batch, int32_t max_pages_per_seq,
                    int32_t total_q_tokens, int32_t max_q_len, int32_t max_kv_len,
                    int32_t num_q_heads, float scale, int32_t causal, void *workspace,
                    size_t workspace_bytes, void *stream) {
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_heads(cache, num_q_heads)) return rc;
  if (causal != 1) return fail(SP_ERR_UNSUPPORTED, "causal=%d (only causal attention)", causal);
  if (int rc = check_scale(scale)) return rc;
  if (batch < 0 || total_q_tokens < 0 || max_pages_per_seq < 0 || max_q_len < 0 || max_kv_len < 0)
    return fail(SP_ERR_BAD_SHAPE, "negative count in sp_attn_prefill");
  if (batch == 0 || total_q_tokens == 0 || max_q_len == 0) return SP_OK;
  if (!q || !out || !cu_seqlens_q || !ctx_lens || !block_table)
    return fail(SP_ERR_NULL, "sp_attn_prefill: NULL argument");
  if (max_pages_per_seq == 0) return fail(SP_ERR_BAD_SHAPE, "max_pages_per_seq=0 with queries");
  return launch_prefill(*cache, q, out, cu_seqlens_q, ctx_lens, block_table, batch, max_pages_per_seq,
                        total_q_tokens, max_q_len, max_kv_len, num_q_heads, scale,
                        workspace_bytes ? workspace : nullptr, workspace_bytes, (hipStream_t)stream);
}

int sp_chunk_step(const sp_cache_desc *cache, const void *k_new, const void *v_new, const void *q, void *out,
                  const int32_t *cu_seqlens_q, const int32_t *ctx_lens, const int32_t *block_table,
                  int32_t batch, int32_t max_pages_per_seq, int32_t total_q_tokens, int32_t max_q_len,
                  int32_t max_kv_len, int32_t num_q_heads, float scale, void *workspace, size_t workspace_bytes,
                  void *stream) {
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_heads(cache, num_q_heads)) return rc;
  if (int rc = check_scale(scale)) return rc;
  if (batch < 0 || total_q_tokens < 0 || max_pages_per_seq < 0 || max_q_len < 0 || max_kv_len < 0)
    return fail(SP_ERR_BAD_SHAPE, "negative count in sp_chunk_step");
  if (batch == 0 || total_q_tokens == 0 || max_q_len == 0) return SP_OK;
  if (!k_new || !v_new || !q || !out || !cu_seqlens_q || !ctx_lens || !block_table)
    return fail(SP_ERR_NULL, "sp_chunk_step: NULL argument");
  if (max_pages_per_seq == 0) return fail(SP_ERR_BAD_SHAPE, "max_pages_per_seq=0 with tokens to append");
  return launch_chunk_step(*cache, k_new, v_new, q, out, cu_seqlens_q, ctx_lens, block_table, batch,
                           max_pages_per_seq, total_q_tokens, max_q_len, max_kv_len, num_q_heads, scale,
                           workspace_bytes ? workspace : nullptr, workspace_bytes, (hipStream_t)stream);
}

static int decode_common(const char *name, const sp_cache_desc *cache, const void *k_new, const void *v_new,
                         const void *q, void *out, const int32_t *seq_lens, const int32_t *block_table,
                         int32_t batch, int32_t max_pages_per_seq, int32_t max_seq_len, int32_t num_q_heads,
                         float scale, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_heads(cache, num_q_heads)) return rc;
  if (int rc = check_scale(scale)) return rc;
  if (batch < 0 || max_pages_per_seq < 0 || max_seq_len < 0)
    return fail(SP_ERR_BAD_SHAPE, "negative count in %s", name);
  if (batch == 0) return SP_OK;
  if (!q || !out || !seq_lens || !block_table) return fail(SP_ERR_NULL, "%s: NULL argument", name);
  if (max_pages_per_seq == 0 && max_seq_len > 0)
    return fail(SP_ERR_BAD_SHAPE, "max_pages_per_seq=0 with max_seq_len=%d", max_seq_len);
  size_t need = decode_workspace_bytes(batch, max_seq_len, num_q_heads, cache->head_dim);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(SP_ERR_WORKSPACE, "decode workspace: need %zu bytes, got %zu", need,
                workspace ? workspace_bytes : (size_t)0);
  return launch_decode(*cache, k_new, v_new, q, out, seq_lens, block_table, batch, max_pages_per_seq,
                       max_seq_len, num_q_heads, scale, workspace, workspace_bytes, (hipStream_t)stream);
}

int sp_attn_decode(const sp_cache_desc *cache, const void *q, void *out, const int32_t *seq_lens,
                   const int32_t *block_table, int32_t batch, int32_t max_pages_per_seq,
                   int32_t max_seq_len, int32_t num_q_heads, float scale, void *workspace,
                   size_t workspace_bytes, void *stream) {
  return decode_common("sp_attn_decode", cache, nullptr, nullptr, q, out, seq_lens, block_table, batch,
                       max_pages_per_seq, max_seq_len, num_q_heads, scale, workspace, workspace_bytes, stream);
}

int sp_attn_decode_static(const sp_cache_desc *cache, const void *q, void *out, const int32_t *seq_lens,
                          const int32_t *block_table, int32_t batch, int32_t max_pages_per_seq, int32_t max_seq_len,
                          int32_t num_q_heads, float scale, void *stream) {
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_heads(cache, num_q_heads)) return rc;
  if (int rc = check_scale(scale)) return rc;
  if (batch < 0 || max_pages_per_seq < 0 || max_seq_len < 0)
    return fail(SP_ERR_BAD_SHAPE, "negative count in sp_attn_decode_static");
  if (batch == 0) return SP_OK;
  if (!q || !out || !seq_lens || !block_table) return fail(SP_ERR_NULL, "sp_attn_decode_static: NULL argument");
  if (max_pages_per_seq == 0 && max_seq_len > 0)
    return fail(SP_ERR_BAD_SHAPE, "max_pages_per_seq=0 with max_seq_len=%d", max_seq_len);
  return launch_decode_static(*cache, q, out, seq_lens, block_table, batch, max_pages_per_seq, max_seq_len,
                              num_q_heads, scale, (hipStream_t)stream);
}

int sp_decode_step(const sp_cache_desc *cache, const void *k_new, const void *v_new, const void *q, void *out,
                   const int32_t *seq_lens, const int32_t *block_table, int32_t batch,
                   int32_t max_pages_per_seq, int32_t max_seq_len, int32_t num_q_heads, float scale,
                   void *workspace, size_t workspace_bytes, void *stream) {
  if (batch > 0 && (!k_new || !v_new)) return fail(SP_ERR_NULL, "sp_decode_step: NULL k_new / v_new");
  return decode_common("sp_decode_step", cache, k_new, v_new, q, out, seq_lens, block_table, batch,
                       max_pages_per_seq, max_seq_len, num_q_heads, scale, workspace, workspace_bytes, stream);
}

int sp_attn_cross(const sp_cache_desc *cache, const void *q, void *out, const int32_t *cu_seqlens_q, const int32_t *kv_lens,
                  const int32_t *block_table, int32_t batch, int32_t max_pages_per_seq, int32_t total_q_tokens, int32_t max_q_len,
                  int32_t max_kv_len, int32_t num_q_heads, float scale, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_heads(cache, num_q_heads)) return rc;
  if (int rc = check_scale(scale)) return rc;
  if (batch < 0 || total_q_tokens < 0 || max_pages_per_seq < 0 || max_q_len < 0 || max_kv_len < 0)
    return fail(SP_ERR_BAD_SHAPE, "negative count in sp_attn_cross");
  if (batch == 0 || total_q_tokens == 0 || max_q_len == 0) return SP_OK;
  if (!q || !out || !cu_seqlens_q || !kv_lens || (!block_table && max_pages_per_seq > 0)) return fail(SP_ERR_NULL, "sp_attn_cross: NULL argument");
  if (max_pages_per_seq == 0 && max_kv_len > 0) return fail(SP_ERR_BAD_SHAPE, "max_pages_per_seq=0 with max_kv_len=%d", max_kv_len);
  return launch_cross(*cache, q, out, cu_seqlens_q, kv_lens, block_table, batch, max_pages_per_seq, total_q_tokens, max_q_len, max_kv_len,
                      num_q_heads, scale, workspace_bytes ? workspace : nullptr, workspace_bytes, (hipStream_t)stream);
}

size_t sp_attn_cross_workspace_size(int32_t batch, int32_t total_q_tokens, int32_t max_q_len, int32_t max_kv_len, int32_t num_q_heads,
                                    int32_t num_kv_heads, int32_t head_dim) {
  if (batch <= 0 || total_q_tokens <= 0 || max_q_len <= 0 || max_kv_len < 0 || num_q_heads <= 0 || num_kv_heads <= 0 || head_dim <= 0 ||
      num_q_heads % num_kv_heads != 0)
    return 0;
  return cross_workspace_bytes(batch, total_q_tokens, max_q_len, max_kv_len, num_q_heads, num_kv_heads, head_dim);
}

int sp_norm_rope_append(const sp_cache_desc *cache, const void *q, const void *k, const void *v, int64_t q_stride, int64_t k_stride,
                        int64_t v_stride, void *q_out, const void *q_weight, const void *k_weight, float eps, const sp_rope_desc *rope,
                        const int32_t *positions, const int32_t *cu_seqlens_new, const int32_t *ctx_lens, const int32_t *block_table,
                        int32_t batch, int32_t max_pages_per_seq, int32_t total_new_tokens, int32_t num_q_heads, void *stream) {
  if (int rc = check_cache(cache)) return rc;
  if (batch < 0 || total_new_tokens < 0 || max_pages_per_seq < 0 || num_q_heads < 0)
    return fail(SP_ERR_BAD_SHAPE, "negative count (batch=%d total_new_tokens=%d max_pages=%d num_q_heads=%d)", batch, total_new_tokens,
                max_pages_per_seq, num_q_heads);
  if (num_q_heads > 65536 || cache->num_kv_heads > 65536)
    return fail(SP_ERR_UNSUPPORTED, "num_q_heads=%d num_kv_heads=%d (at most 65536)", num_q_heads, cache->num_kv_heads);
  if ((q_weight || k_weight) && (!(eps >= 0.0f) || !std::isfinite(eps)))
    return fail(SP_ERR_UNSUPPORTED, "eps=%g must be finite and not negative", (double)eps);
  if (rope && rope->rotary_dim != 0) {
    if (rope->rotary_dim < 0 || rope->rotary_dim > cache->head_dim || rope->rotary_dim % 16 != 0)
      return fail(SP_ERR_UNSUPPORTED, "rotary_dim=%d must be a multiple of 16 up to head_dim=%d", rope->rotary_dim, cache->head_dim);
    if (rope->interleaved != 0 && rope->interleaved != 1) return fail(SP_ERR_UNSUPPORTED, "interleaved=%d (0 or 1)", rope->interleaved);
    if (rope->num_positions <= 0) return fail(SP_ERR_BAD_SHAPE, "num_positions=%d must be positive", rope->num_positions);
  }
  if (batch == 0 || total_new_tokens == 0) return SP_OK;
  const bool kv = k || v;
  if ((!k != !v) || (!kv && num_q_heads == 0)) return fail(SP_ERR_NULL, "sp_norm_rope_append: k and v, queries, or both");
  if ((num_q_heads > 0 && (!q || !q_out)) || !cu_seqlens_new || !ctx_lens || (kv && !block_table) ||
      (rope && rope->rotary_dim != 0 && !rope->cos_sin))
    return fail(SP_ERR_NULL, "sp_norm_rope_append: NULL argument");
  if (kv && max_pages_per_seq == 0) return fail(SP_ERR_BAD_SHAPE, "max_pages_per_seq=0 with tokens to append");
  const int64_t q_row = (int64_t)num_q_heads * cache->head_dim, kv_row = (int64_t)cache->num_kv_heads * cache->head_dim, most = INT64_MAX / 4 / total_new_tokens;
  if ((num_q_heads > 0 && (q_stride < q_row || q_stride > most)) || (kv && (k_stride < kv_row || k_stride > most || v_stride < kv_row || v_stride > most)))
    return fail(SP_ERR_BAD_SHAPE, "strides q %lld k %lld v %lld: tokens must not overlap", (long long)q_stride, (long long)k_stride, (long long)v_stride);
  if (num_q_heads > 0) {
    // a lane group writes a row after it has read the same row, and nothing else
    const long last = total_new_tokens - 1L, out_bytes = 2L * total_new_tokens * q_row;
    const bool in_place = q_out == q && (q_stride == q_row || total_new_tokens == 1);
    if ((!in_place && !apart(q_out, out_bytes, q, 2 * (last * q_stride + q_row))) ||
        (kv && (!apart(q_out, out_bytes, k, 2 * (last * k_stride + kv_row)) || !apart(q_out, out_bytes, v, 2 * (last * v_stride + kv_row)))))
      return fail(SP_ERR_UNSUPPORTED, "sp_norm_rope_append: q_out overlaps q, k or v");
  }
  return launch_norm_rope_append(*cache, q, k, v, q_stride, k_stride, v_stride, q_out, q_weight, k_weight, eps, rope, positions,
                                 cu_seqlens_new, ctx_lens, block_table, batch, max_pages_per_seq, total_new_tokens, num_q_heads,
                                 (hipStream_t)stream);
}

static int check_table(const sp_page_table *t) {
  if (!t) return fail(SP_ERR_NULL, "page table is NULL");
  if (t->num_pages <= 0 || t->num_rows < 0 || t->max_pages_per_seq < 0)
    return fail(SP_ERR_BAD_SHAPE, "num_pages=%d num_rows=%d max_pages_per_seq=%d", t->num_pages, t->num_rows, t->max_pages_per_seq);
  if (!t->ref_counts || (t->num_rows > 0 && (!t->seq_lens || (t->max_pages_per_seq > 0 && !t->block_table))))
    return fail(SP_ERR_NULL, "page table: NULL array");
  return SP_OK;
}

// A workgroup of 256 threads per entry, or per row: a launch has fewer than 2^32 threads.  Asked before the first of a call's launches.
constexpr int kMostEntries = 16000000;
static int check_entries(const char *name, int n) {
  return n <= kMostEntries ? SP_OK : fail(SP_ERR_UNSUPPORTED, "%s: %d entries (at most %d)", name, n, kMostEntries);
}

static int check_pages_workspace(const char *name, const sp_page_table *t, int n, const void *workspace, size_t bytes) {
  const size_t need = pages_workspace_bytes(t->num_pages, n);
  if (!workspace || bytes < need) return fail(SP_ERR_WORKSPACE, "%s workspace: need %zu bytes, got %zu", name, need, workspace ? bytes : (size_t)0);
  if ((uintptr_t)workspace % 16 != 0) return fail(SP_ERR_WORKSPACE, "%s workspace: not on a 16-byte boundary", name);
  return SP_OK;
}

int sp_pages_reserve(const sp_page_table *table, const int32_t *rows, const int32_t *new_lens, int32_t n, int32_t *shortfall,
                     void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_table(table)) return rc;
  if (n < 0) return fail(SP_ERR_BAD_SHAPE, "negative count in sp_pages_reserve");
  if (n == 0) return SP_OK;
  if (!rows || !new_lens || !shortfall) return fail(SP_ERR_NULL, "sp_pages_reserve: NULL argument");
  if (int rc = check_entries("sp_pages_reserve", n)) return rc;
  if (int rc = check_pages_workspace("sp_pages_reserve", table, n, workspace, workspace_bytes)) return rc;
  return launch_pages_reserve(*table, rows, new_lens, n, shortfall, workspace, (hipStream_t)stream);
}

int sp_pages_fork(const sp_page_table *table, const int32_t *parents, const int32_t *children, int32_t n, int32_t *copy_src,
                  int32_t *copy_dst, int32_t *copy_rows, int32_t *shortfall, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_table(table)) return rc;
  if (n < 0) return fail(SP_ERR_BAD_SHAPE, "negative count in sp_pages_fork");
  if (n == 0) return SP_OK;
  if (!parents || !children || !copy_src || !copy_dst || !copy_rows || !shortfall) return fail(SP_ERR_NULL, "sp_pages_fork: NULL argument");
  if (int rc = check_entries("sp_pages_fork", n)) return rc;
  if (int rc = check_pages_workspace("sp_pages_fork", table, n, workspace, workspace_bytes)) return rc;
  return launch_pages_fork(*table, parents, children, n, copy_src, copy_dst, copy_rows, shortfall, workspace, (hipStream_t)stream);
}

int sp_pages_release(const sp_page_table *table, const int32_t *rows, const int32_t *keep_lens, int32_t n, void *stream) {
  if (int rc = check_table(table)) return rc;
  if (n < 0) return fail(SP_ERR_BAD_SHAPE, "negative count in sp_pages_release");
  if (n == 0) return SP_OK;
  if (!rows) return fail(SP_ERR_NULL, "sp_pages_release: NULL argument");
  if (int rc = check_entries("sp_pages_release", n)) return rc;
  return launch_pages_release(*table, rows, keep_lens, n, (hipStream_t)stream);
}

int sp_pages_compact(const sp_page_table *table, int32_t *new_block_table, int32_t *new_ref_counts, int32_t *move_src, int32_t *move_dst,
                     int32_t *moved, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_table(table)) return rc;
  if ((table->num_rows > 0 && table->max_pages_per_seq > 0 && !new_block_table) || !new_ref_counts || !moved ||
      (table->num_pages > 1 && (!move_src || !move_dst)))
    return fail(SP_ERR_NULL, "sp_pages_compact: NULL argument");
  if (int rc = check_entries("sp_pages_compact, rows", table->num_rows)) return rc;
  if (int rc = check_pages_workspace("sp_pages_compact", table, 0, workspace, workspace_bytes)) return rc;
  return launch_pages_compact(*table, new_block_table, new_ref_counts, move_src, move_dst, moved, workspace, (hipStream_t)stream);
}

int sp_pages_copy(const sp_cache_desc *caches, int32_t num_caches, const int32_t *src, const int32_t *dst, const int32_t *rows,
                  const int32_t *count, int32_t n, void *stream) {
  if (n < 0 || num_caches < 0) return fail(SP_ERR_BAD_SHAPE, "negative count in sp_pages_copy");
  if (num_caches > 0 && !caches) return fail(SP_ERR_NULL, "sp_pages_copy: NULL argument");
  for (int i = 0; i < num_caches; ++i) {
    if (int rc = check_cache(caches + i)) return rc;
    if (caches[i].num_pages != caches[0].num_pages || caches[i].num_kv_heads != caches[0].num_kv_heads || caches[i].head_dim != caches[0].head_dim)
      return fail(SP_ERR_BAD_SHAPE, "sp_pages_copy: cache %d is not of the same shape as the first", i);
  }
  if (n == 0 || num_caches == 0) return SP_OK;
  if (caches[0].num_kv_heads > 65536) return fail(SP_ERR_UNSUPPORTED, "num_kv_heads=%d (at most 65536)", caches[0].num_kv_heads);
  if (!src || !dst) return fail(SP_ERR_NULL, "sp_pages_copy: NULL argument");
  return launch_pages_copy(caches, num_caches, src, dst, rows, count, n, (hipStream_t)stream);
}

size_t sp_pages_workspace_size(int32_t num_pages, int32_t n) { return num_pages <= 0 || n < 0 ? 0 : pages_workspace_bytes(num_pages, n); }

static int validate_pages(const sp_page_table *table) {
  std::vector<int32_t> entries((size_t)table->num_rows * table->max_pages_per_seq), refs(table->num_pages), lens(table->num_rows),
      held(table->num_pages, 0);
  hipError_t e = hipMemcpy(refs.data(), table->ref_counts, refs.size() * 4, hipMemcpyDeviceToHost);
  if (e == hipSuccess && !lens.empty()) e = hipMemcpy(lens.data(), table->seq_lens, lens.size() * 4, hipMemcpyDeviceToHost);
  if (e == hipSuccess && !entries.empty()) e = hipMemcpy(entries.data(), table->block_table, entries.size() * 4, hipMemcpyDeviceToHost);
  if (e != hipSuccess) return fail(SP_ERR_HIP, "hipMemcpy: %s", hipGetErrorString(e));
  for (int s = 0; s < table->num_rows; ++s) {
    const long pages = ((long)lens[s] + kPage - 1) / kPage;
    if (lens[s] < 0 || pages > table->max_pages_per_seq)
      return fail(SP_ERR_BAD_SHAPE, "seq_lens[%d]=%d does not fit a row of %d pages", s, lens[s], table->max_pages_per_seq);
    for (long p = 0; p < pages; ++p) {
      const int32_t pg = entries[(size_t)s * table->max_pages_per_seq + p];
      if (pg < 0 || pg >= table->num_pages) return fail(SP_ERR_BAD_SHAPE, "block_table[%d][%ld]=%d outside [0,%d)", s, p, pg, table->num_pages);
      ++held[pg];
    }
  }
  for (int p = 0; p < table->num_pages; ++p)
    if (held[p] != refs[p]) return fail(SP_ERR_BAD_SHAPE, "ref_counts[%d]=%d, held by %d entries", p, refs[p], held[p]);
  return SP_OK;
}

int sp_debug_validate_pages(const sp_page_table *table) {
  if (int rc = check_table(table)) return rc;
  return checked("sp_debug_validate_pages", [&] { return validate_pages(table); });
}

static int ulysses_common(bool pack, const void *src, void *dst, int32_t tokens, int32_t num_heads,
                          int32_t head_dim, int32_t world, void *stream) {
  if (tokens < 0 || num_heads <= 0 || world <= 0)
    return fail(SP_ERR_BAD_SHAPE, "tokens=%d num_heads=%d world=%d", tokens, num_heads, world);
  if (num_heads % world != 0)
    return fail(SP_ERR_BAD_SHAPE, "num_heads=%d is not a multiple of world=%d", num_heads, world);
  if (head_dim <= 0 || head_dim % 8 != 0)
    return fail(SP_ERR_UNSUPPORTED, "head_dim=%d must be a positive multiple of 8", head_dim);
  if (tokens == 0) return SP_OK;
  if (!src || !dst) return fail(SP_ERR_NULL, "ulysses permute: NULL buffer");
  if (src == dst) return fail(SP_ERR_UNSUPPORTED, "ulysses permute: in-place use is not supported");
  return launch_ulysses(pack, src, dst, tokens, num_heads, head_dim, world, (hipStream_t)stream);
}

int sp_ulysses_pack(const void *x, void *send, int32_t tokens, int32_t num_heads, int32_t head_dim,
                    int32_t world, void *stream) {
  return ulysses_common(true, x, send, tokens, num_heads, head_dim, world, stream);
}

int sp_ulysses_unpack(const void *recv, void *y, int32_t tokens, int32_t num_heads, int32_t head_dim,
                      int32_t world, void *stream) {
  return ulysses_common(false, recv, y, tokens, num_heads, head_dim, world, stream);
}

size_t sp_attn_prefill_workspace_size(int32_t batch, int32_t total_q_tokens, int32_t max_q_len,
                                      int32_t max_kv_len, int32_t num_q_heads, int32_t num_kv_heads,
                                      int32_t head_dim) {
  if (batch <= 0 || total_q_tokens <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || head_dim <= 0 ||
      num_q_heads % num_kv_heads != 0)
    return 0;
  return prefill_workspace_bytes(batch, total_q_tokens, max_q_len, max_kv_len, num_q_heads, num_kv_heads,
                                 head_dim);
}

size_t sp_attn_decode_workspace_size(int32_t batch, int32_t max_seq_len, int32_t num_q_heads,
                                     int32_t head_dim) {
  if (batch <= 0 || max_seq_len < 0 || num_q_heads <= 0 || head_dim <= 0) return 0;
  return decode_workspace_bytes(batch, max_seq_len, num_q_heads, head_dim);
}

static int validate_metadata(const sp_cache_desc *cache, const int32_t *seq_lens,
                             const int32_t *block_table, int32_t batch, int32_t max_pages_per_seq) {
  if (int rc = check_cache(cache)) return rc;
  if (batch < 0 || max_pages_per_seq < 0) return fail(SP_ERR_BAD_SHAPE, "negative count");
  if (batch == 0) return SP_OK;
  if (!seq_lens || !block_table) return fail(SP_ERR_NULL, "NULL metadata");
  std::vector<int32_t> lens(batch), bt((size_t)batch * max_pages_per_seq);
  hipError_t e = hipMemcpy(lens.data(), seq_lens, lens.size() * 4, hipMemcpyDeviceToHost);
  if (e == hipSuccess && !bt.empty())
    e = hipMemcpy(bt.data(), block_table, bt.size() * 4, hipMemcpyDeviceToHost);
  if (e != hipSuccess) return fail(SP_ERR_HIP, "hipMemcpy: %s", hipGetErrorString(e));
  for (int s = 0; s < batch; ++s) {
    if (lens[s] < 0) return fail(SP_ERR_BAD_SHAPE, "seq_lens[%d]=%d is negative", s, lens[s]);
    int pages = (lens[s] + kPage - 1) / kPage;
    if (pages > max_pages_per_seq)
      return fail(SP_ERR_BAD_SHAPE, "sequence %d needs %d pages > max_pages_per_seq=%d", s, pages,
                  max_pages_per_seq);
    for (int p = 0; p < pages; ++p) {
      int32_t pg = bt[(size_t)s * max_pages_per_seq + p];
      if (pg < 0 || pg >= cache->num_pages)
        return fail(SP_ERR_BAD_SHAPE, "block_table[%d][%d]=%d outside [0,%d)", s, p, pg, cache->num_pages);
    }
  }
  return SP_OK;
}

static int validate_hints(const int32_t *cu_seqlens, const int32_t *lens, int32_t batch, int32_t total_tokens,
                          int32_t max_q_len, int32_t max_len) {
  if (batch < 0) return fail(SP_ERR_BAD_SHAPE, "negative batch");
  if (batch == 0) return SP_OK;
  if (!lens) return fail(SP_ERR_NULL, "NULL length array");
  std::vector<int32_t> ln(batch), cu(cu_seqlens ? batch + 1 : 0);
  hipError_t e = hipMemcpy(ln.data(), lens, ln.size() * 4, hipMemcpyDeviceToHost);
  if (e == hipSuccess && cu_seqlens) e = hipMemcpy(cu.data(), cu_seqlens, cu.size() * 4, hipMemcpyDeviceToHost);
  if (e != hipSuccess) return fail(SP_ERR_HIP, "hipMemcpy: %s", hipGetErrorString(e));
  if (cu_seqlens) {
    if (cu[0] < 0) return fail(SP_ERR_BAD_SHAPE, "cu_seqlens[0]=%d is negative", cu[0]);
    if (cu[batch] > total_tokens)
      return fail(SP_ERR_BAD_SHAPE, "cu_seqlens[%d]=%d exceeds total_tokens=%d", batch, cu[batch], total_tokens);
  }
  for (int s = 0; s < batch; ++s) {
    if (ln[s] < 0) return fail(SP_ERR_BAD_SHAPE, "lens[%d]=%d is negative", s, ln[s]);
    long reach = ln[s];
    if (cu_seqlens) {
      const long n = (long)cu[s + 1] - cu[s];
      if (n < 0) return fail(SP_ERR_BAD_SHAPE, "cu_seqlens decreases at sequence %d (%d -> %d)", s, cu[s], cu[s + 1]);
      if (n > max_q_len) return fail(SP_ERR_BAD_SHAPE, "sequence %d has %ld tokens > max_q_len=%d", s, n, max_q_len);
      reach += n;
    }
    if (reach > max_len)
      return fail(SP_ERR_BAD_SHAPE, "sequence %d reaches %ld keys > the length hint %d", s, reach, max_len);
  }
  return SP_OK;
}

int sp_debug_validate_metadata(const sp_cache_desc *cache, const int32_t *seq_lens, const int32_t *block_table, int32_t batch,
                               int32_t max_pages_per_seq) {
  return checked("sp_debug_validate_metadata", [&] { return validate_metadata(cache, seq_lens, block_table, batch, max_pages_per_seq); });
}

int sp_debug_validate_hints(const int32_t *cu_seqlens, const int32_t *lens, int32_t batch, int32_t total_tokens, int32_t max_q_len,
                            int32_t max_len) {
  return checked("sp_debug_validate_hints", [&] { return validate_hints(cu_seqlens, lens, batch, total_tokens, max_q_len, max_len); });
}

int sp_debug_set_tuning(const char *key, int32_t value) {
  if (!key) return fail(SP_ERR_NULL, "tuning key is NULL");
  if (!strcmp(key, "decode_chunk")) {
    if (value != 0 && (value < 128 || value > 1024 || value % 32 != 0))
      return fail(SP_ERR_UNSUPPORTED, "decode_chunk=%d (0, or a multiple of 32 in [128, 1024])", value);
    set_decode_chunk(value);
    return SP_OK;
  }
  if (!strcmp(key, "decode_ring")) {
    if (value < 0 || value > 4) return fail(SP_ERR_UNSUPPORTED, "decode_ring=%d (0..4)", value);
    set_decode_ring(value);
    return SP_OK;
  }
  if (!strcmp(key, "decode_form")) {
    if (value < 0 || value > 3) return fail(SP_ERR_UNSUPPORTED, "decode_form=%d (0..3)", value);
    set_decode_form(value);
    return SP_OK;
  }
  if (!strcmp(key, "decode_fuse")) {
    if (value < 0 || value > 2) return fail(SP_ERR_UNSUPPORTED, "decode_fuse=%d (0, 1 or 2)", value);
    set_decode_fuse(value);
    return SP_OK;
  }
  if (!strcmp(key, "prefill_kv_splits")) {
    if (value < 0 || value > 16) return fail(SP_ERR_UNSUPPORTED, "prefill_kv_splits=%d (0..16)", value);
    set_prefill_kv_splits(value);
    return SP_OK;
  }
  if (!strcmp(key, "prefill_split")) {
    if (value < 0 || value > 2) return fail(SP_ERR_UNSUPPORTED, "prefill_split=%d (0, 1 or 2)", value);
    set_prefill_split(value);
    return SP_OK;
  }
  if (!strcmp(key, "prefill_cut")) {
    if (value < 0 || value > 2) return fail(SP_ERR_UNSUPPORTED, "prefill_cut=%d (0, 1 or 2)", value);
    set_prefill_cut(value);
    return SP_OK;
  }
  if (!strcmp(key, "combine_form")) {
    if (value < 0 || value > 2) return fail(SP_ERR_UNSUPPORTED, "combine_form=%d (0, 1 or 2)", value);
    set_combine_form(value);
    return SP_OK;
  }
  if (!strcmp(key, "prefill_order")) {
    if (value < 0 || value > 2) return fail(SP_ERR_UNSUPPORTED, "prefill_order=%d (0, 1 or 2)", value);
    set_prefill_order(value);
    return SP_OK;
  }
  if (!strcmp(key, "prefill_short_chunk")) {
    if (value < 0 || value > 1) return fail(SP_ERR_UNSUPPORTED, "prefill_short_chunk=%d (0 or 1)", value);
    set_prefill_short_chunk(value);
    return SP_OK;
  }
  return fail(SP_ERR_UNSUPPORTED, "unknown tuning key '%s'", key);
}

const char *sp_status_string(int status) {
  switch (status) {
    case SP_OK: return "SP_OK";
    case SP_ERR_NULL: return "SP_ERR_NULL";
    case SP_ERR_BAD_SHAPE: return "SP_ERR_BAD_SHAPE";
    case SP_ERR_UNSUPPORTED: return "SP_ERR_UNSUPPORTED";
    case SP_ERR_WORKSPACE: return "SP_ERR_WORKSPACE";
    case SP_ERR_HIP: return "SP_ERR_HIP";
    default: return "SP_ERR_UNKNOWN";
  }
}

const char *sp_last_error(void) { return g_err; }

int sp_version(void) { return 100; }

}  // extern "C"
