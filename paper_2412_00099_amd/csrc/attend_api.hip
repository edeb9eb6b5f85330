// C entry points of attention and of the cache's pages: argument checks and launches, nothing else.
#include <algorithm>
#include <cmath>

#include "attend.h"
#include "rows.h"

using namespace moe;

namespace {

constexpr int64_t kMaxRows = MOE_ROWS_LIMIT;
constexpr int64_t kMaxStride = 1 << 23;  // elements: a tile of rows stays within 32 bits
constexpr int32_t kFar = 1 << 30;        // of fewer rows than kMaxRows: windows and sinks from here on are all the same

bool off(const void *p, int by) { return reinterpret_cast<uintptr_t>(p) % by != 0; }

int check_heads(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_kv_heads < 1 || n_heads < n_kv_heads || n_heads > MOE_ATTEND_MAX_HEADS || n_heads % n_kv_heads != 0)
    return fail(MOE_EINVAL, "bad n_heads=%d or n_kv_heads=%d", n_heads, n_kv_heads);
  if (head_dim < 8 || head_dim > MOE_ATTEND_MAX_DIM || head_dim % 8 != 0)
    return fail(MOE_EINVAL, "head_dim=%d is not a multiple of 8 in 8..%d", head_dim, MOE_ATTEND_MAX_DIM);
  return MOE_OK;
}

int check_seen(float softmax_scale, int32_t window, int32_t sinks) {
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale)) return fail(MOE_EINVAL, "softmax_scale must be finite and positive");
  if (window < 0 || sinks < 0) return fail(MOE_EINVAL, "bad window=%d or sinks=%d", window, sinks);
  return MOE_OK;
}

int check_seqs(int32_t n_seqs) {
  if (n_seqs < 0 || n_seqs > MOE_ATTEND_MAX_SEQS) return fail(MOE_EINVAL, "n_seqs=%d is not in 0..%d", n_seqs, MOE_ATTEND_MAX_SEQS);
  return MOE_OK;
}

// bf16 rows that are read 16 bytes at a time
int check_rows(const char *name, const void *p, int64_t token, int64_t head, int32_t n_heads, int32_t head_dim) {
  if (token < head_dim || token > kMaxStride || token % 8 != 0 || (n_heads > 1 && (head < head_dim || head > kMaxStride * MOE_ATTEND_MAX_HEADS)) || head % 8 != 0)
    return fail(MOE_EINVAL, "%s: strides have to be multiples of 8, %d or more and not larger than %lld", name, head_dim, (long long)kMaxStride);
  if (off(p, 16)) return fail(MOE_EINVAL, "%s has to be 16-byte aligned", name);
  return MOE_OK;
}

int page_bits(int32_t page) {
  int bits = 4;
  while (bits < 10 && (1 << bits) < page) ++bits;
  return (1 << bits) == page ? bits : -1;
}

int check_cache(const void *k, const void *v, int32_t fmt, int64_t page_stride, int32_t n_pages, int32_t page, const float *k_scale,
                const float *v_scale, int32_t n_kv_heads, int32_t head_dim) {
  if (fmt != MOE_R_BF16 && fmt != MOE_R_INT8) return fail(MOE_EINVAL, "a cache is bf16 or int8, not format %d", fmt);
  if (page_bits(page) < 0) return fail(MOE_EINVAL, "page=%d is not a power of two in 16..1024", page);
  if (n_pages < 0 || (int64_t)n_pages * page > INT32_MAX) return fail(MOE_EINVAL, "bad n_pages=%d", n_pages);
  if (page_stride < (int64_t)n_kv_heads * page * head_dim || page_stride > (int64_t)1 << 40 || page_stride * row_elem(fmt) % 16 != 0)
    return fail(MOE_EINVAL, "pages overlap or are not 16-byte aligned: bad page_stride=%lld", (long long)page_stride);
  if (n_pages > 0 && (!k || !v)) return fail(MOE_EINVAL, "k_pages_dev or v_pages_dev is NULL");
  if ((fmt == MOE_R_INT8) != (k_scale != nullptr) || (fmt == MOE_R_INT8) != (v_scale != nullptr))
    return fail(MOE_EINVAL, "k_scale_dev and v_scale_dev go with 8-bit codes");
  if (off(k, 16) || off(v, 16) || off(k_scale, 4) || off(v_scale, 4)) return fail(MOE_EINVAL, "a pointer of the cache is not aligned");
  return MOE_OK;
}

CacheParams cache(const void *k, const void *v, int64_t page_stride, int32_t n_pages, int32_t page, const float *k_scale, const float *v_scale,
                  int32_t n_kv_heads, int32_t head_dim) {
  return {const_cast<void *>(k), const_cast<void *>(v), const_cast<float *>(k_scale), const_cast<float *>(v_scale),
          page_stride, n_pages, page_bits(page), n_kv_heads, head_dim};
}

int check_attend_rows(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k, int64_t k_stride, int64_t k_head_stride,
                      const void *v, int64_t v_stride, int64_t v_head_stride, const int32_t *offsets, const int32_t *k_offsets,
                      int32_t n_seqs, int32_t n_rows, int32_t n_k_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                      float softmax_scale, int32_t window, int32_t sinks) {
  if (const int bad = check_heads(n_heads, n_kv_heads, head_dim)) return bad;
  if (const int bad = check_seen(softmax_scale, window, sinks)) return bad;
  if (const int bad = check_seqs(n_seqs)) return bad;
  if (n_rows < 0 || n_rows >= kMaxRows || n_k_rows < 0 || n_k_rows >= kMaxRows) return fail(MOE_EINVAL, "bad n_rows=%d or n_k_rows=%d", n_rows, n_k_rows);
  if (!k_offsets && n_k_rows != n_rows) return fail(MOE_EINVAL, "without k_offsets_dev q and k have the same rows");
  if (const int bad = check_rows("q_dev", q, q_stride, q_head_stride, n_heads, head_dim)) return bad;
  if (const int bad = check_rows("k_dev", k, k_stride, k_head_stride, n_kv_heads, head_dim)) return bad;
  if (const int bad = check_rows("v_dev", v, v_stride, v_head_stride, n_kv_heads, head_dim)) return bad;
  if (!offsets) return fail(MOE_EINVAL, "offsets_dev is NULL");
  if ((n_rows > 0 && !q) || (n_k_rows > 0 && (!k || !v))) return fail(MOE_EINVAL, "q_dev, k_dev or v_dev is NULL");
  if (off(offsets, 4) || off(k_offsets, 4)) return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  return MOE_OK;
}

AttendRowsParams rows_params(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k, int64_t k_stride, int64_t k_head_stride,
                             const void *v, int64_t v_stride, int64_t v_head_stride, const int32_t *offsets, const int32_t *k_offsets,
                             int32_t n_seqs, int32_t n_rows, int32_t n_k_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                             float softmax_scale, int32_t window, int32_t sinks) {
  AttendRowsParams p{};
  p.q = {q, q_stride, q_head_stride};
  p.k = {k, k_stride, k_head_stride};
  p.v = {v, v_stride, v_head_stride};
  p.offsets = offsets;
  p.k_offsets = k_offsets ? k_offsets : offsets;
  p.n_seqs = n_seqs;
  p.n_rows = n_rows;
  p.n_k_rows = n_k_rows;
  p.heads = n_heads;
  p.kv_heads = n_kv_heads;
  p.dim = head_dim;
  p.window = std::min(window, kFar);
  p.sinks = window > 0 ? std::min(sinks, kFar) : 0;
  p.scale = softmax_scale;
  return p;
}

}  // namespace

extern "C" {

int moe_plan_pages(const int32_t *have, const int32_t *more, int32_t n_seqs, int32_t page, const int32_t *free_pages, int32_t n_free,
                   const int32_t *used, int32_t *table, int32_t table_pages, int32_t *offsets, int32_t *slots, int32_t *positions,
                   int32_t n_tokens, int32_t *lengths, int32_t *used_out, void *stream) {
  if (const int bad = check_seqs(n_seqs)) return bad;
  if (page_bits(page) < 0) return fail(MOE_EINVAL, "page=%d is not a power of two in 16..1024", page);
  if (n_free < 0 || table_pages < 0) return fail(MOE_EINVAL, "bad n_free=%d or table_pages=%d", n_free, table_pages);
  if (n_tokens < 0 || n_tokens >= kMaxRows) return fail(MOE_EINVAL, "bad n_tokens=%d", n_tokens);
  if (!offsets || !used_out || (n_seqs > 0 && (!have || !more || !lengths)) || (n_seqs > 0 && table_pages > 0 && !table) ||
      (n_free > 0 && !free_pages) || (n_tokens > 0 && (!slots || !positions)))
    return fail(MOE_EINVAL, "a pointer is NULL");
  if (off(have, 4) || off(more, 4) || off(free_pages, 4) || off(used, 4) || off(table, 4) || off(offsets, 4) || off(slots, 4) || off(positions, 4) ||
      off(lengths, 4) || off(used_out, 4))
    return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  if (used_out == used || (n_seqs > 0 && (lengths == have || lengths == more))) return fail(MOE_EINVAL, "a result overlaps what is read");
  const PlanPagesParams p{have, more, free_pages, used, table, offsets, slots, positions, lengths, used_out, n_seqs, page_bits(page), n_free, table_pages, n_tokens};
  HIP_TRY(launch_plan_pages(p, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

int moe_store_pages(const void *k, const void *v, int32_t fmt, int64_t k_stride, int64_t k_head_stride, int64_t v_stride, int64_t v_head_stride,
                    const int32_t *slots, int32_t n_rows, int32_t n_kv_heads, int32_t head_dim, void *k_pages, void *v_pages, int32_t cache_fmt,
                    int64_t page_stride, int32_t n_pages, int32_t page, float *k_scale, float *v_scale, void *stream) {
  if (const int bad = check_heads(n_kv_heads, n_kv_heads, head_dim)) return bad;
  if (fmt != MOE_R_FP32 && fmt != MOE_R_BF16) return fail(MOE_EINVAL, "bad fmt=%d", fmt);
  if (n_rows < 0 || n_rows >= kMaxRows) return fail(MOE_EINVAL, "bad n_rows=%d", n_rows);
  if (const int bad = check_cache(k_pages, v_pages, cache_fmt, page_stride, n_pages, page, k_scale, v_scale, n_kv_heads, head_dim)) return bad;
  if (k_stride < 0 || v_stride < 0 || k_head_stride < 0 || v_head_stride < 0) return fail(MOE_EINVAL, "a stride is negative");
  if (n_rows == 0 || n_pages == 0) return MOE_OK;
  if (!k || !v || !slots) return fail(MOE_EINVAL, "k_dev, v_dev or slots_dev is NULL");
  if (off(k, row_elem(fmt)) || off(v, row_elem(fmt)) || off(slots, 4)) return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  HIP_TRY(launch_store_pages(cache(k_pages, v_pages, page_stride, n_pages, page, k_scale, v_scale, n_kv_heads, head_dim), cache_fmt,
                             {k, k_stride, k_head_stride}, {v, v_stride, v_head_stride}, fmt, slots, n_rows, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

size_t moe_attend_pages_bytes(int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_seqs <= 0 || n_seqs > MOE_ATTEND_MAX_SEQS || n_kv_heads < 1 || n_heads < n_kv_heads || n_heads > MOE_ATTEND_MAX_HEADS || head_dim < 8 ||
      head_dim > MOE_ATTEND_MAX_DIM)
    return 0;
  return attend_pages_bytes(n_seqs, n_heads, n_kv_heads, head_dim);
}

int moe_attend_pages(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k_pages, const void *v_pages, int32_t cache_fmt,
                     int64_t page_stride, int32_t n_pages, int32_t page, const float *k_scale, const float *v_scale, const int32_t *table,
                     int32_t table_pages, const int32_t *lengths, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                     float softmax_scale, int32_t window, int32_t sinks, void *y, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int bad = check_heads(n_heads, n_kv_heads, head_dim)) return bad;
  if (const int bad = check_seen(softmax_scale, window, sinks)) return bad;
  if (const int bad = check_seqs(n_seqs)) return bad;
  if (table_pages < 0) return fail(MOE_EINVAL, "bad table_pages=%d", table_pages);
  if (const int bad = check_cache(k_pages, v_pages, cache_fmt, page_stride, n_pages, page, k_scale, v_scale, n_kv_heads, head_dim)) return bad;
  if (const int bad = check_rows("q_dev", q, q_stride, q_head_stride, n_heads, head_dim)) return bad;
  if (n_seqs == 0) return MOE_OK;
  if (!q || !lengths || !y || (table_pages > 0 && !table)) return fail(MOE_EINVAL, "q_dev, table_dev, lengths_dev or y_dev is NULL");
  if (off(table, 4) || off(lengths, 4) || off(y, 16)) return fail(MOE_EINVAL, "a pointer is not aligned");
  const size_t need = moe_attend_pages_bytes(n_seqs, n_heads, n_kv_heads, head_dim);
  if (!workspace || off(workspace, 16) || workspace_bytes < need) return fail(MOE_EINVAL, "a workspace of %zu bytes, 16-byte aligned, is needed", need);
  AttendPagesParams p{};
  p.c = cache(k_pages, v_pages, page_stride, n_pages, page, k_scale, v_scale, n_kv_heads, head_dim);
  p.q = {q, q_stride, q_head_stride};
  p.table = table;
  p.lengths = lengths;
  p.y = static_cast<uint16_t *>(y);
  p.parts = static_cast<float *>(workspace);
  p.scale = softmax_scale;
  p.n_seqs = n_seqs;
  p.table_pages = table_pages;
  p.heads = n_heads;
  p.window = window;  // (a table may hold a page many times: 2^31 - 1 tokens are possible)
  p.sinks = window > 0 ? sinks : 0;
  HIP_TRY(launch_attend_pages(p, cache_fmt, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

size_t moe_attend_rows_bytes(int32_t n_rows, int32_t n_k_rows, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_rows < 0 || n_rows >= kMaxRows || n_k_rows < 0 || n_k_rows >= kMaxRows || n_seqs < 0 || n_seqs > MOE_ATTEND_MAX_SEQS || n_kv_heads < 1 ||
      n_heads < n_kv_heads || n_heads > MOE_ATTEND_MAX_HEADS || head_dim < 8 || head_dim > MOE_ATTEND_MAX_DIM)
    return 0;
  return attend_rows_bytes(n_rows, n_k_rows, n_seqs, n_heads, head_dim);
}

int moe_attend_rows(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k, int64_t k_stride, int64_t k_head_stride, const void *v,
                    int64_t v_stride, int64_t v_head_stride, const int32_t *offsets, const int32_t *k_offsets, int32_t n_seqs, int32_t n_rows,
                    int32_t n_k_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float softmax_scale, int32_t window, int32_t sinks,
                    void *y, void *y_low, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int bad = check_attend_rows(q, q_stride, q_head_stride, k, k_stride, k_head_stride, v, v_stride, v_head_stride, offsets, k_offsets,
                                        n_seqs, n_rows, n_k_rows, n_heads, n_kv_heads, head_dim, softmax_scale, window, sinks))
    return bad;
  if (n_rows == 0) return MOE_OK;
  if (!y || off(y, 16) || off(y_low, 16) || off(lse, 4)) return fail(MOE_EINVAL, "y_dev is NULL, or a pointer is not aligned");
  const size_t need = moe_attend_rows_bytes(n_rows, n_k_rows, n_seqs, n_heads, n_kv_heads, head_dim);
  if (need > 0 && (!workspace || off(workspace, 16) || workspace_bytes < need))
    return fail(MOE_EINVAL, "a workspace of %zu bytes, 16-byte aligned, is needed", need);
  AttendRowsParams p = rows_params(q, q_stride, q_head_stride, k, k_stride, k_head_stride, v, v_stride, v_head_stride, offsets, k_offsets, n_seqs,
                                   n_rows, n_k_rows, n_heads, n_kv_heads, head_dim, softmax_scale, window, sinks);
  p.y = static_cast<uint16_t *>(y);
  p.low = static_cast<uint16_t *>(y_low);
  p.lse = lse;
  HIP_TRY(launch_attend_rows(p, static_cast<uint8_t *>(workspace), static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

size_t moe_attend_rows_backward_bytes(int32_t n_rows, int32_t n_k_rows, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_rows < 0 || n_rows >= kMaxRows || n_k_rows < 0 || n_k_rows >= kMaxRows || n_seqs < 0 || n_seqs > MOE_ATTEND_MAX_SEQS || n_kv_heads < 1 ||
      n_heads < n_kv_heads || n_heads > MOE_ATTEND_MAX_HEADS || head_dim < 8 || head_dim > MOE_ATTEND_MAX_DIM)
    return 0;
  return attend_rows_backward_bytes(n_rows, n_k_rows, n_seqs, n_heads, n_kv_heads, head_dim);
}

int moe_attend_rows_backward(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k, int64_t k_stride, int64_t k_head_stride,
                             const void *v, int64_t v_stride, int64_t v_head_stride, const int32_t *offsets, const int32_t *k_offsets,
                             int32_t n_seqs, int32_t n_rows, int32_t n_k_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                             float softmax_scale, int32_t window, int32_t sinks, const void *y, const void *y_low, const float *lse, const void *dy,
                             void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int bad = check_attend_rows(q, q_stride, q_head_stride, k, k_stride, k_head_stride, v, v_stride, v_head_stride, offsets, k_offsets,
                                        n_seqs, n_rows, n_k_rows, n_heads, n_kv_heads, head_dim, softmax_scale, window, sinks))
    return bad;
  if (n_rows > 0 && (!y || !lse || !dy || !dq)) return fail(MOE_EINVAL, "y_dev, lse_dev, dy_dev or dq_dev is NULL");
  if (n_k_rows > 0 && (!dk || !dv)) return fail(MOE_EINVAL, "dk_dev or dv_dev is NULL");
  if (off(y, 16) || off(y_low, 16) || off(dy, 16) || off(dq, 16) || off(dk, 16) || off(dv, 16) || off(lse, 4)) return fail(MOE_EINVAL, "a pointer is not aligned");
  const size_t need = moe_attend_rows_backward_bytes(n_rows, n_k_rows, n_seqs, n_heads, n_kv_heads, head_dim);
  if (n_rows == 0 && n_k_rows == 0) return MOE_OK;
  if (!workspace || off(workspace, 16) || workspace_bytes < need)
    return fail(MOE_EINVAL, "a workspace of %zu bytes, 16-byte aligned, is needed", need);
  AttendRowsParams p = rows_params(q, q_stride, q_head_stride, k, k_stride, k_head_stride, v, v_stride, v_head_stride, offsets, k_offsets, n_seqs,
                                   n_rows, n_k_rows, n_heads, n_kv_heads, head_dim, softmax_scale, window, sinks);
  p.y = static_cast<uint16_t *>(const_cast<void *>(y));
  p.low = static_cast<uint16_t *>(const_cast<void *>(y_low));
  p.lse = const_cast<float *>(lse);
  p.dy = static_cast<const uint16_t *>(dy);
  p.dq = static_cast<uint16_t *>(dq);
  p.dk = static_cast<uint16_t *>(dk);
  p.dv = static_cast<uint16_t *>(dv);
  HIP_TRY(launch_attend_rows_backward(p, static_cast<uint8_t *>(workspace), static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

}  // extern "C"
