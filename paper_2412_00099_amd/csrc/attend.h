// Attention: what the translation units share.
#pragma once

#include "common.h"

namespace moe {

// elements between tokens and between heads
struct HeadRows {
  const void *at;
  int64_t token, head;
};

// ---- pages.hip ----
struct PlanPagesParams {
  const int32_t *have, *more, *free, *used;  // used may be NULL
  int32_t *table, *offsets, *slots, *positions, *lengths, *used_out;
  int32_t n_seqs, page_bits, n_free, table_pages, n_tokens;
};
hipError_t launch_plan_pages(const PlanPagesParams &p, hipStream_t s);

// A cache: [n_pages][kv_heads][page][dim], pages `page_stride` elements apart; scales [n_pages][kv_heads][page]
struct CacheParams {
  void *k, *v;
  float *k_scale, *v_scale;
  int64_t page_stride;
  int32_t n_pages, page_bits, kv_heads, dim;  // a page has 1 << page_bits tokens
};
hipError_t launch_store_pages(const CacheParams &c, int cache_fmt, const HeadRows &k, const HeadRows &v, int fmt, const int32_t *slots,
                              int n_rows, hipStream_t s);

// ---- attend_pages.hip ----
struct AttendPagesParams {
  CacheParams c;
  HeadRows q;
  const int32_t *table, *lengths;
  uint16_t *y;
  float *parts;        // see attend_pages.hip
  float scale;
  int32_t n_seqs, table_pages, heads, window, sinks;
};
size_t attend_pages_bytes(int n_seqs, int heads, int kv_heads, int dim);
hipError_t launch_attend_pages(const AttendPagesParams &p, int cache_fmt, hipStream_t s);

// ---- attend_rows.hip ----
// Some of the queries that see some keys: see attend_rows.hip
struct KeyPiece {
  int sequence, part, first, count;  // tiles `first` on of the list
  int index, of, slot;               // which of how many pieces; where the sums of the list's first piece are (of > 1)
};
struct AttendRowsParams {
  HeadRows q, k, v;
  const int32_t *offsets, *k_offsets;
  int32_t n_seqs, n_rows, n_k_rows, heads, kv_heads, dim, window, sinks;
  float scale;
  uint16_t *y;
  uint16_t *low;  // y's rounding, or NULL
  float *lse;     // [heads][n_rows], forward: may be NULL
  int32_t splits; // shares of the keys of 128 queries; more than one, forward: stats [parts][splits][heads][128 queries][4], sums [...][128][dim]
  // backward
  const uint16_t *dy;
  uint16_t *dq, *dk, *dv;
  float *stats;  // [2][heads][n_rows]: -lse to the base 2, -<dy, y>
  int32_t *n_pieces;
  KeyPiece *pieces;
  float *sums;  // [max_slots][kv_heads][128 keys][2][dim]: of pieces
  float *q_sums;  // [parts][splits][heads][128 queries][dim]: of shares
  int32_t max_pieces, max_slots, shares;
};
size_t attend_rows_bytes(int n_rows, int n_k_rows, int n_seqs, int heads, int dim);
hipError_t launch_attend_rows(const AttendRowsParams &p, uint8_t *workspace, hipStream_t s);
size_t attend_rows_backward_bytes(int n_rows, int n_k_rows, int n_seqs, int heads, int kv_heads, int dim);
hipError_t launch_attend_rows_backward(const AttendRowsParams &p, uint8_t *workspace, hipStream_t s);

}  // namespace moe
