// Attention and the cache's pages for tensors: as the row operators are (rows_torch.cpp).
#include "tensors.h"

#include <c10/core/InferenceMode.h>

#include <cmath>
#include <tuple>

namespace {

// [tokens, heads, dim], the values of a head dense
struct Heads {
  int32_t n, h, d;
  int64_t token, head;
};
Heads heads_of(const Tensor &t, const char *name) {
  if (t.dim() != 3 || (t.stride(2) != 1 && t.size(2) > 1)) wrong(std::string(name) + " has to be [tokens, heads, dim] with dense heads");
  Heads r{size32(t.size(0)), size32(t.size(1)), size32(t.size(2)), 0, 0};
  // (what there is only one of has no stride)
  r.head = r.h > 1 ? t.stride(1) : r.d;
  r.token = r.n > 1 ? t.stride(0) : r.d;
  return r;
}
void bf16(const Tensor &t, const char *name) {
  if (t.scalar_type() != at::kBFloat16) wrong(std::string(name) + ": " + c10::toString(t.scalar_type()) + " is not bfloat16");
}
float scale_of(std::optional<double> scale, int32_t dim) { return (float)(scale ? *scale : 1.0 / std::sqrt((double)std::max(dim, 1))); }
int32_t size_or_all(int64_t v) { return (int32_t)std::max<int64_t>(std::min<int64_t>(v, INT_MAX), -1); }
bool within(const Heads &q) { return q.n < MOE_ROWS_LIMIT && q.h <= MOE_ATTEND_MAX_HEADS && q.d <= MOE_ATTEND_MAX_DIM; }

// [pages, heads, tokens of a page, dim]; pages may lie apart
struct Pages {
  int32_t n, h, page, d, fmt;
  int64_t stride;
};
Pages pages_of(const Tensor &k, const Tensor &v, const Maybe &k_scale, const Maybe &v_scale) {
  if (k.dim() != 4 || k.sizes() != v.sizes() || k.scalar_type() != v.scalar_type()) wrong("k_pages and v_pages have to be [pages, heads, page, dim] of one type");
  if (k.scalar_type() != at::kBFloat16 && k.scalar_type() != at::kChar) wrong(std::string("k_pages: ") + c10::toString(k.scalar_type()) + " is neither bfloat16 nor int8");
  Pages r{size32(k.size(0)), size32(k.size(1)), size32(k.size(2)), size32(k.size(3)), k.scalar_type() == at::kChar ? MOE_R_INT8 : MOE_R_BF16, 0};
  r.stride = r.n > 1 ? k.stride(0) : (int64_t)r.h * r.page * r.d;
  for (const Tensor *t : {&k, &v}) {
    bool dense = r.n <= 1 || t->stride(0) == r.stride;
    int64_t inner = 1;
    for (int i = 3; i > 0; --i) {
      dense &= t->size(i) <= 1 || t->stride(i) == inner;
      inner *= t->size(i);
    }
    if (!dense) wrong("the pages have to be dense, and of k and v equally far apart");
  }
  dense(k_scale, {r.n, r.h, r.page}, at::kFloat, "k_scale");
  dense(v_scale, {r.n, r.h, r.page}, at::kFloat, "v_scale");
  return r;
}

// (PyTorch refuses to count their changes, but only once they are made)
void writable(const Tensor &t, const char *name) {
  if (t.is_inference() && !c10::InferenceMode::is_enabled()) wrong(std::string(name) + " is of inference mode: it is written to in that mode only");
}
void writable(const Maybe &t, const char *name) {
  if (t) writable(*t, name);
}
void written(const Tensor &t) { t.unsafeGetTensorImpl()->bump_version(); }
void written(const Maybe &t) {
  if (t) written(*t);
}

std::tuple<Tensor, Tensor, Tensor, Tensor, Tensor> plan_pages(const Tensor &have, const Tensor &more, const Tensor &table, const Tensor &free,
                                                              int page, int64_t n_tokens, const Maybe &used) {
  if (have.dim() != 1 || table.dim() != 2 || free.dim() != 1) wrong("have and more have to be [sequences], table [sequences, pages], free [pages]");
  const int32_t n = size32(have.size(0)), width = size32(table.size(1)), n_free = size32(free.size(0));
  dense(have, {n}, at::kInt, "have");
  dense(more, {n}, at::kInt, "more");
  dense(table, {n, width}, at::kInt, "table");
  dense(free, {n_free}, at::kInt, "free");
  dense(used, {1}, at::kInt, "used");
  writable(table, "table");
  const int32_t t = size_or_all(n_tokens);
  const Place on(have);
  on.has(more, table, free, used);
  const bool ok = n <= MOE_ATTEND_MAX_SEQS && t >= 0 && t < MOE_ROWS_LIMIT;
  const Tensor offsets = fresh(have, {(int64_t)n + 1}, at::kInt, ok), slots = fresh(have, {t}, at::kInt, ok), positions = fresh(have, {t}, at::kInt, ok),
               lengths = fresh(have, {n}, at::kInt, ok), used_out = fresh(have, {1}, at::kInt, ok);
  check(moe_plan_pages(ints(have), ints(more), n, page, ints(free), n_free, static_cast<const int32_t *>(at_(used)), to_ints(table), width,
                       to_ints(offsets), to_ints(slots), to_ints(positions), t, to_ints(lengths), to_ints(used_out), on.stream()),
        "moe_plan_pages");
  written(table);
  return {offsets, slots, positions, lengths, used_out};
}

void store_pages(const Tensor &k, const Tensor &v, const Tensor &slots, const Tensor &k_pages, const Tensor &v_pages, const Maybe &k_scale,
                 const Maybe &v_scale) {
  no_history(k, v, k_pages, v_pages, k_scale, v_scale);
  const int fmt = format(k, "k");
  const Heads hk = heads_of(k, "k"), hv = heads_of(v, "v");
  const Pages c = pages_of(k_pages, v_pages, k_scale, v_scale);
  if (v.scalar_type() != k.scalar_type() || v.sizes() != k.sizes()) wrong("v has to have the shape and type of k");
  if (c.h != hk.h || c.d != hk.d) wrong("k has other heads than k_pages");
  dense(slots, {hk.n}, at::kInt, "slots");
  writable(k_pages, "k_pages");
  writable(v_pages, "v_pages");
  writable(k_scale, "k_scale");
  writable(v_scale, "v_scale");
  const Place on(k);
  on.has(v, slots, k_pages, v_pages, k_scale, v_scale);
  check(moe_store_pages(k.const_data_ptr(), v.const_data_ptr(), fmt, hk.token, hk.head, hv.token, hv.head, ints(slots), hk.n, hk.h, hk.d,
                        k_pages.mutable_data_ptr(), v_pages.mutable_data_ptr(), c.fmt, c.stride, c.n, c.page, to_floats(k_scale), to_floats(v_scale),
                        on.stream()),
        "moe_store_pages");
  written(k_pages);
  written(v_pages);
  written(k_scale);
  written(v_scale);
}

Tensor attend_pages(const Tensor &q, const Tensor &k_pages, const Tensor &v_pages, const Tensor &table, const Tensor &lengths, const Maybe &k_scale,
                    const Maybe &v_scale, std::optional<double> scale, int64_t window, int64_t sinks) {
  no_history(q, k_pages, v_pages, k_scale, v_scale);
  bf16(q, "q");
  const Heads h = heads_of(q, "q");
  const Pages c = pages_of(k_pages, v_pages, k_scale, v_scale);
  if (c.d != h.d) wrong("q has another dim than k_pages");
  if (table.dim() != 2) wrong("table has to be [sequences, pages]");
  const int32_t width = size32(table.size(1));
  dense(table, {h.n, width}, at::kInt, "table");
  dense(lengths, {h.n}, at::kInt, "lengths");
  const Place on(q);
  on.has(k_pages, v_pages, table, lengths, k_scale, v_scale);
  const bool ok = within(h) && h.n <= MOE_ATTEND_MAX_SEQS;
  const Tensor y = fresh(q, {h.n, h.h, h.d}, at::kBFloat16, ok);
  Maybe work;
  const size_t need = moe_attend_pages_bytes(h.n, h.h, c.h, h.d);
  if (need) work = fresh(q, {(int64_t)need}, at::kByte, ok);
  check(moe_attend_pages(q.const_data_ptr(), h.token, h.head, k_pages.const_data_ptr(), v_pages.const_data_ptr(), c.fmt, c.stride, c.n, c.page,
                         floats(k_scale), floats(v_scale), ints(table), width, ints(lengths), h.n, h.h, c.h, h.d, scale_of(scale, h.d),
                         size_or_all(window), size_or_all(sinks), y.mutable_data_ptr(), to(work), need, on.stream()),
        "moe_attend_pages");
  return y;
}

struct Packed {
  Heads q, k, v;
  int32_t n;
  const int32_t *k_offsets;
  bool ok;
};
Packed packed_of(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets, const Maybe &k_offsets) {
  bf16(q, "q");
  bf16(k, "k");
  bf16(v, "v");
  Packed r{heads_of(q, "q"), heads_of(k, "k"), heads_of(v, "v"), 0, nullptr, false};
  if (k.sizes() != v.sizes() || r.q.d != r.k.d) wrong("k and v have to have the same shape, and q their dim");
  if (offsets.dim() != 1 || offsets.size(0) < 1) wrong("offsets has to be [sequences + 1]");
  r.n = size32(offsets.size(0) - 1);
  dense(offsets, {(int64_t)r.n + 1}, at::kInt, "offsets");
  dense(k_offsets, {(int64_t)r.n + 1}, at::kInt, "k_offsets");
  if (!k_offsets && r.k.n != r.q.n) wrong("without k_offsets k has to have the rows of q");
  r.k_offsets = k_offsets ? ints(*k_offsets) : nullptr;
  r.ok = within(r.q) && within(r.k) && r.n <= MOE_ATTEND_MAX_SEQS;
  return r;
}

std::tuple<Tensor, Maybe, Maybe> attend_rows(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets, const Maybe &k_offsets,
                                      std::optional<double> scale, int64_t window, int64_t sinks, bool keep) {
  no_history(q, k, v);
  const Packed r = packed_of(q, k, v, offsets, k_offsets);
  const Place on(q);
  on.has(k, v, offsets, k_offsets);
  const Tensor y = fresh(q, {r.q.n, r.q.h, r.q.d}, at::kBFloat16, r.ok);
  Maybe lse, low;
  if (keep) {
    lse = fresh(q, {r.q.h, r.q.n}, at::kFloat, r.ok);
    low = fresh(q, {r.q.n, r.q.h, r.q.d}, at::kBFloat16, r.ok);
  }
  Maybe work;
  const size_t need = moe_attend_rows_bytes(r.q.n, r.k.n, r.n, r.q.h, r.k.h, r.q.d);
  if (need) work = fresh(q, {(int64_t)need}, at::kByte, r.ok);
  check(moe_attend_rows(q.const_data_ptr(), r.q.token, r.q.head, k.const_data_ptr(), r.k.token, r.k.head, v.const_data_ptr(), r.v.token, r.v.head,
                        ints(offsets), r.k_offsets, r.n, r.q.n, r.k.n, r.q.h, r.k.h, r.q.d, scale_of(scale, r.q.d), size_or_all(window),
                        size_or_all(sinks), y.mutable_data_ptr(), to(low), to_floats(lse), to(work), need, on.stream()),
        "moe_attend_rows");
  return {y, lse, low};
}

std::tuple<Tensor, Tensor, Tensor> attend_rows_backward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets, const Tensor &y,
                                                        const Tensor &lse, const Maybe &low, const Tensor &dy, const Maybe &k_offsets, std::optional<double> scale,
                                                        int64_t window, int64_t sinks) {
  no_history(q, k, v, y, lse, low, dy);
  const Packed r = packed_of(q, k, v, offsets, k_offsets);
  dense(y, {r.q.n, r.q.h, r.q.d}, at::kBFloat16, "y");
  dense(low, {r.q.n, r.q.h, r.q.d}, at::kBFloat16, "kept.low");
  dense(dy, {r.q.n, r.q.h, r.q.d}, at::kBFloat16, "dy");
  dense(lse, {r.q.h, r.q.n}, at::kFloat, "kept.lse");
  const Place on(q);
  on.has(k, v, offsets, k_offsets, y, lse, low, dy);
  const Tensor dq = fresh(q, {r.q.n, r.q.h, r.q.d}, at::kBFloat16, r.ok), dk = fresh(k, {r.k.n, r.k.h, r.k.d}, at::kBFloat16, r.ok),
               dv = fresh(v, {r.k.n, r.k.h, r.k.d}, at::kBFloat16, r.ok);
  Maybe work;
  const size_t need = moe_attend_rows_backward_bytes(r.q.n, r.k.n, r.n, r.q.h, r.k.h, r.q.d);
  if (need) work = fresh(q, {(int64_t)need}, at::kByte, r.ok);
  check(moe_attend_rows_backward(q.const_data_ptr(), r.q.token, r.q.head, k.const_data_ptr(), r.k.token, r.k.head, v.const_data_ptr(), r.v.token,
                                 r.v.head, ints(offsets), r.k_offsets, r.n, r.q.n, r.k.n, r.q.h, r.k.h, r.q.d, scale_of(scale, r.q.d),
                                 size_or_all(window), size_or_all(sinks), y.const_data_ptr(), at_(low), floats(lse), dy.const_data_ptr(), dq.mutable_data_ptr(),
                                 dk.mutable_data_ptr(), dv.mutable_data_ptr(), to(work), need, on.stream()),
        "moe_attend_rows_backward");
  return {dq, dk, dv};
}

}  // namespace

void bind_attention(py::module &m) {
  m.def("plan_pages", &plan_pages);
  m.def("store_pages", &store_pages);
  m.def("attend_pages", &attend_pages);
  m.def("attend_rows", &attend_rows);
  m.def("attend_rows_backward", &attend_rows_backward);
}
