// The row operators for tensors, the part that every call goes through: checks of shapes, types, places and history, the outputs from
// PyTorch's allocator, the current stream, the call of the C entry point.  In Python this took 10.5 us a call where the kernel takes 3 (a
// norm of 37 rows), here 5.9.
#include "tensors.h"

#include <tuple>

namespace {

std::tuple<Tensor, Tensor, Maybe, Tensor> norm_rows(const Tensor &h, const Maybe &y, const Maybe &gain, double eps, int x_fmt) {
  no_history(h, y, gain);
  const int h_fmt = format(h, "h");
  const Rows r = rows_of(h, "h");
  int y_fmt = h_fmt;
  int64_t y_stride = r.d;
  if (y) {
    y_fmt = format(*y, "y");
    const Rows ry = rows_of(*y, "y");
    if (ry.n != r.n || ry.d != r.d) wrong("y has to have the shape of h");
    y_stride = ry.stride;
  }
  dense(gain, {r.d}, at::kFloat, "gain");
  const Place on(h);
  on.has(y, gain);
  const bool ok = within(r.n, r.d);
  const Tensor h_out = y ? fresh(h, {r.n, r.d}, h.scalar_type(), ok) : h;
  const Tensor x = fresh(h, {r.n, r.d}, x_fmt == MOE_R_FP32 ? at::kFloat : x_fmt == MOE_R_BF16 ? at::kBFloat16 : at::kChar, ok);
  const Tensor rstd = fresh(h, {r.n}, at::kFloat, ok);
  Maybe scale;
  if (x_fmt == MOE_R_INT8) scale = fresh(h, {r.n}, at::kFloat, ok);
  check(moe_norm_rows(h.const_data_ptr(), h_fmt, r.stride, at_(y), y_fmt, y_stride, floats(gain), (float)eps, r.n, r.d,
                      y ? h_out.mutable_data_ptr() : nullptr, x.mutable_data_ptr(), x_fmt, to_floats(scale), to_floats(rstd), on.stream()),
        "moe_norm_rows");
  return {h_out, x, scale, rstd};
}

std::tuple<Tensor, Maybe> norm_rows_backward(const Tensor &rows, const Maybe &gain, const Tensor &rstd, const Tensor &dx, const Maybe &dh) {
  no_history(rows, gain, rstd, dx, dh);
  const int h_fmt = format(rows, "h"), x_fmt = format(dx, "dx");
  const Rows r = rows_of(rows, "h");
  dense(dx, {r.n, r.d}, {}, "dx");
  dense(dh, {r.n, r.d}, rows.scalar_type(), "dh");
  dense(gain, {r.d}, at::kFloat, "gain");
  dense(rstd, {r.n}, at::kFloat, "rstd");
  const Place on(rows);
  on.has(gain, rstd, dx, dh);
  // (without y norm_rows hands back the rows that it was given, which may lie apart; the library takes dense ones)
  const Tensor h = rows.contiguous();
  const bool ok = within(r.n, r.d);
  const Tensor out = fresh(h, {r.n, r.d}, h.scalar_type(), ok);
  Maybe dgain, work;
  const size_t need = gain ? moe_norm_rows_backward_bytes(r.n, r.d) : 0;
  if (gain) dgain = fresh(h, {r.d}, at::kFloat, ok);
  if (need) work = fresh(h, {(int64_t)need}, at::kByte, ok);
  check(moe_norm_rows_backward(h.const_data_ptr(), h_fmt, floats(gain), floats(rstd), dx.const_data_ptr(), x_fmt, at_(dh), r.n, r.d,
                               out.mutable_data_ptr(), to_floats(dgain), to(work), need, on.stream()),
        "moe_norm_rows_backward");
  return {out, dgain};
}

struct Order {
  int32_t t, k, e;
  bool within(int64_t hidden) const { return k <= MOE_MAX_TOPK && e <= MOE_ROWS_MAX_EXPERTS && ::within((int64_t)t * k, hidden); }
};

std::tuple<Tensor, Tensor, Tensor> sort_tokens(const Tensor &ids, int n_experts) {
  if (ids.dim() != 2) wrong("ids has to be [tokens, top_k]");
  const int32_t t = size32(ids.size(0)), k = size32(ids.size(1));
  dense(ids, {t, k}, at::kInt, "ids");
  if (n_experts < 1) wrong("n_experts has to be 1 or more");
  const Place on(ids);
  const bool ok = Order{t, k, n_experts}.within(1);
  const Tensor offsets = fresh(ids, {(int64_t)n_experts + 1}, at::kInt, ok), row_of = fresh(ids, {t, k}, at::kInt, ok),
               entry_of = fresh(ids, {(int64_t)t * k}, at::kInt, ok);
  Maybe work;
  const size_t need = moe_sort_tokens_bytes(t, k, n_experts);
  if (need) work = fresh(ids, {(int64_t)need}, at::kByte, ok);
  check(moe_sort_tokens(ints(ids), t, k, n_experts, to_ints(offsets), to_ints(row_of), to_ints(entry_of), to(work), need, on.stream()),
        "moe_sort_tokens");
  return {offsets, row_of, entry_of};
}

Order order_of(const Tensor &offsets, const Tensor &row_of) {
  if (row_of.dim() != 2 || offsets.dim() != 1) wrong("row_of has to be [tokens, top_k], offsets [n_experts + 1]");
  const Order o{size32(row_of.size(0)), size32(row_of.size(1)), size32(offsets.size(0) - 1)};
  dense(row_of, {o.t, o.k}, at::kInt, "row_of");
  dense(offsets, {o.e + 1}, at::kInt, "offsets");
  return o;
}

std::tuple<Tensor, Maybe> gather_rows(const Tensor &x, const Tensor &offsets, const Tensor &row_of, const Maybe &scale) {
  no_history(x, scale);
  const Order o = order_of(offsets, row_of);
  const int fmt = format(x, "x", true);
  const Rows r = rows_of(x, "x");
  if (r.n != o.t) wrong("x has to have a row for each token");
  dense(scale, {o.t}, at::kFloat, "scale");
  const Place on(x);
  on.has(scale, row_of, offsets);
  const int64_t n = (int64_t)o.t * o.k;
  const bool ok = o.within(r.d);
  const Tensor xs = fresh(x, {n, r.d}, x.scalar_type(), ok);
  Maybe xs_scale;
  if (scale) xs_scale = fresh(x, {n}, at::kFloat, ok);
  check(moe_gather_rows(x.const_data_ptr(), fmt, r.stride, floats(scale), ints(row_of), ints(offsets), o.t, o.k, o.e, r.d, xs.mutable_data_ptr(),
                        to_floats(xs_scale), on.stream()),
        "moe_gather_rows");
  return {xs, xs_scale};
}

// y_fmt: of the result; -1: that of base, or of ys
Tensor combine_rows(const Tensor &ys, const Tensor &offsets, const Tensor &row_of, const Maybe &weight, const Maybe &base, int y_fmt) {
  no_history(ys, weight, base);
  const Order o = order_of(offsets, row_of);
  const int ys_fmt = format(ys, "ys"), base_fmt = base ? format(*base, "base") : ys_fmt;
  const int64_t n = (int64_t)o.t * o.k;
  const int32_t d = ys.dim() > 0 ? size32(ys.size(-1)) : 0;
  dense(ys, {n, d}, {}, "ys");
  dense(weight, {o.t, o.k}, at::kFloat, "weight");
  if (y_fmt < 0) y_fmt = base_fmt;
  const at::ScalarType type = y_fmt == MOE_R_FP32 ? at::kFloat : at::kBFloat16;
  dense(base, {o.t, d}, type, "base");
  const Place on(ys);
  on.has(weight, base, row_of);
  const Tensor y = fresh(ys, {o.t, d}, type, Order{o.t, o.k, 1}.within(d));
  check(moe_combine_rows(ys.const_data_ptr(), ys_fmt, ints(row_of), floats(weight), at_(base), o.t, o.k, d, y.mutable_data_ptr(), y_fmt, on.stream()),
        "moe_combine_rows");
  return y;
}

std::tuple<Tensor, Maybe> combine_rows_backward(const Tensor &dy, const Tensor &ys, const Tensor &offsets, const Tensor &row_of, const Maybe &weight) {
  no_history(dy, ys, weight);
  const Order o = order_of(offsets, row_of);
  const int dy_fmt = format(dy, "dy"), ys_fmt = format(ys, "ys");
  const int64_t n = (int64_t)o.t * o.k;
  const int32_t d = dy.dim() > 0 ? size32(dy.size(-1)) : 0;
  dense(dy, {o.t, d}, {}, "dy");
  dense(ys, {n, d}, {}, "ys");
  dense(weight, {o.t, o.k}, at::kFloat, "weight");
  const Place on(dy);
  on.has(ys, weight, row_of, offsets);
  const bool ok = o.within(d);
  const Tensor dys = fresh(ys, {n, d}, ys.scalar_type(), ok);
  Maybe dweight;
  if (weight) dweight = fresh(ys, {o.t, o.k}, at::kFloat, ok);
  check(moe_combine_rows_backward(dy.const_data_ptr(), dy_fmt, ys.const_data_ptr(), ys_fmt, ints(row_of), ints(offsets), floats(weight), o.t, o.k, o.e,
                                  d, dys.mutable_data_ptr(), to_floats(dweight), on.stream()),
        "moe_combine_rows_backward");
  return {dys, dweight};
}

struct Shape {
  int32_t e, n, d, pitch;
  int64_t blob;  // bytes, at least `bytes` if ok
  int64_t bytes;
  bool ok;       // see fresh
};
Shape shape_of(int fmt, const Tensor &blobs, int inter, const Tensor &xs, const Tensor &offsets) {
  if (offsets.dim() != 1 || offsets.size(0) < 2 || blobs.dim() < 1 || !blobs.is_contiguous() || blobs.size(0) != offsets.size(0) - 1)
    wrong("blobs has to be contiguous, one blob for each expert of offsets");
  const at::ScalarType type = blobs.scalar_type();
  if (type != at::kByte && type != at::kChar && !(type == at::kBFloat16 && fmt == MOE_W_BF16))
    wrong(std::string("blobs: packed experts are bytes") + (fmt == MOE_W_BF16 ? " or bfloat16, not " : ", not ") + c10::toString(type));
  const int32_t e = size32(blobs.size(0));
  dense(offsets, {(int64_t)e + 1}, at::kInt, "offsets");
  if (xs.dim() != 2) wrong("xs has to be a matrix");
  if (inter < 0 || inter > INT_MAX - 64) wrong("bad inter");
  Shape s{e, size32(xs.size(0)), size32(xs.size(1)), (inter + 63) / 64 * 64, (int64_t)blobs.nbytes() / e, 0, false};
  s.bytes = (int64_t)moe_blob_bytes(fmt, s.d, inter);
  s.ok = s.bytes > 0 && s.bytes <= s.blob && e <= MOE_ROWS_MAX_EXPERTS && within(s.n, s.d);
  dense(xs, {s.n, s.d}, fmt == MOE_W_INT8_PC ? at::kChar : at::kBFloat16, "xs");
  return s;
}

std::tuple<Tensor, Maybe, Maybe> experts_rows(int fmt, const Tensor &blobs, int inter, const Tensor &xs, const Tensor &offsets, const Maybe &scale,
                                              bool keep) {
  no_history(blobs, xs, scale);
  const Shape s = shape_of(fmt, blobs, inter, xs, offsets);
  dense(scale, {s.n}, at::kFloat, "scale");
  const Place on(xs);
  on.has(blobs, offsets, scale);
  const Tensor h = fresh(xs, {s.n, s.pitch}, at::kBFloat16, s.ok), ys = fresh(xs, {s.n, s.d}, at::kBFloat16, s.ok);
  Maybe gu;
  if (keep) gu = fresh(xs, {s.n, 2, s.pitch}, at::kFloat, s.ok);
  check(moe_experts_rows(fmt, s.d, inter, s.e, blobs.const_data_ptr(), s.blob, xs.const_data_ptr(), floats(scale), ints(offsets), s.n,
                         h.mutable_data_ptr(), to_floats(gu), ys.mutable_data_ptr(), on.stream()),
        "moe_experts_rows");
  return {ys, keep ? Maybe(h) : Maybe(), gu};
}

std::tuple<Maybe, Maybe> experts_rows_backward(int fmt, const Tensor &blobs, int inter, const Tensor &xs, const Tensor &offsets, const Tensor &h,
                                               const Tensor &gu, const Tensor &dys, bool rows, bool weights) {
  no_history(blobs, xs, h, gu, dys);
  const Shape s = shape_of(fmt, blobs, inter, xs, offsets);
  dense(dys, {s.n, s.d}, at::kBFloat16, "dys");
  dense(h, {s.n, s.pitch}, at::kBFloat16, "kept.h");
  dense(gu, {s.n, 2, s.pitch}, at::kFloat, "kept.gu");
  const Place on(xs);
  on.has(blobs, offsets, dys, h, gu);
  const Tensor dgu = fresh(xs, {s.n, 2, s.pitch}, at::kBFloat16, s.ok);
  Maybe dxs, dblobs;
  if (rows) dxs = fresh(xs, {s.n, s.d}, xs.scalar_type(), s.ok);
  if (weights) dblobs = fresh(blobs, blobs.sizes(), blobs.scalar_type(), s.ok);
  check(moe_experts_rows_backward(fmt, s.d, inter, s.e, blobs.const_data_ptr(), s.blob, xs.const_data_ptr(), ints(offsets), s.n, h.const_data_ptr(),
                                  floats(gu), dys.const_data_ptr(), dgu.mutable_data_ptr(), to(dxs), to(dblobs), on.stream()),
        "moe_experts_rows_backward");
  // what lies between blobs has no gradient, and the library leaves it alone
  if (weights && s.blob > s.bytes) dblobs->view({s.e, -1}).view(at::kByte).slice(1, s.bytes).zero_();
  return {dxs, dblobs};
}

}  // namespace

PYBIND11_MODULE(_rows, m) {
  m.def("raise_as", [](py::object type) { error_type = new py::object(std::move(type)); });
  m.def("norm_rows", &norm_rows);
  m.def("norm_rows_backward", &norm_rows_backward);
  m.def("sort_tokens", &sort_tokens);
  m.def("gather_rows", &gather_rows);
  m.def("combine_rows", &combine_rows);
  m.def("combine_rows_backward", &combine_rows_backward);
  m.def("experts_rows", &experts_rows);
  m.def("experts_rows_backward", &experts_rows_backward);
  bind_attention(m);
}
