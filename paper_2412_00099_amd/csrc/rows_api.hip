// C entry points of the operators on many rows: argument checks and launches, nothing else.
#include <cmath>

#include "rows.h"

using namespace moe;

namespace {

constexpr int64_t kMaxRows = MOE_ROWS_LIMIT;

bool float_rows(int32_t f) { return f == MOE_R_FP32 || f == MOE_R_BF16; }
bool off(const void *p, int by) { return reinterpret_cast<uintptr_t>(p) % by != 0; }

// compute units of the current device; looked up once per device
hipError_t compute_units(int *cus) {
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  return static_scratch_setup(dev, nullptr, cus);
}

int check_order(int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t hidden) {
  if (n_tokens < 0 || top_k < 1 || top_k > MOE_MAX_TOPK || (int64_t)n_tokens * top_k >= kMaxRows)
    return fail(MOE_EINVAL, "bad n_tokens=%d or top_k=%d", n_tokens, top_k);
  if (n_experts < 1 || n_experts > kRowMaxExperts) return fail(MOE_EINVAL, "n_experts=%d is not in 1..%d", n_experts, kRowMaxExperts);
  if (hidden < 1 || hidden > kRowMaxHidden) return fail(MOE_EINVAL, "hidden=%d is not in 1..%d", hidden, kRowMaxHidden);
  return MOE_OK;
}

int check_experts(int32_t weight_fmt, int32_t hidden, int32_t inter, int32_t n_experts, const void *blobs, int64_t blob_stride,
                  const void *offsets, int32_t n_rows) {
  if (weight_fmt != MOE_W_BF16 && weight_fmt != MOE_W_INT8_PC)
    return fail(MOE_EINVAL, "experts on rows take bf16 or int8 blobs, not weight format %d", weight_fmt);
  const size_t bytes = moe_blob_bytes(weight_fmt, hidden, inter);
  if (bytes == 0 || hidden > kRowMaxHidden)
    return fail(MOE_EINVAL, "unsupported shape hidden=%d inter=%d for weight format %d", hidden, inter, weight_fmt);
  if (bytes >= 0xf0000000u) return fail(MOE_EINVAL, "a blob of %zu bytes is too large", bytes);
  if (n_experts < 1 || n_experts > kRowMaxExperts) return fail(MOE_EINVAL, "n_experts=%d is not in 1..%d", n_experts, kRowMaxExperts);
  if (n_rows < 0 || n_rows >= kMaxRows) return fail(MOE_EINVAL, "bad n_rows=%d", n_rows);
  if (!blobs || !offsets) return fail(MOE_EINVAL, "blobs_dev or offsets_dev is NULL");
  if (blob_stride < (int64_t)bytes || blob_stride % 16 != 0 || off(blobs, 16))
    return fail(MOE_EINVAL, "blobs need a stride of at least %zu bytes and 16-byte alignment", bytes);
  return MOE_OK;
}

}  // namespace

extern "C" {

int moe_norm_rows(const void *h, int32_t h_fmt, int64_t h_stride, const void *y, int32_t y_fmt, int64_t y_stride, const float *gain,
                  float eps, int32_t n_rows, int32_t hidden, void *h_out, void *x, int32_t x_fmt, float *scale, float *rstd, void *stream) {
  if (!float_rows(h_fmt) || (y && !float_rows(y_fmt)) || row_elem(x_fmt) == 0)
    return fail(MOE_EINVAL, "bad h_fmt=%d, y_fmt=%d or x_fmt=%d", h_fmt, y_fmt, x_fmt);
  if (hidden < 1 || hidden > kRowMaxHidden) return fail(MOE_EINVAL, "hidden=%d is not in 1..%d", hidden, kRowMaxHidden);
  if (n_rows < 0 || n_rows >= kMaxRows) return fail(MOE_EINVAL, "bad n_rows=%d", n_rows);
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MOE_EINVAL, "eps must be finite and not negative");
  if (h_stride < hidden || (y && y_stride < hidden)) return fail(MOE_EINVAL, "rows overlap: a stride is smaller than hidden=%d", hidden);
  if (n_rows == 0) return MOE_OK;
  if (!h || !x) return fail(MOE_EINVAL, "h_dev or x_dev is NULL");
  if (y && !h_out) return fail(MOE_EINVAL, "with y_dev h_out_dev is needed");
  if (h_out == h && h_stride != hidden) return fail(MOE_EINVAL, "h_out_dev can be h_dev for dense rows only");
  if ((x_fmt == MOE_R_INT8) != (scale != nullptr)) return fail(MOE_EINVAL, "scale_dev goes with 8-bit codes");
  if (off(h, row_elem(h_fmt)) || (y && off(y, row_elem(y_fmt))) || off(h_out, row_elem(h_fmt)) || off(x, row_elem(x_fmt)) || off(gain, 4) ||
      off(scale, 4) || off(rstd, 4))
    return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  NormRowsParams p{h, y, gain, h_out, x, scale, rstd, h_stride, y_stride, n_rows, hidden, h_fmt, y_fmt, x_fmt, eps};
  int cus = 0;
  HIP_TRY(compute_units(&cus));
  HIP_TRY(launch_norm_rows(p, cus, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

size_t moe_norm_rows_backward_bytes(int32_t n_rows, int32_t hidden) {
  if (n_rows <= 0 || hidden < 1 || hidden > kRowMaxHidden) return 0;
  return (size_t)norm_rows_backward_parts(n_rows, hidden) * hidden * sizeof(float);
}

int moe_norm_rows_backward(const void *h_out, int32_t h_fmt, const float *gain, const float *rstd, const void *dx, int32_t x_fmt,
                           const void *dh_in, int32_t n_rows, int32_t hidden, void *dh, float *dgain, void *workspace,
                           size_t workspace_bytes, void *stream) {
  if (!float_rows(h_fmt) || !float_rows(x_fmt)) return fail(MOE_EINVAL, "bad h_fmt=%d or x_fmt=%d", h_fmt, x_fmt);
  if (hidden < 1 || hidden > kRowMaxHidden) return fail(MOE_EINVAL, "hidden=%d is not in 1..%d", hidden, kRowMaxHidden);
  if (n_rows < 0 || n_rows >= kMaxRows) return fail(MOE_EINVAL, "bad n_rows=%d", n_rows);
  if (n_rows > 0 && (!h_out || !rstd || !dx || !dh)) return fail(MOE_EINVAL, "h_out_dev, rstd_dev, dx_dev or dh_dev is NULL");
  if (off(h_out, row_elem(h_fmt)) || off(dx, row_elem(x_fmt)) || off(dh_in, row_elem(h_fmt)) || off(dh, row_elem(h_fmt)) || off(gain, 4) ||
      off(rstd, 4) || off(dgain, 4))
    return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  if (dgain && n_rows > 0 && (!workspace || off(workspace, 16) || workspace_bytes < moe_norm_rows_backward_bytes(n_rows, hidden)))
    return fail(MOE_EINVAL, "dgain_dev needs a workspace of %zu bytes, 16-byte aligned", moe_norm_rows_backward_bytes(n_rows, hidden));
  NormRowsBackwardParams p{h_out, gain, rstd, dx, dh_in, dh, dgain, static_cast<float *>(workspace), n_rows, hidden, h_fmt, x_fmt};
  HIP_TRY(launch_norm_rows_backward(p, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

size_t moe_sort_tokens_bytes(int32_t n_tokens, int32_t top_k, int32_t n_experts) {
  if (n_tokens <= 0 || top_k < 1 || n_experts < 1) return 0;
  return sort_tokens_bytes((int64_t)n_tokens * top_k, n_experts);
}

int moe_sort_tokens(const int32_t *ids, int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t *offsets, int32_t *row_of,
                    int32_t *entry_of, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int bad = check_order(n_tokens, top_k, n_experts, 1)) return bad;
  if (!offsets || (n_tokens > 0 && (!ids || !row_of || !entry_of))) return fail(MOE_EINVAL, "a pointer is NULL");
  if (off(ids, 4) || off(offsets, 4) || off(row_of, 4) || off(entry_of, 4) || off(workspace, 4))
    return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  const size_t need = moe_sort_tokens_bytes(n_tokens, top_k, n_experts);
  if (need > 0 && (!workspace || workspace_bytes < need)) return fail(MOE_EINVAL, "a workspace of %zu bytes is needed", need);
  HIP_TRY(launch_sort_tokens(ids, (int64_t)n_tokens * top_k, n_experts, offsets, row_of, entry_of, workspace, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

int moe_gather_rows(const void *x, int32_t fmt, int64_t x_stride, const float *scale, const int32_t *row_of, const int32_t *offsets,
                    int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t hidden, void *xs, float *xs_scale, void *stream) {
  if (const int bad = check_order(n_tokens, top_k, n_experts, hidden)) return bad;
  if (row_elem(fmt) == 0) return fail(MOE_EINVAL, "bad fmt=%d", fmt);
  if (x_stride < hidden) return fail(MOE_EINVAL, "rows overlap: x_stride is smaller than hidden=%d", hidden);
  if (n_tokens == 0) return MOE_OK;
  if (!x || !row_of || !offsets || !xs) return fail(MOE_EINVAL, "a pointer is NULL");
  if ((scale != nullptr) != (xs_scale != nullptr)) return fail(MOE_EINVAL, "scale_dev and xs_scale_dev go together");
  if (off(x, row_elem(fmt)) || off(xs, row_elem(fmt)) || off(scale, 4) || off(xs_scale, 4) || off(row_of, 4) || off(offsets, 4))
    return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  const OrderParams o{row_of, offsets, n_tokens, top_k, n_experts, hidden};
  HIP_TRY(launch_gather_rows(o, x, fmt, x_stride, scale, xs, xs_scale, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

int moe_combine_rows(const void *ys, int32_t ys_fmt, const int32_t *row_of, const float *weight, const void *base, int32_t n_tokens,
                     int32_t top_k, int32_t hidden, void *y, int32_t y_fmt, void *stream) {
  if (const int bad = check_order(n_tokens, top_k, 1, hidden)) return bad;
  if (!float_rows(ys_fmt) || !float_rows(y_fmt)) return fail(MOE_EINVAL, "bad ys_fmt=%d or y_fmt=%d", ys_fmt, y_fmt);
  if (n_tokens == 0) return MOE_OK;
  if (!ys || !row_of || !y) return fail(MOE_EINVAL, "a pointer is NULL");
  if (off(ys, row_elem(ys_fmt)) || off(y, row_elem(y_fmt)) || off(base, row_elem(y_fmt)) || off(weight, 4) || off(row_of, 4))
    return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  const OrderParams o{row_of, nullptr, n_tokens, top_k, 0, hidden};
  HIP_TRY(launch_combine_rows(o, ys, ys_fmt, weight, base, y, y_fmt, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

int moe_combine_rows_backward(const void *dy, int32_t dy_fmt, const void *ys, int32_t ys_fmt, const int32_t *row_of, const int32_t *offsets,
                              const float *weight, int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t hidden, void *dys,
                              float *dweight, void *stream) {
  if (const int bad = check_order(n_tokens, top_k, n_experts, hidden)) return bad;
  if (!float_rows(dy_fmt) || !float_rows(ys_fmt)) return fail(MOE_EINVAL, "bad dy_fmt=%d or ys_fmt=%d", dy_fmt, ys_fmt);
  if (n_tokens == 0) return MOE_OK;
  if (!dy || !row_of || !offsets || !dys) return fail(MOE_EINVAL, "a pointer is NULL");
  if (dweight && !ys) return fail(MOE_EINVAL, "dweight_dev needs ys_dev");
  if (off(dy, row_elem(dy_fmt)) || off(ys, row_elem(ys_fmt)) || off(dys, row_elem(ys_fmt)) || off(weight, 4) || off(dweight, 4) ||
      off(row_of, 4) || off(offsets, 4))
    return fail(MOE_EINVAL, "a pointer is not aligned to its type");
  const OrderParams o{row_of, offsets, n_tokens, top_k, n_experts, hidden};
  HIP_TRY(launch_combine_rows_backward(o, dy, dy_fmt, ys, ys_fmt, weight, dys, dweight, static_cast<hipStream_t>(stream)));
  return MOE_OK;
}

int moe_experts_rows(int32_t weight_fmt, int32_t hidden, int32_t inter, int32_t n_experts, const void *blobs, int64_t blob_stride,
                     const void *xs, const float *scale, const int32_t *offsets, int32_t n_rows, void *h, float *gu, void *ys, void *stream) {
  if (const int bad = check_experts(weight_fmt, hidden, inter, n_experts, blobs, blob_stride, offsets, n_rows)) return bad;
  if (n_rows == 0) return MOE_OK;
  if (!xs || !h || !ys) return fail(MOE_EINVAL, "xs_dev, h_dev or ys_dev is NULL");
  if ((weight_fmt == MOE_W_INT8_PC) != (scale != nullptr)) return fail(MOE_EINVAL, "scale_dev goes with int8 blobs");
  if (off(xs, 16) || off(h, 16) || off(gu, 16) || off(ys, 16) || off(scale, 4) || off(offsets, 4))
    return fail(MOE_EINVAL, "xs_dev, h_dev, gu_dev and ys_dev have to be 16-byte aligned");
  const ExpertRowsParams p{static_cast<const uint8_t *>(blobs), blob_stride, offsets, n_experts, n_rows, hidden, inter};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  int cus = 0;
  HIP_TRY(compute_units(&cus));
  HIP_TRY(launch_experts_up(p, weight_fmt, xs, scale, static_cast<uint16_t *>(h), gu, cus, s));
  HIP_TRY(launch_experts_down(p, weight_fmt, static_cast<const uint16_t *>(h), static_cast<uint16_t *>(ys), cus, s));
  return MOE_OK;
}

int moe_experts_rows_backward(int32_t weight_fmt, int32_t hidden, int32_t inter, int32_t n_experts, const void *blobs, int64_t blob_stride,
                              const void *xs, const int32_t *offsets, int32_t n_rows, const void *h, const float *gu, const void *dys, void *dgu,
                              void *dxs, void *dblobs, void *stream) {
  if (weight_fmt != MOE_W_BF16) return fail(MOE_EINVAL, "gradients are of bf16 blobs, not of weight format %d", weight_fmt);
  if (const int bad = check_experts(weight_fmt, hidden, inter, n_experts, blobs, blob_stride, offsets, n_rows)) return bad;
  if (n_rows > 0 && (!xs || !h || !gu || !dys || !dgu)) return fail(MOE_EINVAL, "xs_dev, h_dev, gu_dev, dys_dev or dgu_dev is NULL");
  if (off(xs, 16) || off(h, 16) || off(gu, 16) || off(dys, 16) || off(dgu, 16) || off(dxs, 16) || off(dblobs, 16) || off(offsets, 4))
    return fail(MOE_EINVAL, "a pointer is not 16-byte aligned");
  const ExpertRowsParams p{static_cast<const uint8_t *>(blobs), blob_stride, offsets, n_experts, n_rows, hidden, inter};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const uint16_t *x16 = static_cast<const uint16_t *>(xs), *d16 = static_cast<const uint16_t *>(dys), *h16 = static_cast<const uint16_t *>(h);
  uint16_t *dgu16 = static_cast<uint16_t *>(dgu);
  int cus = 0;
  HIP_TRY(compute_units(&cus));
  if (n_rows > 0 && (dxs || dblobs)) HIP_TRY(launch_experts_dgu(p, d16, gu, dgu16, cus, s));
  if (n_rows > 0 && dxs) HIP_TRY(launch_experts_dx(p, dgu16, static_cast<uint16_t *>(dxs), cus, s));
  if (dblobs) HIP_TRY(launch_experts_dw(p, x16, d16, h16, dgu16, static_cast<uint8_t *>(dblobs), cus, s));
  return MOE_OK;
}

}  // extern "C"
