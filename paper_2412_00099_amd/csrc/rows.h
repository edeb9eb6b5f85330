// Operators on many rows at once (norm, order of the tokens by expert, resident experts): what the translation units share.
#pragma once

#include "common.h"
#include "row_grid.h"

namespace moe {

constexpr int kRowMaxExperts = MOE_ROWS_MAX_EXPERTS;  // of a sort or of a launch over sorted rows
constexpr int kRowMaxHidden = MOE_ROWS_MAX_HIDDEN;    // width of a row

// bytes of one element of a row (moe_row_fmt), 0: unknown
__host__ __device__ constexpr int row_elem(int fmt) {
  return fmt == MOE_R_FP32 ? 4 : fmt == MOE_R_BF16 ? 2 : fmt == MOE_R_INT8 ? 1 : 0;
}

// ---- rows_norm.hip ----
struct NormRowsParams {
  const void *h, *y;  // y may be NULL
  const float *gain;  // NULL: ones
  void *h_out, *x;    // h_out may be NULL (then y is too) or h
  float *scale;       // per row, x_fmt int8 only
  float *rstd;        // per row, may be NULL
  int64_t h_stride, y_stride;  // elements
  int32_t n_rows, hidden, h_fmt, y_fmt, x_fmt;
  float eps;
};
hipError_t launch_norm_rows(const NormRowsParams &p, int n_cus, hipStream_t s);
struct NormRowsBackwardParams {
  const void *h;       // the stored h_out of the forward, dense
  const float *gain, *rstd;
  const void *dx, *dh;  // dh (h_fmt) may be NULL
  void *dh_out;         // h_fmt
  float *dgain;         // may be NULL
  float *partial;       // [norm_rows_backward_parts][hidden], with dgain
  int32_t n_rows, hidden, h_fmt, x_fmt;
};
// rows of `partial`: workgroups of the launch
int norm_rows_backward_parts(int n_rows, int hidden);
hipError_t launch_norm_rows_backward(const NormRowsBackwardParams &p, hipStream_t s);

// ---- rows_order.hip ----
size_t sort_tokens_bytes(int64_t n, int n_experts);
hipError_t launch_sort_tokens(const int32_t *ids, int64_t n, int n_experts, int32_t *offsets, int32_t *row_of, int32_t *entry_of,
                              void *workspace, hipStream_t s);
struct OrderParams {
  const int32_t *row_of;   // [n_tokens][top_k]
  const int32_t *offsets;  // [n_experts + 1]
  int32_t n_tokens, top_k, n_experts, hidden;
};
hipError_t launch_gather_rows(const OrderParams &o, const void *x, int fmt, int64_t x_stride, const float *scale, void *xs, float *xs_scale,
                              hipStream_t s);
hipError_t launch_combine_rows(const OrderParams &o, const void *ys, int ys_fmt, const float *weight, const void *base, void *y, int y_fmt,
                               hipStream_t s);
hipError_t launch_combine_rows_backward(const OrderParams &o, const void *dy, int dy_fmt, const void *ys, int ys_fmt, const float *weight,
                                        void *dys, float *dweight, hipStream_t s);

// ---- rows_experts.hip ----
struct ExpertRowsParams {
  const uint8_t *blobs;
  int64_t blob_stride;     // bytes
  const int32_t *offsets;  // [n_experts + 1]
  int32_t n_experts, n_rows, hidden, inter;
};
// row length of the arrays over the records: a whole number of the kernels' tiles
__host__ __device__ constexpr int expert_rows_pitch(int inter) { return (inter + 63) / 64 * 64; }
// h [n_rows][pitch] = silu(x Wg^T) * (x Wu^T); gu (may be NULL) fp32 [n_rows][2][pitch]: the two products
hipError_t launch_experts_up(const ExpertRowsParams &p, int weight_fmt, const void *xs, const float *scale, uint16_t *h, float *gu, int n_cus,
                             hipStream_t s);
hipError_t launch_experts_down(const ExpertRowsParams &p, int weight_fmt, const uint16_t *h, uint16_t *ys, int n_cus, hipStream_t s);
// dgu [n_rows][2][pitch]: the gradients of the two products
hipError_t launch_experts_dgu(const ExpertRowsParams &p, const uint16_t *dys, const float *gu, uint16_t *dgu, int n_cus, hipStream_t s);
hipError_t launch_experts_dx(const ExpertRowsParams &p, const uint16_t *dgu, uint16_t *dxs, int n_cus, hipStream_t s);
hipError_t launch_experts_dw(const ExpertRowsParams &p, const uint16_t *xs, const uint16_t *dys, const uint16_t *h, const uint16_t *dgu,
                             uint8_t *dblobs, int n_cus, hipStream_t s);

// ---- device helpers ----
#if defined(__HIPCC__)
// for lambdas that are called in several places: as calls they would keep their captures in memory
#define MOE_ROWS_INLINE __attribute__((always_inline))
// the workgroup's place in a grid of row_grid
__device__ __forceinline__ int64_t row_group() { return blockIdx.y * kRowGridX + blockIdx.x; }
typedef uint32_t rows_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t rows_u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  b2 v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}

// (16 bytes may begin at any element of their type: the same instructions)
typedef uint32_t rows_u32x4_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t rows_u32x4_bf16 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t rows_u32x4_codes __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t rows_u32x2_codes __attribute__((ext_vector_type(2), aligned(1)));

// ONCE: read by nobody else in the launch, so it need not push anything out of the caches
template <bool ONCE>
__device__ __forceinline__ rows_u32x4 load16(const float *p) {
  const rows_u32x4_f32 *q = reinterpret_cast<const rows_u32x4_f32 *>(p);
  if constexpr (ONCE) return __builtin_nontemporal_load(q);
  else return *q;
}
template <bool ONCE>
__device__ __forceinline__ rows_u32x4 load16(const uint16_t *p) {
  const rows_u32x4_bf16 *q = reinterpret_cast<const rows_u32x4_bf16 *>(p);
  if constexpr (ONCE) return __builtin_nontemporal_load(q);
  else return *q;
}
template <bool ONCE, typename T>
__device__ __forceinline__ T load_one(const T *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
// VEC columns from c on, of a row of d >= VEC: the last unit begins where it has VEC, and its first `skip` columns belong to the
// unit before it.
struct RowUnit {
  int at, skip;
};
template <int VEC>
__device__ __forceinline__ RowUnit row_unit(int c, int d) {
  RowUnit u;
  u.at = min(c, d - VEC);
  u.skip = c - u.at;
  return u;
}
// VEC elements of type FMT (VEC 8: 16-byte accesses; 1: one element).
template <int FMT, int VEC, bool ONCE = false>
__device__ __forceinline__ void load_row(const void *p, int64_t at, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    if constexpr (FMT == MOE_R_FP32)
      v[0] = load_one<ONCE>(static_cast<const float *>(p) + at);
    else
      v[0] = __uint_as_float((uint32_t)load_one<ONCE>(static_cast<const uint16_t *>(p) + at) << 16);
  } else if constexpr (FMT == MOE_R_FP32) {
    const rows_u32x4 a = load16<ONCE>(static_cast<const float *>(p) + at), b = load16<ONCE>(static_cast<const float *>(p) + at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __uint_as_float(a[i]);
      v[4 + i] = __uint_as_float(b[i]);
    }
  } else {
    const rows_u32x4 a = load16<ONCE>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_lo(a[i]);
      v[2 * i + 1] = bf16_hi(a[i]);
    }
  }
}
template <int FMT, int VEC>
__device__ __forceinline__ void store_row(void *p, int64_t at, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    if constexpr (FMT == MOE_R_FP32)
      static_cast<float *>(p)[at] = v[0];
    else
      static_cast<uint16_t *>(p)[at] = (uint16_t)pack_bf16(v[0], 0.f);
  } else if constexpr (FMT == MOE_R_FP32) {
    rows_u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __float_as_uint(v[i]);
      b[i] = __float_as_uint(v[4 + i]);
    }
    rows_u32x4_f32 *q = reinterpret_cast<rows_u32x4_f32 *>(static_cast<float *>(p) + at);
    q[0] = a;
    q[1] = b;
  } else {
    rows_u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<rows_u32x4_bf16 *>(static_cast<uint16_t *>(p) + at) = a;
  }
}
// those of the unit that belong to it; at: of the row's first element
template <int FMT, int VEC>
__device__ __forceinline__ void store_unit(void *p, int64_t at, const RowUnit &u, const float (&v)[VEC]) {
  if (u.skip == 0) {
    store_row<FMT>(p, at + u.at, v);
  } else {
#pragma unroll
    for (int i = 1; i < VEC; ++i) {
      const float one[1] = {v[i]};
      if (i >= u.skip) store_row<FMT>(p, at + u.at + i, one);
    }
  }
}
// v as the type keeps it
template <int FMT>
__device__ __forceinline__ float as_stored(float v) {
  if constexpr (FMT == MOE_R_FP32) return v;
  return bf16_lo(pack_bf16(v, 0.f));
}
#endif

}  // namespace moe
