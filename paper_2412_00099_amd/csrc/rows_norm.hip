// Residual addition and root-mean-square norm of many rows, and its gradient.
//
//   h' = h + y (rounded to h's type), r = 1 / sqrt(mean h'^2 + eps), x = h' r gain
//   8 bits: v = h' gain, q = round(v (127 (1 / max|v|))), scale = max|v| / 127 * r.  The codes do not depend on r, so they are the
//   same however the sum of squares is split over lanes, and both reductions of a row run together.
//   backward, n = h' r: dh = dh' + r (dx gain - n mean(dx gain n)), dgain = sum over the rows of dx n
// Bound by memory: every row is read once into registers and written once.  All sums are in 32 bits.
#include "rows.h"

namespace moe {
namespace {

constexpr int kMaxWaves = 16;

// A row belongs to a wavefront or to a whole workgroup; `part` holds one value per wavefront.
struct RowLanes {
  int lane, wave, waves;  // waves of the row
};
__device__ __forceinline__ float row_sum(float v, const RowLanes &l, float *part) {
  v = wave_sum(v);
  if (l.waves == 1) return v;
  if (l.lane == 0) part[l.wave] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < l.waves; ++w) s += part[w];
  return s;
}
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
  return v;
}

// Lane t of a row's lanes holds elements (j * lanes + t) * VEC ...
template <int H, int Y, int X, int VEC, int NV>
__global__ __launch_bounds__(1024) void norm_rows_kernel(const NormRowsParams p, const int waves) {
  __shared__ float part_ss[kMaxWaves];
  __shared__ uint32_t part_top[kMaxWaves];
  RowLanes l;
  l.lane = threadIdx.x & 63;
  l.waves = waves;
  int64_t row;
  if (waves == 1) {
    l.wave = 0;
    row = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
    if (row >= p.n_rows) return;  // (no barrier in this form)
  } else {
    l.wave = threadIdx.x >> 6;
    row = blockIdx.x;
  }
  const int t = l.wave * 64 + l.lane, step = waves * 64 * VEC, d = p.hidden;
  float h[NV][VEC], y[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = j * step + t * VEC;
    if (at < d) {
      load_row<H>(p.h, row * p.h_stride + at, h[j]);
      if constexpr (Y >= 0) load_row<Y>(p.y, row * p.y_stride + at, y[j]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[j][i] = y[j][i] = 0.f;
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if constexpr (Y >= 0) h[j][i] = as_stored<H>(h[j][i] + y[j][i]);
      ss = __builtin_fmaf(h[j][i], h[j][i], ss);
    }
    const int at = j * step + t * VEC;
    if (at < d && p.h_out) store_row<H>(p.h_out, row * d + at, h[j]);
  }
  // the largest |h gain| of the row by its bits: infinities and NaN come out on top
  uint32_t top = 0;
  if (X == MOE_R_INT8 || p.gain) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = j * step + t * VEC;
      float g[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[i] = 1.f;
      if (p.gain && at < d) load_row<MOE_R_FP32>(p.gain, at, g);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if constexpr (X == MOE_R_INT8) {
          h[j][i] *= g[i];
          top = max(top, __float_as_uint(h[j][i]) & 0x7fffffffu);
        } else {
          y[j][i] = g[i];
        }
      }
    }
  }
  ss = wave_sum(ss);
  if constexpr (X == MOE_R_INT8) top = wave_max_bits(top);
  if (waves > 1) {
    if (l.lane == 0) {
      part_ss[l.wave] = ss;
      part_top[l.wave] = top;
    }
    __syncthreads();
    ss = 0.f;
    for (int w = 0; w < waves; ++w) {
      ss += part_ss[w];
      top = max(top, part_top[w]);
    }
  }
  const float r = 1.0f / sqrtf(ss / (float)d + p.eps);
  if (t == 0 && p.rstd) p.rstd[row] = r;
  if constexpr (X == MOE_R_INT8) {
    // A row of (nearly) zeros has codes and scale 0; one that holds an infinity or NaN has codes 0 and scale NaN.
    const float m = __uint_as_float(top);
    const bool finite = top < 0x7f800000u, some = finite && m >= 1e-30f;
    const float inv = some ? 127.0f * (1.0f / m) : 0.f;
    if (t == 0) p.scale[row] = some ? m / 127.0f * r : finite ? 0.f : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = j * step + t * VEC;
      if (at >= d) continue;
      int8_t q[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) q[i] = some ? (int8_t)(int)rintf(h[j][i] * inv) : (int8_t)0;
      int8_t *o = static_cast<int8_t *>(p.x) + row * d + at;
      if constexpr (VEC == 8)
        *reinterpret_cast<rows_u32x2 *>(o) = __builtin_bit_cast(rows_u32x2, q);
      else
        o[0] = q[0];
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = j * step + t * VEC;
      if (at >= d) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        h[j][i] *= r;
        if (p.gain) h[j][i] *= y[j][i];
      }
      store_row<X>(p.x, row * d + at, h[j]);
    }
  }
}

constexpr int kBackParts = 512;  // workgroups of the backward launch at most: two per compute unit

template <int H, int X, int VEC, int NV>
__global__ __launch_bounds__(1024) void norm_rows_backward_kernel(const NormRowsBackwardParams p, const int waves) {
  __shared__ float part[2][kMaxWaves];
  RowLanes l;
  l.lane = threadIdx.x & 63;
  l.wave = threadIdx.x >> 6;
  l.waves = waves;
  const int t = threadIdx.x, step = waves * 64 * VEC, d = p.hidden;
  float gain[NV][VEC], dgain[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = j * step + t * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      gain[j][i] = 1.f;
      dgain[j][i] = 0.f;
    }
    if (p.gain && at < d) load_row<MOE_R_FP32>(p.gain, at, gain[j]);
  }
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.n_rows; row += gridDim.x, turn ^= 1) {
    float n[NV][VEC], g[NV][VEC];
    const float r = p.rstd[row];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = j * step + t * VEC;
      if (at < d) {
        load_row<H>(p.h, row * d + at, n[j]);
        load_row<X>(p.dx, row * d + at, g[j]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) n[j][i] = g[j][i] = 0.f;
      }
    }
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        n[j][i] *= r;
        dgain[j][i] = __builtin_fmaf(g[j][i], n[j][i], dgain[j][i]);
        g[j][i] *= gain[j][i];
        dot = __builtin_fmaf(g[j][i], n[j][i], dot);
      }
    // (two sets of words in turn: the next row's first is written only behind this row's barrier)
    dot = row_sum(dot, l, part[turn]) / (float)d;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = j * step + t * VEC;
      if (at >= d) continue;
      float up[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) up[i] = 0.f;
      if (p.dh) load_row<H>(p.dh, row * d + at, up);
#pragma unroll
      for (int i = 0; i < VEC; ++i) up[i] = __builtin_fmaf(r, g[j][i] - n[j][i] * dot, up[i]);
      store_row<H>(p.dh_out, row * d + at, up);
    }
  }
  if (p.dgain) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = j * step + t * VEC;
      if (at < d) store_row<MOE_R_FP32>(p.partial, (int64_t)blockIdx.x * d + at, dgain[j]);
    }
  }
}

// dgain: 64 columns a workgroup, its wavefronts share the rows of `partial`; always in the same order
__global__ __launch_bounds__(1024) void sum_parts_kernel(const float *partial, int parts, int d, float *out) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float v = 0.f;
  if (c < d)
    for (int i = wave; i < parts; i += 16) v += partial[(int64_t)i * d + c];
  s[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && c < d) {
    for (int w = 1; w < 16; ++w) v += s[w][lane];
    out[c] = v;
  }
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <int N>
struct Const {
  static constexpr int value = N;
};

}  // namespace

hipError_t launch_norm_rows(const NormRowsParams &p, int n_cus, hipStream_t s) {
  const int d = p.hidden;
  // 16-byte accesses where every row allows them (8 bytes for the 8-bit codes)
  const bool wide = d % 8 == 0 && p.h_stride % 8 == 0 && aligned16(p.h) && (!p.y || (p.y_stride % 8 == 0 && aligned16(p.y))) &&
                    (!p.gain || aligned16(p.gain)) && (!p.h_out || aligned16(p.h_out)) &&
                    reinterpret_cast<uintptr_t>(p.x) % (p.x_fmt == MOE_R_INT8 ? 8 : 16) == 0;
  const int vec = wide ? 8 : 1, most = wide ? 4 : 8;
  int waves = 1;
  while ((int64_t)waves * 64 * vec * most < d) waves *= 2;
  // few rows: a row over more wavefronts, one step each
  while (p.n_rows < 4 * n_cus && waves < kMaxWaves && waves * 64 * vec < d) waves *= 2;
  const int nv = (d + waves * 64 * vec - 1) / (waves * 64 * vec);
  const int rows_per_wg = waves == 1 ? 4 : 1;
  const dim3 grid((uint32_t)((p.n_rows + rows_per_wg - 1) / rows_per_wg)), block(waves == 1 ? 256 : waves * 64);
  const auto go = [&](auto H, auto Y, auto X) {
    const auto with = [&](auto VEC, auto NV) {
      hipLaunchKernelGGL((norm_rows_kernel<decltype(H)::value, decltype(Y)::value, decltype(X)::value, decltype(VEC)::value, decltype(NV)::value>),
                         grid, block, 0, s, p, waves);
    };
    if (wide) {
      if (nv == 1) with(Const<8>{}, Const<1>{});
      else if (nv == 2) with(Const<8>{}, Const<2>{});
      else with(Const<8>{}, Const<4>{});
    } else {
      if (nv <= 2) with(Const<1>{}, Const<2>{});
      else with(Const<1>{}, Const<8>{});
    }
  };
  const auto x = [&](auto H, auto Y) {
    if (p.x_fmt == MOE_R_FP32) go(H, Y, Const<MOE_R_FP32>{});
    else if (p.x_fmt == MOE_R_BF16) go(H, Y, Const<MOE_R_BF16>{});
    else go(H, Y, Const<MOE_R_INT8>{});
  };
  const auto y = [&](auto H) {
    if (!p.y) x(H, Const<-1>{});
    else if (p.y_fmt == MOE_R_FP32) x(H, Const<MOE_R_FP32>{});
    else x(H, Const<MOE_R_BF16>{});
  };
  if (p.h_fmt == MOE_R_FP32) y(Const<MOE_R_FP32>{});
  else y(Const<MOE_R_BF16>{});
  return hipGetLastError();
}

int norm_rows_backward_parts(int n_rows, int hidden) { return n_rows < kBackParts ? n_rows : kBackParts; }

hipError_t launch_norm_rows_backward(const NormRowsBackwardParams &p, hipStream_t s) {
  const int d = p.hidden;
  const bool wide = d % 8 == 0 && aligned16(p.h) && aligned16(p.dx) && (!p.dh || aligned16(p.dh)) && aligned16(p.dh_out) &&
                    (!p.gain || aligned16(p.gain)) && (!p.dgain || aligned16(p.partial));
  const int vec = wide ? 8 : 1, most = wide ? 2 : 8;
  int waves = 1;
  while ((int64_t)waves * 64 * vec * most < d) waves *= 2;
  const int nv = (d + waves * 64 * vec - 1) / (waves * 64 * vec), parts = norm_rows_backward_parts(p.n_rows, d);
  const auto go = [&](auto H, auto X) {
    const auto with = [&](auto VEC, auto NV) {
      if (parts == 0) return;  // (no rows: dgain is zero)
      hipLaunchKernelGGL((norm_rows_backward_kernel<decltype(H)::value, decltype(X)::value, decltype(VEC)::value, decltype(NV)::value>),
                         dim3(parts), dim3(waves * 64), 0, s, p, waves);
    };
    if (wide) {
      if (nv == 1) with(Const<8>{}, Const<1>{});
      else with(Const<8>{}, Const<2>{});
    } else {
      if (nv <= 2) with(Const<1>{}, Const<2>{});
      else with(Const<1>{}, Const<8>{});
    }
  };
  const auto x = [&](auto H) {
    if (p.x_fmt == MOE_R_FP32) go(H, Const<MOE_R_FP32>{});
    else go(H, Const<MOE_R_BF16>{});
  };
  if (p.h_fmt == MOE_R_FP32) x(Const<MOE_R_FP32>{});
  else x(Const<MOE_R_BF16>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.dgain) return e;
  hipLaunchKernelGGL(sum_parts_kernel, dim3((d + 63) / 64), dim3(1024), 0, s, p.partial, parts, d, p.dgain);
  return hipGetLastError();
}

}  // namespace moe
