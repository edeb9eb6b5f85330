// Residual addition and root-mean-square norm of many rows, and its gradient.
//
//   h' = h + y (rounded to h's type), r = 1 / sqrt(mean h'^2 + eps), x = h' r gain
//   8 bits: v = h' gain, q = round(v (127 (1 / max|v|))), scale = max|v| / 127 * r.  The codes do not depend on r, so they are the
//   same however the sum of squares is split over lanes, and both reductions of a row run together.
//   backward, n = h' r: dh = dh' + r (dx gain - n mean(dx gain n)), dgain = sum over the rows of dx n
// Bound by memory: every row is read once into registers and written once.  All sums are in 32 bits.
// Measured: 16384 rows of 4096, fp32 + bf16 -> fp32 and 8 bits, 738 MB in 149 us (5.0 TB/s); 4096 rows of 2048, fp32 + bf16 -> fp32
// and bf16, 101 MB in 20 us (5.0 TB/s); its gradient, with the gain's, 23 + 5 us; one row 3.0 us.
#include <algorithm>

#include "rows.h"

namespace moe {
namespace {

constexpr int kMaxWaves = 16;

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
  // a row belongs to a wavefront or to the whole workgroup
  const int lane = threadIdx.x & 63, wave = waves == 1 ? 0 : threadIdx.x >> 6;
  int64_t row = row_group();
  if (waves == 1) row = row * (blockDim.x >> 6) + (threadIdx.x >> 6);
  if (row >= p.n_rows) return;  // (ahead of the barrier only with all of the row's wavefronts)
  const int t = wave * 64 + lane, step = waves * 64 * VEC, d = p.hidden;
  float h[NV][VEC], y[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = j * step + t * VEC;
    if (c < d) {
      const RowUnit u = row_unit<VEC>(c, d);
      load_row<H>(p.h, row * p.h_stride + u.at, h[j]);
      if constexpr (Y >= 0) load_row<Y>(p.y, row * p.y_stride + u.at, y[j]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[j][i] = y[j][i] = 0.f;
    }
  }
  // (what belongs to the unit before is no part of the sums, nor is it written: it may be the result already)
  if (VEC > 1 && d % VEC) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = j * step + t * VEC, skip = c < d ? c - min(c, d - VEC) : 0;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        h[j][i] = i < skip ? 0.f : h[j][i];
        if constexpr (Y >= 0) y[j][i] = i < skip ? 0.f : y[j][i];
      }
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
    const int c = j * step + t * VEC;
    if (c < d && p.h_out) store_unit<H>(p.h_out, row * d, row_unit<VEC>(c, d), h[j]);
  }
  // the largest |h gain| of the row by its bits: infinities and NaN come out on top
  uint32_t top = 0;
  if (X == MOE_R_INT8 || p.gain) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = j * step + t * VEC;
      float g[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[i] = 1.f;
      if (p.gain && c < d) load_row<MOE_R_FP32>(p.gain, row_unit<VEC>(c, d).at, g);
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
    if (lane == 0) {
      part_ss[wave] = ss;
      part_top[wave] = top;
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
      const int c = j * step + t * VEC;
      if (c >= d) continue;
      const RowUnit u = row_unit<VEC>(c, d);
      int8_t q[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) q[i] = some ? (int8_t)(int)rintf(h[j][i] * inv) : (int8_t)0;
      int8_t *o = static_cast<int8_t *>(p.x) + row * d + u.at;
      if constexpr (VEC == 8) {
        if (u.skip == 0) {
          *reinterpret_cast<rows_u32x2_codes *>(o) = __builtin_bit_cast(rows_u32x2, q);
        } else {
#pragma unroll
          for (int i = 1; i < VEC; ++i)
            if (i >= u.skip) o[i] = q[i];
        }
      } else {
        o[0] = q[0];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = j * step + t * VEC;
      if (c >= d) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        h[j][i] *= r;
        if (p.gain) h[j][i] *= y[j][i];
      }
      store_unit<X>(p.x, row * d, row_unit<VEC>(c, d), h[j]);
    }
  }
}

constexpr int kBackParts = 512;  // workgroups of the backward launch at most: two per compute unit
constexpr int kBackWaves = 8;    // of a workgroup; a row has some of them, the others take other rows

// (with the rows of the workgroup one after the other on all its wavefronts a compute unit had 4 of them, too few for the memory:
// 4096 x 2048, h fp32, x bf16 took 31 us)
template <int H, int X, int VEC, int NV>
__global__ __launch_bounds__(kBackWaves * 64) void norm_rows_backward_kernel(const NormRowsBackwardParams p, const int waves) {
  __shared__ float part[2][kBackWaves];
  extern __shared__ float sums[];  // [groups - 1][hidden]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = wave / waves, groups = kBackWaves / waves;
  const int t = threadIdx.x - group * waves * 64, step = waves * 64 * VEC, d = p.hidden;
  float gain[NV][VEC], dgain[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = j * step + t * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      gain[j][i] = 1.f;
      dgain[j][i] = 0.f;
    }
    if (p.gain && c < d) load_row<MOE_R_FP32>(p.gain, row_unit<VEC>(c, d).at, gain[j]);
  }
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * groups; row0 < p.n_rows; row0 += (int64_t)gridDim.x * groups, turn ^= 1) {
    const int64_t row = row0 + group;
    const bool there = row < p.n_rows;  // (a group without a row goes along for the barrier)
    float n[NV][VEC], g[NV][VEC], up[NV][VEC];
    const float r = there ? p.rstd[row] : 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = j * step + t * VEC;
      if (there && c < d) {
        const RowUnit u = row_unit<VEC>(c, d);
        load_row<H>(p.h, row * d + u.at, n[j]);
        load_row<X>(p.dx, row * d + u.at, g[j]);
        if (p.dh) load_row<H>(p.dh, row * d + u.at, up[j]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) n[j][i] = g[j][i] = 0.f;
      }
    }
    // (what belongs to the unit before is no part of the sums)
    if (VEC > 1 && d % VEC) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = j * step + t * VEC, skip = c < d ? c - min(c, d - VEC) : 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          n[j][i] = i < skip ? 0.f : n[j][i];
          g[j][i] = i < skip ? 0.f : g[j][i];
        }
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
    dot = wave_sum(dot);
    if (waves > 1) {
      // (two sets of words in turn: the next row's first is written only behind this row's barrier)
      if (lane == 0) part[turn][wave] = dot;
      __syncthreads();
      dot = 0.f;
      for (int w = 0; w < waves; ++w) dot += part[turn][group * waves + w];
    }
    dot /= (float)d;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = j * step + t * VEC;
      if (!there || c >= d) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) up[j][i] = __builtin_fmaf(r, g[j][i] - n[j][i] * dot, p.dh ? up[j][i] : 0.f);
      store_unit<H>(p.dh_out, row * d, row_unit<VEC>(c, d), up[j]);
    }
  }
  if (!p.dgain) return;
  // the groups' sums, always in the same order
  if (group > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = j * step + t * VEC;
      if (c >= d) continue;
      const RowUnit u = row_unit<VEC>(c, d);
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (i >= u.skip) sums[(group - 1) * d + u.at + i] = dgain[j][i];
    }
  }
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = j * step + t * VEC;
    if (c >= d) continue;
    const RowUnit u = row_unit<VEC>(c, d);
    for (int k = 0; k < groups - 1; ++k)
#pragma unroll
      for (int i = 0; i < VEC; ++i) dgain[j][i] += sums[k * d + u.at + i];
    store_unit<MOE_R_FP32>(p.partial, (int64_t)blockIdx.x * d, u, dgain[j]);
  }
}

// dgain: 32 columns a workgroup, 32 threads a column share the rows of `partial`; always in the same order
__global__ __launch_bounds__(1024) void sum_parts_kernel(const float *partial, int parts, int d, float *out) {
  __shared__ float s[32][33];
  const int col = threadIdx.x & 31, of = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
  float v[kBackParts / 32];
#pragma unroll
  for (int i = 0; i < kBackParts / 32; ++i) {
    const int k = of + i * 32;
    v[i] = c < d && k < parts ? partial[(int64_t)k * d + c] : 0.f;
  }
#pragma unroll
  for (int i = 1; i < kBackParts / 32; ++i) v[0] += v[i];
  s[of][col] = v[0];
  __syncthreads();
  if (of == 0 && c < d) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += s[i][col];
    out[c] = sum;
  }
}

template <int N>
struct Const {
  static constexpr int value = N;
};

}  // namespace

hipError_t launch_norm_rows(const NormRowsParams &p, int n_cus, hipStream_t s) {
  const int d = p.hidden;
  // Units of 8 columns wherever a row begins, the last one over the one before it; rows of fewer by single columns.  4096 rows of
  // 8191, fp32 and bf16: 88 us, by single columns 107; all in bf16 48 and 57, the backward 92 and 180.
  const bool wide = d >= 8;
  const int vec = wide ? 8 : 1, most = 4;
  int waves = 1;
  while ((int64_t)waves * 64 * vec * most < d) waves *= 2;
  // few rows: a row over more wavefronts, one step each (64 rows of 2048: 3.1 us, otherwise 4.7; 600 rows 4.7 and 5.8)
  while (p.n_rows < 4 * n_cus && waves < kMaxWaves && waves * 64 * vec < d) waves *= 2;
  const int nv = (d + waves * 64 * vec - 1) / (waves * 64 * vec);
  const int rows_per_wg = waves == 1 ? 4 : 1;
  const RowGrid g = row_grid(((int64_t)p.n_rows + rows_per_wg - 1) / rows_per_wg);
  const dim3 grid(g.x, g.y), block(waves == 1 ? 256 : waves * 64);
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
      with(Const<1>{}, Const<1>{});
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

namespace {
struct BackShape {
  int vec, waves, nv, groups, parts;
};
// wavefronts of a row, so that a lane has at most 16 of its columns (of which it keeps five values each in registers)
BackShape back_shape(int n_rows, int hidden, bool wide) {
  BackShape b;
  b.vec = wide ? 8 : 1;
  const int most = 2;
  b.waves = 1;
  while (b.waves * 64 * b.vec * most < hidden) b.waves *= 2;
  b.nv = (hidden + b.waves * 64 * b.vec - 1) / (b.waves * 64 * b.vec);
  b.groups = kBackWaves / b.waves;
  b.parts = std::min((n_rows + b.groups - 1) / b.groups, kBackParts);
  return b;
}
}  // namespace

int norm_rows_backward_parts(int n_rows, int hidden) { return std::min(n_rows, kBackParts); }

hipError_t launch_norm_rows_backward(const NormRowsBackwardParams &p, hipStream_t s) {
  const int d = p.hidden;
  const bool wide = d >= 8;
  const BackShape b = back_shape(p.n_rows, d, wide);
  const int nv = b.nv, parts = b.parts;
  const size_t lds = p.dgain ? (size_t)(b.groups - 1) * d * sizeof(float) : 0;
  const auto go = [&](auto H, auto X) {
    const auto with = [&](auto VEC, auto NV) {
      if (parts == 0) return;  // (no rows: dgain is zero)
      hipLaunchKernelGGL((norm_rows_backward_kernel<decltype(H)::value, decltype(X)::value, decltype(VEC)::value, decltype(NV)::value>),
                         dim3(parts), dim3(kBackWaves * 64), lds, s, p, b.waves);
    };
    if (wide) {
      if (nv == 1) with(Const<8>{}, Const<1>{});
      else with(Const<8>{}, Const<2>{});
    } else {
      with(Const<1>{}, Const<1>{});
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
  hipLaunchKernelGGL(sum_parts_kernel, dim3((d + 31) / 32), dim3(1024), 0, s, p.partial, parts, d, p.dgain);
  return hipGetLastError();
}

}  // namespace moe
