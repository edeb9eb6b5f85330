// Tokens sorted by the expert that takes them, their rows brought into that order and the results brought back.
//
// A place is a token's k-th choice, place = token * top_k + k.  The sort is a stable counting sort: an expert's rows come in
// the order of the tokens, so the result does not depend on timing (the only atomics add whole numbers up).  Places without an expert (an id outside
// 0..n_experts-1) have no row; as many rows at the end of the order belong to nobody and are filled with zeros.
#include "rows.h"

namespace moe {
namespace {

constexpr int kSortWaves = 16, kSortThreads = kSortWaves * 64;
constexpr int kSortBlocks = 256;      // workgroups of the two-launch form at most
// Places that one workgroup sorts by itself (2044 take 4.8 us, in two launches 6.6; 4000 7.1 and 6.8; 8000 11.8 and 8.1; 16384 25 and
// 9).  More are counted by a launch of their own first, since no workgroup knows another's counts within one.
constexpr int kSortSingle = 4096;
constexpr int kSortChunk = 1024;      // places a workgroup takes at least in the two-launch form: one for each thread

// Lanes of the wavefront that hold the same key as this one.  BITS: bits of a key.
template <int BITS>
__device__ __forceinline__ uint64_t same_key(int key) {
  uint64_t m = ~0ull;
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const bool one = (key >> b) & 1;
    const uint64_t v = __ballot(one);
    m &= one ? v : ~v;
  }
  return m;
}
__device__ __forceinline__ int key_of(const int32_t *ids, int64_t at, int64_t end, int n_experts) {
  const int id = at < end ? ids[at] : -1;
  return (uint32_t)id < (uint32_t)n_experts ? id : n_experts;  // n_experts: no row
}

// counts[wave][expert] of the places begin..end, a contiguous part for each wavefront
template <int BITS>
__device__ __forceinline__ void count_places(const int32_t *ids, int64_t begin, int64_t end, int64_t per_wave, int n_experts, int *counts,
                                             int pitch) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t w0 = begin + wave * per_wave, w1 = min(end, w0 + per_wave);
  for (int64_t at = w0; at < w1; at += 64) {
    const int key = key_of(ids, at + lane, w1, n_experts);
    const uint64_t m = same_key<BITS>(key);
    if (key < n_experts && (m & ((1ull << lane) - 1)) == 0) counts[wave * pitch + key] += __popcll(m);
  }
}
// the same walk with counts turned into the first free row of each (wavefront, expert)
template <int BITS>
__device__ __forceinline__ void place_rows(const int32_t *ids, int64_t begin, int64_t end, int64_t per_wave, int n_experts, int *next, int pitch,
                                           int32_t *row_of, int32_t *entry_of) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t w0 = begin + wave * per_wave, w1 = min(end, w0 + per_wave);
  for (int64_t at = w0; at < w1; at += 64) {
    const int key = key_of(ids, at + lane, w1, n_experts);
    const uint64_t m = same_key<BITS>(key);
    const uint64_t before = m & ((1ull << lane) - 1);
    int row = -1;
    if (key < n_experts) {
      row = next[wave * pitch + key] + __popcll(before);
      entry_of[row] = (int32_t)(at + lane);
    }
    if (at + lane < w1) row_of[at + lane] = row;
    __builtin_amdgcn_wave_barrier();
    if (key < n_experts && before == 0) next[wave * pitch + key] += __popcll(m);
    __builtin_amdgcn_wave_barrier();
  }
}

// exclusive sum over the threads of the workgroup (1024); `s` holds 16 words
__device__ __forceinline__ int block_scan(int v, int *s, int &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) s[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    const int c = s[w];
    if (w < wave) before += c;
    all += c;
  }
  total = all;
  return before + x - v;
}

// BLOCKS = false: one workgroup sorts everything.  BLOCKS = true: workgroup b takes places b * chunk ..; hist [workgroups]
// [n_experts] holds what each counts.
template <int BITS, bool BLOCKS>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(const int32_t *ids, int64_t n, int n_experts, int64_t chunk, const int32_t *hist,
                                                            int32_t *offsets, int32_t *row_of, int32_t *entry_of) {
  extern __shared__ int counts[];  // [kSortWaves][n_experts], two words per expert, 16 words
  int *sum_all = counts + kSortWaves * n_experts, *sum_earlier = sum_all + n_experts, *scratch = sum_earlier + n_experts;
  const int e = threadIdx.x;
  const int64_t begin = BLOCKS ? blockIdx.x * chunk : 0, end = BLOCKS ? min(n, begin + chunk) : n;
  const int64_t per_wave = ((end - begin + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  for (int i = threadIdx.x; i < (kSortWaves + 2) * n_experts; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  if constexpr (BLOCKS) {
    // what all workgroups and those before this one have counted: whole numbers, the order of the additions is of no matter
    const int parts = kSortThreads / n_experts, k = threadIdx.x / n_experts, x = threadIdx.x - k * n_experts;
    if (k < parts) {
      int all = 0, earlier = 0;
#pragma unroll 8
      for (int b = k; b < (int)gridDim.x; b += parts) {
        const int c = hist[b * n_experts + x];
        all += c;
        earlier += b < (int)blockIdx.x ? c : 0;
      }
      atomicAdd(&sum_all[x], all);
      atomicAdd(&sum_earlier[x], earlier);
    }
  }
  count_places<BITS>(ids, begin, end, per_wave, n_experts, counts, n_experts);
  __syncthreads();
  // this expert's places in all of the input and in the workgroups before this one
  int all = 0, earlier = 0;
  if (e < n_experts) {
    if constexpr (BLOCKS) {
      all = sum_all[e];
      earlier = sum_earlier[e];
    } else {
      for (int w = 0; w < kSortWaves; ++w) all += counts[w * n_experts + e];
    }
  }
  int total;
  const int first = block_scan(all, scratch, total);
  if (e < n_experts) {
    if (blockIdx.x == 0) offsets[e] = first;
    int at = first + earlier;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = counts[w * n_experts + e];
      counts[w * n_experts + e] = at;
      at += c;
    }
  }
  if (blockIdx.x == 0 && e == 0) offsets[n_experts] = total;
  __syncthreads();
  place_rows<BITS>(ids, begin, end, per_wave, n_experts, counts, n_experts, row_of, entry_of);
  // rows of nobody
  for (int64_t r = total + (int64_t)blockIdx.x * kSortThreads + threadIdx.x; r < n; r += (int64_t)gridDim.x * kSortThreads) entry_of[r] = -1;
}

template <int BITS>
__global__ __launch_bounds__(kSortThreads) void histogram_kernel(const int32_t *ids, int64_t n, int n_experts, int64_t chunk, int32_t *hist) {
  extern __shared__ int counts[];
  const int64_t begin = blockIdx.x * chunk, end = min(n, begin + chunk);
  const int64_t per_wave = ((end - begin + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  for (int i = threadIdx.x; i < kSortWaves * n_experts; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  count_places<BITS>(ids, begin, end, per_wave, n_experts, counts, n_experts);
  __syncthreads();
  if ((int)threadIdx.x < n_experts) {
    int c = 0;
    for (int w = 0; w < kSortWaves; ++w) c += counts[w * n_experts + threadIdx.x];
    hist[blockIdx.x * n_experts + threadIdx.x] = c;
  }
}

int64_t sort_chunk(int64_t n) {
  const int64_t even = (n + kSortBlocks - 1) / kSortBlocks;
  return even > kSortChunk ? (even + 1023) / 1024 * 1024 : kSortChunk;
}

// The rows (and weights) of token t: lane k loads place k, all of them in one request.  -1: none (whatever lies outside the order
// counts as none).
struct Places {
  int row_v;
  float weight_v;
  __device__ __forceinline__ Places(const OrderParams &o, int64_t t, const float *weight, int lane) {
    const int64_t at = t * o.top_k + min(lane, o.top_k - 1);
    row_v = o.row_of[at];
    if ((uint32_t)row_v >= (uint32_t)o.n_tokens * (uint32_t)o.top_k || lane >= o.top_k) row_v = -1;
    weight_v = weight ? weight[at] : 1.f;
  }
  __device__ __forceinline__ int row(int k) const { return __builtin_amdgcn_readlane(row_v, k); }
  __device__ __forceinline__ float weight(int k) const { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight_v), k)); }
};
// how many rows belong to somebody
__device__ __forceinline__ int64_t rows_used(const OrderParams &o) { return max(0, o.offsets[o.n_experts]); }

// ---- rows into the order ----
// A wavefront takes a token: it reads the row once and writes it to each of its places.  V: 16 bytes wherever the row begins (the
// last unit begins where it has 16 and writes again what the one before has written), or single bytes of a shorter row.  Memory
// bounds it: 8191 rows of 2048 bf16 to eight places each 50 us (6.0 TB/s); 4096 rows of 2047 to four places 17.4 us by
// elements of 2 bytes, 14.5 so.
template <typename V>
__global__ __launch_bounds__(256) void gather_kernel(const OrderParams o, const uint8_t *x, int64_t x_stride, int row_bytes, const float *scale,
                                                     uint8_t *xs, float *xs_scale) {
  const int lane = threadIdx.x & 63;
  const int64_t t = row_group() * 4 + (threadIdx.x >> 6);
  if (t >= o.n_tokens) return;
  const Places places(o, t, nullptr, lane);
  int row[MOE_MAX_TOPK];
#pragma unroll
  for (int k = 0; k < MOE_MAX_TOPK; ++k) row[k] = places.row(k);
  const uint8_t *in = x + t * x_stride;
  constexpr int U = 4, B = sizeof(V);  // units in flight per lane; bytes of one
  for (int c = lane * B; c < row_bytes; c += 64 * B * U) {
    V v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const V *>(in + min(c + u * 64 * B, row_bytes - B));
#pragma unroll
    for (int k = 0; k < MOE_MAX_TOPK; ++k) {
      if (row[k] < 0) continue;
      uint8_t *to = xs + (int64_t)row[k] * row_bytes;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c + u * 64 * B < row_bytes) *reinterpret_cast<V *>(to + min(c + u * 64 * B, row_bytes - B)) = v[u];
    }
  }
  if (scale && lane < o.top_k) {
    if (places.row_v >= 0) xs_scale[places.row_v] = scale[t];
  }
  // rows of nobody: as many as there are places without a row, one token's wavefront after the other
  const int64_t n = (int64_t)o.n_tokens * o.top_k;
  for (int64_t r = rows_used(o) + t; r < n; r += o.n_tokens) {
    for (int c = lane * B; c < row_bytes; c += 64 * B) *reinterpret_cast<V *>(xs + r * row_bytes + min(c, row_bytes - B)) = V{};
    if (scale && lane == 0) xs_scale[r] = 0.f;
  }
}

// ---- results back ----
// y = base + sum over k of weight * row, in the order of k.  KC: top_k rounded up to a power of two.  Places without a row read
// one that is there (or nothing at all if there is none) and are left out by a selection, not by a weight of 0.  A wavefront takes
// a token, CH units of a row at a time, so that it reads a row's bytes one after the other (8191 x 8 rows of 2048 bf16 onto fp32:
// 117 us by single units, 110 so, 92 with loads that leave the caches alone: 4.4 TB/s).  Memory bounds it.
template <int YS, int Y, int VEC, int KC, int CH>
__global__ __launch_bounds__(256) void combine_kernel(const OrderParams o, const void *ys, const float *weight, const void *base, void *y) {
  const int lane = threadIdx.x & 63;
  const int64_t t = row_group() * 4 + (threadIdx.x >> 6);
  if (t >= o.n_tokens) return;
  const int d = o.hidden;
  const Places places(o, t, weight, lane);
  int row[KC];
  float w[KC];
  int some = -1;
#pragma unroll
  for (int k = 0; k < KC; ++k) {
    row[k] = places.row(k);
    w[k] = places.weight(k);
    if (row[k] >= 0) some = row[k];
  }
  for (int c = lane * VEC; c < d; c += 64 * VEC * CH) {
    // (units behind the last one load it again)
    RowUnit unit[CH];
#pragma unroll
    for (int u = 0; u < CH; ++u) unit[u] = row_unit<VEC>(c + u * 64 * VEC, d);
    float acc[CH][VEC], b[CH][VEC];
    if (base)
#pragma unroll
      for (int u = 0; u < CH; ++u) load_row<Y>(base, t * d + unit[u].at, b[u]);
#pragma unroll
    for (int u = 0; u < CH; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) acc[u][i] = 0.f;
    if (some >= 0) {
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const int64_t from = (int64_t)(row[k] >= 0 ? row[k] : some) * d;
#pragma unroll
        for (int u = 0; u < CH; ++u) {
          float v[VEC];
          load_row<YS, VEC, true>(ys, from + unit[u].at, v);
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[u][i] = row[k] >= 0 ? __builtin_fmaf(w[k], v[i], acc[u][i]) : acc[u][i];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      if (c + u * 64 * VEC >= d) continue;
      if (base)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[u][i] += b[u][i];
      store_unit<Y>(y, t * d, unit[u], acc[u]);
    }
  }
}

// dys[row] = weight * dy[token], dweight = <dy[token], ys[row]>.  A wavefront takes a token, so that its row of dy is read once and
// the dot products stay in registers.  Memory bounds it: 4096 x 4 rows of 2048 bf16, 151 MB in 29 us (5.2 TB/s).
template <int DY, int YS, int VEC>
__global__ __launch_bounds__(256) void combine_backward_kernel(const OrderParams o, const void *dy, const void *ys, const float *weight, void *dys,
                                                               float *dweight) {
  const int lane = threadIdx.x & 63;
  const int64_t t = row_group() * 4 + (threadIdx.x >> 6);
  if (t >= o.n_tokens) return;
  const int d = o.hidden;
  const Places places(o, t, weight, lane);
  int row[MOE_MAX_TOPK];
  float w[MOE_MAX_TOPK], dot[MOE_MAX_TOPK];
#pragma unroll
  for (int k = 0; k < MOE_MAX_TOPK; ++k) {
    row[k] = places.row(k);
    w[k] = places.weight(k);
    dot[k] = 0.f;
  }
  for (int c = lane * VEC; c < d; c += 64 * VEC) {
    const RowUnit u = row_unit<VEC>(c, d);
    float g[VEC];
    load_row<DY>(dy, t * d + u.at, g);
#pragma unroll
    for (int k = 0; k < MOE_MAX_TOPK; ++k) {
      if (row[k] < 0) continue;
      const int64_t at = (int64_t)row[k] * d;
      float v[VEC];
      if (dweight) {
        load_row<YS, VEC, true>(ys, at + u.at, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) dot[k] = i >= u.skip ? __builtin_fmaf(g[i], v[i], dot[k]) : dot[k];
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = w[k] * g[i];
      store_unit<YS>(dys, at, u, v);
    }
  }
  if (dweight) {
#pragma unroll
    for (int k = 0; k < MOE_MAX_TOPK; ++k) {
      if (k >= o.top_k) continue;
      const float s = wave_sum(dot[k]);
      if (lane == 0) dweight[t * o.top_k + k] = row[k] >= 0 ? s : 0.f;
    }
  }
  const int64_t n = (int64_t)o.n_tokens * o.top_k;
  for (int64_t r = rows_used(o) + t; r < n; r += o.n_tokens) {
    float zero[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) zero[i] = 0.f;
    for (int c = lane * VEC; c < d; c += 64 * VEC) store_row<YS>(dys, r * d + row_unit<VEC>(c, d).at, zero);
  }
}

template <int N>
struct Const {
  static constexpr int value = N;
};

}  // namespace

size_t sort_tokens_bytes(int64_t n, int n_experts) {
  if (n <= kSortSingle) return 0;
  return (size_t)((n + sort_chunk(n) - 1) / sort_chunk(n)) * n_experts * sizeof(int32_t);
}

hipError_t launch_sort_tokens(const int32_t *ids, int64_t n, int n_experts, int32_t *offsets, int32_t *row_of, int32_t *entry_of,
                              void *workspace, hipStream_t s) {
  int32_t *hist = static_cast<int32_t *>(workspace);
  const size_t lds = ((size_t)(kSortWaves + 2) * n_experts + 16) * sizeof(int);
  const auto go = [&](auto BITS) {
    constexpr int B = decltype(BITS)::value;
    if (n <= kSortSingle) {
      hipLaunchKernelGGL((sort_kernel<B, false>), dim3(1), dim3(kSortThreads), lds, s, ids, n, n_experts, (int64_t)0, hist, offsets, row_of, entry_of);
      return;
    }
    const int64_t chunk = sort_chunk(n);
    const dim3 grid((uint32_t)((n + chunk - 1) / chunk));
    hipLaunchKernelGGL((histogram_kernel<B>), grid, dim3(kSortThreads), lds, s, ids, n, n_experts, chunk, hist);
    hipLaunchKernelGGL((sort_kernel<B, true>), grid, dim3(kSortThreads), lds, s, ids, n, n_experts, chunk, hist, offsets, row_of, entry_of);
  };
  // (keys 0..n_experts)
  if (n_experts < 64) go(Const<6>{});
  else if (n_experts < 128) go(Const<7>{});
  else go(Const<10>{});
  return hipGetLastError();
}

hipError_t launch_gather_rows(const OrderParams &o, const void *x, int fmt, int64_t x_stride, const float *scale, void *xs, float *xs_scale,
                              hipStream_t s) {
  const int64_t row = (int64_t)o.hidden * row_elem(fmt), stride = x_stride * row_elem(fmt);
  const RowGrid g = row_grid(((int64_t)o.n_tokens + 3) / 4);
  const dim3 grid(g.x, g.y), block(256);
  const auto go = [&](auto v) {
    using V = decltype(v);
    hipLaunchKernelGGL((gather_kernel<V>), grid, block, 0, s, o, static_cast<const uint8_t *>(x), stride, (int)row, scale,
                       static_cast<uint8_t *>(xs), xs_scale);
  };
  if (row >= 16) go(rows_u32x4_codes{});
  else go(uint8_t{});
  return hipGetLastError();
}

hipError_t launch_combine_rows(const OrderParams &o, const void *ys, int ys_fmt, const float *weight, const void *base, void *y, int y_fmt,
                               hipStream_t s) {
  // Units of 8 columns wherever a row begins, the last one over the one before it; rows of fewer by single columns.  4096 x 4 rows of
  // 2047 bf16: 16 us, by single columns 64.
  const bool wide = o.hidden >= 8;
  const RowGrid g = row_grid(((int64_t)o.n_tokens + 3) / 4);
  const dim3 grid(g.x, g.y), block(256);
  const auto go = [&](auto YS, auto Y) {
    const auto with = [&](auto VEC, auto KC) {
      const auto go_on = [&](auto CH) {
        hipLaunchKernelGGL((combine_kernel<decltype(YS)::value, decltype(Y)::value, decltype(VEC)::value, decltype(KC)::value, decltype(CH)::value>),
                           grid, block, 0, s, o, ys, weight, base, y);
      };
      // (4096 x 4 rows: of 2048 columns 13 us by four units, 17 by one; of 512 columns 4.4 by one, 6.4 by four)
      if (o.hidden <= 64 * decltype(VEC)::value * 2) go_on(Const<1>{});
      else go_on(Const<4>{});
    };
    const auto k = [&](auto VEC) {
      if (o.top_k == 1) with(VEC, Const<1>{});
      else if (o.top_k == 2) with(VEC, Const<2>{});
      else if (o.top_k <= 4) with(VEC, Const<4>{});
      else with(VEC, Const<8>{});
    };
    if (wide) k(Const<8>{});
    else k(Const<1>{});
  };
  const auto y_of = [&](auto YS) {
    if (y_fmt == MOE_R_FP32) go(YS, Const<MOE_R_FP32>{});
    else go(YS, Const<MOE_R_BF16>{});
  };
  if (ys_fmt == MOE_R_FP32) y_of(Const<MOE_R_FP32>{});
  else y_of(Const<MOE_R_BF16>{});
  return hipGetLastError();
}

hipError_t launch_combine_rows_backward(const OrderParams &o, const void *dy, int dy_fmt, const void *ys, int ys_fmt, const float *weight,
                                        void *dys, float *dweight, hipStream_t s) {
  const bool wide = o.hidden >= 8;  // (see above; 4096 x 4 rows of 2047 bf16: 31 us, by single columns 97)
  const RowGrid g = row_grid(((int64_t)o.n_tokens + 3) / 4);
  const dim3 grid(g.x, g.y), block(256);
  const auto go = [&](auto DY, auto YS) {
    const auto with = [&](auto VEC) {
      hipLaunchKernelGGL((combine_backward_kernel<decltype(DY)::value, decltype(YS)::value, decltype(VEC)::value>), grid, block, 0, s, o, dy, ys,
                         weight, dys, dweight);
    };
    if (wide) with(Const<8>{});
    else with(Const<1>{});
  };
  const auto ys_of = [&](auto DY) {
    if (ys_fmt == MOE_R_FP32) go(DY, Const<MOE_R_FP32>{});
    else go(DY, Const<MOE_R_BF16>{});
  };
  if (dy_fmt == MOE_R_FP32) ys_of(Const<MOE_R_FP32>{});
  else ys_of(Const<MOE_R_BF16>{});
  return hipGetLastError();
}

}  // namespace moe
