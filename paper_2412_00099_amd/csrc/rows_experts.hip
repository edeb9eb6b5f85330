// SwiGLU experts on rows sorted by expert, straight on the blobs (record i = gate row i | up row i | column i of down, d weights
// each), and their gradients.  Expert e takes rows offsets[e] .. offsets[e+1]:
//
//   G = X Wg^T, U = X Wu^T, H = silu(G) U, Y = H Wd^T
//   dH = dY Wd, dG = dH U s (1 + G (1 - s)), dU = dH G s (s = sigmoid G), dX = dG Wg + dU Wu
//   dWg = dG^T X, dWu = dU^T X, dWd^T = H^T dY
//
// Three forms of product, all on the matrix cores with sums in 32 bits:
//   rows_kernel     both operands have the summed index side by side (X with gate / up rows, dY with down columns)
//   columns_kernel  the summed index are the records, so the weights' side is transposed on its way out of LDS
//   weights_kernel  the summed index are the rows: both sides are transposed
// H, G, U and their gradients pass through memory rounded to bf16, as the rows do.  With 8-bit weights the rows of the first
// product are 8-bit codes too (whole-number sums, exact), H stays bf16 and the weights of down are widened to bf16, which holds
// every code exactly.
//
// Which expert and which of its rows a workgroup has is worked out from `offsets` on the device; the grid is the most that
// n_rows rows can need and workgroups without a tile leave.  All loads go through buffer resources that end where the expert's
// rows or records end: what lies beyond arrives as zeros.
#include "rows.h"

namespace moe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __amdgpu_buffer_rsrc_t Buffer;
#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T *)(p))

constexpr int kTile = 128;              // rows and columns of a workgroup's tile
constexpr int kStepBytes = 128;         // bytes of a row that a step takes: 64 bf16 or 128 8-bit values
constexpr int kBlock = 256;
constexpr int kTileBytes = kTile * kStepBytes;  // 16 KB, one operand's part of a step

__device__ __forceinline__ Buffer buffer_of(const void *base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}
// 16 bytes per lane straight into LDS, lane after lane from `lds` (the same in every lane)
__device__ __forceinline__ void to_lds(Buffer b, uint32_t off, uint32_t at, uint8_t *lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b, LDS_PTR(void, lds), 16, off, at, 0, 0);
}
__device__ __forceinline__ void wait_loads_and_meet() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x4 mma(i32x4 a, i32x4 b, i32x4 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// The tile of a workgroup.
struct Tile {
  int expert;    // n_experts: the rows of nobody; -1: no tile
  int row0, rows;
  int col;
};
// Tiles in the order expert, column, row, so that the workgroups that share weights are neighbours; the list is dealt to the
// eight XCDs in eight parts, since workgroups go to them in turn and each has an L2 of its own.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ Tile search_tile(const ExpertRowsParams &p, int n_cols, bool nobody, int block) {
  const int lane = threadIdx.x & 63, groups = p.n_experts + (nobody ? 1 : 0);
  int total = 0;
  for (int e0 = 0; e0 < groups; e0 += 64) {
    const int e = e0 + lane;
    int c = 0;
    if (e < groups) {
      const int a = min(max(p.offsets[e], 0), p.n_rows), b = e < p.n_experts ? min(p.offsets[e + 1], p.n_rows) : p.n_rows;
      c = max(b - a, 0);
    }
    int t = (c + kTile - 1) / kTile;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) t += __shfl_xor(t, o);
    total += t;
  }
  total = uniform(total) * n_cols;
  Tile r;
  r.expert = -1;
  r.row0 = r.rows = r.col = 0;
  const int part = (total + 7) / 8, in_part = block >> 3, want = (block & 7) * part + in_part;
  if (in_part >= part || want >= total) return r;
  int before = 0;
  for (int e0 = 0; e0 < groups; e0 += 64) {
    const int e = e0 + lane;
    int a = 0, c = 0;
    if (e < groups) {
      a = min(max(p.offsets[e], 0), p.n_rows);
      const int b = e < p.n_experts ? min(p.offsets[e + 1], p.n_rows) : p.n_rows;
      c = max(b - a, 0);
    }
    const int t = (c + kTile - 1) / kTile * n_cols;
    int upto = t;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    const uint64_t past = __ballot(before + upto > want);
    if (past != 0) {
      const int l = __ffsll((unsigned long long)past) - 1;
      const int left = want - before - __shfl(upto - t, l), count = __shfl(c, l), row_tiles = (count + kTile - 1) / kTile;
      r.expert = e0 + l;
      r.col = left / row_tiles;
      const int rt = left - r.col * row_tiles;
      r.row0 = __shfl(a, l) + rt * kTile;
      r.rows = min(kTile, count - rt * kTile);
      return r;
    }
    before += uniform(__shfl(upto, 63));
  }
  return r;
}
// (in scalar registers: it makes the buffer resources)
__device__ __forceinline__ Tile find_tile(const ExpertRowsParams &p, int n_cols, bool nobody, int block) {
  Tile t = search_tile(p, n_cols, nobody, block);
  t.expert = uniform(t.expert);
  t.row0 = uniform(t.row0);
  t.rows = uniform(t.rows);
  t.col = uniform(t.col);
  return t;
}
int tile_grid(const ExpertRowsParams &p, int n_cols, bool nobody) {
  const int64_t groups = p.n_experts + (nobody ? 1 : 0);
  const int64_t tiles = (p.n_rows / kTile + (groups < p.n_rows ? groups : p.n_rows)) * n_cols;
  return (int)((tiles + 7) / 8 * 8);
}

// ---- LDS images -------------------------------------------------------------------------------------------
// Side by side: 128 rows of 128 bytes.  16-byte chunk c of row r lies at c ^ (r / 2 % 8): the 16 rows that a fragment reads at
// one chunk then cover all banks.
__device__ __forceinline__ int chunk_at(int r, int c) { return c ^ ((r >> 1) & 7); }
__device__ __forceinline__ i32x4 fragment(const uint8_t *tile, int r, int chunk) {
  return *reinterpret_cast<const i32x4 *>(tile + r * kStepBytes + chunk_at(r, chunk) * 16);
}
// Transposed, 16-bit: 64 rows (the summed index) of 128 columns, 256 bytes.  The 32 bytes of 16 columns move as one: group g of
// row k lies at g ^ f(k), so that the 8 rows that are read together lie in different banks.
__device__ __forceinline__ int swap16(int k) { return (k & 3) | ((k >> 1) & 4); }
// the fragment of 16 columns (group g) and 32 rows from k0 on: the lane's column, 8 rows
__device__ __forceinline__ i32x4 fragment_t16(const uint8_t *tile, int g, int k0, int lane) {
  const int j = lane & 15, k = k0 + (lane >> 4) * 8 + (j >> 2);
  const uint8_t *at = tile + k * 256 + ((g ^ swap16(k)) * 32) + (j & 3) * 8;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + 4 * 256));
  return __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Transposed, 8-bit: 64 rows of 128 columns, 128 bytes; 16 columns are 16 bytes, group g of row k at g ^ (k % 8).  The codes
// q + 128 are widened to bf16 (exact).
__device__ __forceinline__ i32x4 fragment_t8(const uint8_t *tile, int g, int k0, int lane) {
  const int j = lane & 15, k = k0 + (lane >> 4) * 8 + (j >> 1);
  const uint8_t *at = tile + k * 128 + ((g ^ (k & 7)) * 16) + (j & 1) * 8;
  const i32x2 q = __builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(i32x2, at));
  i32x4 v;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const uint32_t u = (uint32_t)q[w];
    const float f0 = (float)(u & 0xff) - 128.f, f1 = (float)((u >> 8) & 0xff) - 128.f, f2 = (float)((u >> 16) & 0xff) - 128.f,
                f3 = (float)(u >> 24) - 128.f;
    // (whole numbers up to 128: the lower halves of the floats are zero)
    v[2 * w] = (int)__builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302);
    v[2 * w + 1] = (int)__builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302);
  }
  return v;
}

// offsets of the lane's loads for 128 rows of 128 bytes: load i of wavefront w covers rows (w * 4 + i) * 8 ..
__device__ __forceinline__ int side_row(int i) { return ((threadIdx.x >> 6) * 4 + i) * 8 + (threadIdx.x & 63) / 8; }
__device__ __forceinline__ uint32_t side_chunk(int r) { return (uint32_t)chunk_at(r, threadIdx.x & 7) * 16; }

__device__ __forceinline__ void store4(uint16_t *p, const float (&v)[4]) {
  rows_u32x2 w;
  w[0] = pack_bf16(v[0], v[1]);
  w[1] = pack_bf16(v[2], v[3]);
  *reinterpret_cast<rows_u32x2 *>(p) = w;
}
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }
__device__ __forceinline__ float half_at(const uint8_t *p, int64_t at) { return (float)reinterpret_cast<const _Float16 *>(p)[at]; }

// ---- rows x rows ----------------------------------------------------------------------------------------------
enum { kUp = 0, kDgu = 1 };
// kUp: 64 records a tile; its LDS rows are 16 gate rows, 16 up rows, 16 gate rows, .., so that a wavefront has both products of
// a record in the same lane and register.  kDgu: 128 records a tile (their down columns).
template <bool INT8, int MODE>
__global__ __launch_bounds__(kBlock) void rows_kernel(const ExpertRowsParams p, const uint8_t *xs, const float *scale, const uint16_t *gu_in,
                                                      uint16_t *h, uint16_t *gu) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][kTileBytes];
  constexpr int REC = MODE == kUp ? 64 : 128;
  constexpr int EL = INT8 ? 1 : 2;
  const int pitch = expert_rows_pitch(p.inter);
  const Tile t = find_tile(p, (pitch + REC - 1) / REC, false, blockIdx.x);
  if (t.expert < 0) return;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
  const uint32_t row_bytes = (uint32_t)p.hidden * EL;
  const uint8_t *blob = p.blobs + t.expert * p.blob_stride;
  const Buffer a = buffer_of(xs + (int64_t)t.row0 * row_bytes, t.rows * row_bytes), b = buffer_of(blob, (uint32_t)p.inter * 3 * row_bytes);
  const int rec0 = t.col * REC;
  uint32_t a_off[4], b_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = side_row(i);
    a_off[i] = (uint32_t)r * row_bytes + side_chunk(r);
    const int rec = rec0 + (MODE == kUp ? (r >> 5) * 16 + (r & 15) : r), which = MODE == kUp ? (r >> 4) & 1 : 2;
    b_off[i] = rec < p.inter ? (uint32_t)(rec * 3 + which) * row_bytes + side_chunk(r) : 0xffffff00u;
  }
  const auto stage = [&](int buf, int k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to_lds(a, a_off[i], k * kStepBytes, &lds[buf][0][(wave * 4 + i) * 1024]);
      to_lds(b, b_off[i], k * kStepBytes, &lds[buf][1][(wave * 4 + i) * 1024]);
    }
  };
  using Acc = std::conditional_t<INT8, i32x4, f32x4>;
  Acc acc[4][4];
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int n = 0; n < 4; ++n) acc[m][n] = Acc{};
  const int steps = row_bytes / kStepBytes;
  stage(0, 0);
  for (int k = 0; k < steps; ++k) {
    wait_loads_and_meet();
    if (k + 1 < steps) stage((k + 1) & 1, k + 1);
    const uint8_t *ta = lds[k & 1][0], *tb = lds[k & 1][1];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      i32x4 x[4], w[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) x[m] = fragment(ta, wm * 64 + m * 16 + (lane & 15), kk * 4 + (lane >> 4));
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        w[n] = fragment(tb, wn * 64 + n * 16 + (lane & 15), kk * 4 + (lane >> 4));
        if constexpr (INT8) w[n] ^= (int)0x80808080;
      }
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = mma(w[n], x[m], acc[m][n]);
    }
  }
  // lane: row lane % 16 of each 16 rows, records (lane / 16) * 4 .. + 3 of each 16 records
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int r = wm * 64 + m * 16 + (lane & 15);
    if (r >= t.rows) continue;
    const int64_t row = t.row0 + r;
    if constexpr (MODE == kUp) {
      const float sx = INT8 ? scale[row] : 1.f;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int rec = rec0 + wn * 32 + n * 16 + (lane >> 4) * 4;
        float g[4], u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[i] = (float)acc[m][2 * n][i];
          u[i] = (float)acc[m][2 * n + 1][i];
          if constexpr (INT8) {
            const uint8_t *tail = blob + (int64_t)p.inter * 3 * row_bytes;
            const bool in = rec + i < p.inter;
            g[i] = in ? g[i] * (sx * half_at(tail, rec + i)) : 0.f;
            u[i] = in ? u[i] * (sx * half_at(tail, p.inter + rec + i)) : 0.f;
          }
          v[i] = g[i] * sigmoid(g[i]) * u[i];
        }
        store4(h + row * pitch + rec, v);
        if (gu) {
          store4(gu + row * 2 * pitch + rec, g);
          store4(gu + (row * 2 + 1) * pitch + rec, u);
        }
      }
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int rec = rec0 + wn * 64 + n * 16 + (lane >> 4) * 4;
        if (rec >= pitch) continue;
        const rows_u32x2 gw = *reinterpret_cast<const rows_u32x2 *>(gu_in + row * 2 * pitch + rec),
                         uw = *reinterpret_cast<const rows_u32x2 *>(gu_in + (row * 2 + 1) * pitch + rec);
        float dg[4], du[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float g = i & 1 ? bf16_hi(gw[i >> 1]) : bf16_lo(gw[i >> 1]), u = i & 1 ? bf16_hi(uw[i >> 1]) : bf16_lo(uw[i >> 1]);
          const float s = sigmoid(g), dh = acc[m][n][i];
          dg[i] = dh * u * (s * (1.f + g * (1.f - s)));
          du[i] = dh * (g * s);
        }
        store4(gu + row * 2 * pitch + rec, dg);
        store4(gu + (row * 2 + 1) * pitch + rec, du);
      }
    }
  }
}

// ---- rows x columns -------------------------------------------------------------------------------------------
// out = sum over `sections` of A_s W_s: A_s = columns s * pitch .. of a (a_pitch elements a row), W_s = part first + s of the
// records.  Down: H with the columns; the gradient of the rows: dG with the gate rows, dU with the up rows.
template <bool INT8>
__global__ __launch_bounds__(kBlock) void columns_kernel(const ExpertRowsParams p, const uint16_t *a_in, int a_pitch, int sections, int first,
                                                         uint16_t *out) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][kTileBytes];
  constexpr int EL = INT8 ? 1 : 2;
  constexpr int W_LOADS = INT8 ? 2 : 4;
  const int pitch = expert_rows_pitch(p.inter);
  const Tile t = find_tile(p, p.hidden / kTile, true, blockIdx.x);
  if (t.expert < 0) return;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
  const int n0 = t.col * kTile;
  if (t.expert == p.n_experts) {  // rows of nobody
    for (int r = threadIdx.x >> 4; r < t.rows; r += kBlock / 16)
      *reinterpret_cast<rows_u32x4 *>(out + (int64_t)(t.row0 + r) * p.hidden + n0 + (threadIdx.x & 15) * 8) = rows_u32x4{};
    return;
  }
  const uint32_t row_bytes = (uint32_t)p.hidden * EL, rec_bytes = 3 * row_bytes, a_bytes = (uint32_t)a_pitch * 2;
  const uint8_t *blob = p.blobs + t.expert * p.blob_stride;
  const Buffer a = buffer_of(a_in + (int64_t)t.row0 * a_pitch, t.rows * a_bytes), b = buffer_of(blob, (uint32_t)p.inter * rec_bytes);
  uint32_t a_off[4], b_off[W_LOADS];
  int b_row[W_LOADS];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = side_row(i);
    a_off[i] = (uint32_t)r * a_bytes + side_chunk(r);
  }
#pragma unroll
  for (int i = 0; i < W_LOADS; ++i) {
    int k, col;
    if constexpr (INT8) {
      k = (wave * W_LOADS + i) * 8 + lane / 8;
      col = ((lane & 7) ^ (k & 7)) * 16;
    } else {
      k = (wave * W_LOADS + i) * 4 + lane / 16;
      col = ((((lane & 15) >> 1) ^ swap16(k)) * 2 + (lane & 1)) * 16;
    }
    b_row[i] = k;
    b_off[i] = (uint32_t)k * rec_bytes + first * row_bytes + n0 * EL + col;
  }
  const int per_section = pitch / 64, steps = per_section * sections;
  const auto stage = [&](int buf, int s) {
    const int sec = s >= per_section ? 1 : 0, k = s - sec * per_section;
#pragma unroll
    for (int i = 0; i < 4; ++i) to_lds(a, a_off[i], s * kStepBytes, &lds[buf][0][(wave * 4 + i) * 1024]);
#pragma unroll
    for (int i = 0; i < W_LOADS; ++i) {
      const uint32_t off = b_row[i] + k * 64 < p.inter ? b_off[i] + (uint32_t)k * 64 * rec_bytes + sec * row_bytes : 0xffffff00u;
      to_lds(b, off, 0, &lds[buf][1][(wave * W_LOADS + i) * 1024]);
    }
  };
  f32x4 acc[4][4];
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int n = 0; n < 4; ++n) acc[m][n] = f32x4{};
  stage(0, 0);
  for (int s = 0; s < steps; ++s) {
    wait_loads_and_meet();
    if (s + 1 < steps) stage((s + 1) & 1, s + 1);
    const uint8_t *ta = lds[s & 1][0], *tb = lds[s & 1][1];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      i32x4 x[4], w[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) x[m] = fragment(ta, wm * 64 + m * 16 + (lane & 15), kk * 4 + (lane >> 4));
#pragma unroll
      for (int n = 0; n < 4; ++n) w[n] = INT8 ? fragment_t8(tb, wn * 4 + n, kk * 32, lane) : fragment_t16(tb, wn * 4 + n, kk * 32, lane);
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = mma(w[n], x[m], acc[m][n]);
    }
  }
  const uint8_t *down_scale = blob + (int64_t)p.inter * rec_bytes + (int64_t)p.inter * 4;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int r = wm * 64 + m * 16 + (lane & 15);
    if (r >= t.rows) continue;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int col = n0 + wn * 64 + n * 16 + (lane >> 4) * 4;
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = INT8 ? acc[m][n][i] * half_at(down_scale, col + i) : acc[m][n][i];
      store4(out + (int64_t)(t.row0 + r) * p.hidden + col, v);
    }
  }
}

// ---- columns x columns: gradients of the weights --------------------------------------------------------------
__global__ __launch_bounds__(kBlock) void weights_kernel(const ExpertRowsParams p, const uint16_t *xs, const uint16_t *dys, const uint16_t *h,
                                                         const uint16_t *dgu, uint8_t *dblobs) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][kTileBytes];
  const int pitch = expert_rows_pitch(p.inter), n_n = p.hidden / kTile, n_m = (p.inter + kTile - 1) / kTile;
  int i0 = blockIdx.x;
  const int n0 = i0 % n_n * kTile;
  i0 /= n_n;
  const int m0 = i0 % n_m * kTile;
  i0 /= n_m;
  const int which = i0 % 3, e = i0 / 3;
  const int row0 = uniform(min(max(p.offsets[e], 0), p.n_rows)), rows = uniform(max(min(p.offsets[e + 1], p.n_rows) - row0, 0));
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
  const uint16_t *a_in = which == 2 ? h : dgu + which * pitch, *b_in = which == 2 ? dys : xs;
  const int a_pitch = which == 2 ? pitch : 2 * pitch;
  uint32_t a_off[4], b_off[4];
  const uint32_t a_bytes = (uint32_t)a_pitch * 2, b_bytes = (uint32_t)p.hidden * 2;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = (wave * 4 + i) * 4 + lane / 16, col = ((((lane & 15) >> 1) ^ swap16(k)) * 2 + (lane & 1)) * 16;
    a_off[i] = (uint32_t)k * a_bytes + col;
    b_off[i] = (uint32_t)k * b_bytes + col;
  }
  const int steps = (rows + 63) / 64;
  const auto stage = [&](int buf, int s) {
    const int64_t r = row0 + s * 64;
    const int n = min(64, rows - s * 64);
    // (the rest of a row behind the tile's columns belongs to the resource; rows behind the expert's do not)
    const Buffer a = buffer_of(a_in + r * a_pitch + m0, n * a_bytes - (m0 + (which == 1 ? pitch : 0)) * 2),
                 b = buffer_of(b_in + r * p.hidden + n0, n * b_bytes - n0 * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to_lds(a, a_off[i], 0, &lds[buf][0][(wave * 4 + i) * 1024]);
      to_lds(b, b_off[i], 0, &lds[buf][1][(wave * 4 + i) * 1024]);
    }
  };
  f32x4 acc[4][4];
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int n = 0; n < 4; ++n) acc[m][n] = f32x4{};
  if (steps > 0) stage(0, 0);
  for (int s = 0; s < steps; ++s) {
    wait_loads_and_meet();
    if (s + 1 < steps) stage((s + 1) & 1, s + 1);
    const uint8_t *ta = lds[s & 1][0], *tb = lds[s & 1][1];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      i32x4 x[4], w[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) x[m] = fragment_t16(ta, wm * 4 + m, kk * 32, lane);
#pragma unroll
      for (int n = 0; n < 4; ++n) w[n] = fragment_t16(tb, wn * 4 + n, kk * 32, lane);
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = mma(w[n], x[m], acc[m][n]);
    }
  }
  uint16_t *out = reinterpret_cast<uint16_t *>(dblobs + e * p.blob_stride);
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int rec = m0 + wm * 64 + m * 16 + (lane & 15);
    if (rec >= p.inter) continue;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const float v[4] = {acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]};
      store4(out + ((int64_t)rec * 3 + which) * p.hidden + n0 + wn * 64 + n * 16 + (lane >> 4) * 4, v);
    }
  }
}

}  // namespace

hipError_t launch_experts_up(const ExpertRowsParams &p, int weight_fmt, const void *xs, const float *scale, uint16_t *h, uint16_t *gu,
                             hipStream_t s) {
  const dim3 grid(tile_grid(p, expert_rows_pitch(p.inter) / 64, false));
  const uint8_t *x = static_cast<const uint8_t *>(xs);
  if (weight_fmt == MOE_W_INT8_PC)
    hipLaunchKernelGGL((rows_kernel<true, kUp>), grid, dim3(kBlock), 0, s, p, x, scale, (const uint16_t *)nullptr, h, gu);
  else
    hipLaunchKernelGGL((rows_kernel<false, kUp>), grid, dim3(kBlock), 0, s, p, x, scale, (const uint16_t *)nullptr, h, gu);
  return hipGetLastError();
}
hipError_t launch_experts_down(const ExpertRowsParams &p, int weight_fmt, const uint16_t *h, uint16_t *ys, hipStream_t s) {
  const dim3 grid(tile_grid(p, p.hidden / kTile, true));
  const int pitch = expert_rows_pitch(p.inter);
  if (weight_fmt == MOE_W_INT8_PC)
    hipLaunchKernelGGL((columns_kernel<true>), grid, dim3(kBlock), 0, s, p, h, pitch, 1, 2, ys);
  else
    hipLaunchKernelGGL((columns_kernel<false>), grid, dim3(kBlock), 0, s, p, h, pitch, 1, 2, ys);
  return hipGetLastError();
}
hipError_t launch_experts_dgu(const ExpertRowsParams &p, const uint16_t *dys, const uint16_t *gu, uint16_t *dgu, hipStream_t s) {
  const dim3 grid(tile_grid(p, (expert_rows_pitch(p.inter) + 127) / 128, false));
  hipLaunchKernelGGL((rows_kernel<false, kDgu>), grid, dim3(kBlock), 0, s, p, reinterpret_cast<const uint8_t *>(dys), (const float *)nullptr, gu,
                     (uint16_t *)nullptr, dgu);
  return hipGetLastError();
}
hipError_t launch_experts_dx(const ExpertRowsParams &p, const uint16_t *dgu, uint16_t *dxs, hipStream_t s) {
  const dim3 grid(tile_grid(p, p.hidden / kTile, true));
  hipLaunchKernelGGL((columns_kernel<false>), grid, dim3(kBlock), 0, s, p, dgu, 2 * expert_rows_pitch(p.inter), 2, 0, dxs);
  return hipGetLastError();
}
hipError_t launch_experts_dw(const ExpertRowsParams &p, const uint16_t *xs, const uint16_t *dys, const uint16_t *h, const uint16_t *dgu,
                             uint8_t *dblobs, hipStream_t s) {
  const dim3 grid(p.n_experts * 3 * ((p.inter + kTile - 1) / kTile) * (p.hidden / kTile));
  hipLaunchKernelGGL(weights_kernel, grid, dim3(kBlock), 0, s, p, xs, dys, h, dgu, dblobs);
  return hipGetLastError();
}

}  // namespace moe
