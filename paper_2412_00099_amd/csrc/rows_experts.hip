// SwiGLU experts on rows sorted by expert, straight on the blobs (record i = gate row i | up row i | column i of down, d weights
// each), and their gradients.  Expert e takes rows offsets[e] .. offsets[e+1]:
//
//   G = X Wg^T, U = X Wu^T, H = silu(G) U, Y = H Wd^T
//   dH = dY Wd, dG = dH U s (1 + G (1 - s)), dU = dH G s (s = sigmoid G), dX = dG Wg + dU Wu
//   dWg = dG^T X, dWu = dU^T X, dWd^T = H^T dY
//
// Three forms of product, all on the matrix cores with sums in 32 bits:
//   kUp, kDgu   both operands have the summed index side by side (X with gate / up rows, dY with down columns)
//   kColumns    the summed index are the records (H with down, dG and dU with gate and up): the weights' side is transposed on
//               its way out of LDS
//   kWeights    the summed index are the rows: both sides are transposed
// H and the gradients of G and U pass through memory rounded to bf16, as the rows do; G and U themselves are kept for the
// backward in 32 bits (rounded to bf16 they were the largest part of the gradients' error).  With 8-bit weights the rows of the
// first product are 8-bit codes too (whole-number sums, exact), H stays bf16 and the weights of down are widened to bf16, which
// holds every code exactly.
//
// A workgroup of eight wavefronts has a compute unit to itself and walks over tiles of up to 256 x 256, a wavefront 128 x 64 of
// it.  The summed index goes through LDS in stages of 64 (8-bit: 128) values, whole 128-byte lines, filled by loads that bypass
// the registers: two stages of the rows' side, which other workgroups of the XCD read too, and three of the weights' side, which
// comes from memory.  A stage is two steps of the matrix cores; the fragments of the next step are read while they work on this
// one's, and there is one barrier a stage.  The next tile's first stages are requested ahead of the results' stores.
//
// Which expert and which of its rows a tile has is worked out from `offsets` on the device.  All loads go through buffer
// resources that end where the expert's rows or records end: what lies beyond arrives as zeros.
#include "rows.h"

namespace moe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __amdgpu_buffer_rsrc_t Buffer;
#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T *)(p))

constexpr int kCols = 256;        // columns of a tile (128 records where each has two products)
constexpr int kMaxBlocks = 8;     // 32-row blocks of a tile at most
constexpr int kWavesWg = 8, kBlock = kWavesWg * 64;
constexpr int kStageBytes = 32768;                 // of one side
constexpr int kRowStages = 2, kWeightStages = 3;   // 160 KB, all of a compute unit's LDS
constexpr uint32_t kWeightBase = kRowStages * kStageBytes, kLdsBytes = (kRowStages + kWeightStages) * kStageBytes;

enum { kUp = 0, kDgu = 1, kColumns = 2, kWeights = 3 };

struct ProductArgs {
  ExpertRowsParams p;
  const uint8_t *a;    // rows' side: xs, dys, h or dgu
  const uint8_t *b;    // kWeights: xs
  const uint8_t *a2, *b2;  // kWeights: h and dys
  const float *scale;  // 8-bit rows
  const float *gu_in;  // kDgu
  uint16_t *out;       // kUp: h; kDgu: dgu; kColumns: ys or dxs
  float *gu_out;       // kUp: or nullptr
  uint8_t *dblobs;     // kWeights
  int32_t a_pitch;     // kColumns: elements of a row of a
  int32_t sections, first;  // kColumns: out = sum over s < sections of columns s * pitch .. of a times part first + s of the records
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ Buffer buffer_of(const void *base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}
// 16 bytes per lane straight into LDS, lane after lane from `lds` (the same in every lane)
__device__ __forceinline__ void to_lds(Buffer b, uint32_t off, uint32_t at, uint8_t *lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b, LDS_PTR(void, lds), 16, off, at, 0, 0);
}
// all but the last N loads of each wavefront of the workgroup have landed, and the reads of LDS that they have issued are done
template <int N>
__device__ __forceinline__ void landed_but() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// the reads of LDS that the workgroup has issued are done
__device__ __forceinline__ void everybody_has_read() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x4 mma(i32x4 a, i32x4 b, i32x4 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// ---- tiles ------------------------------------------------------------------------------------------------
struct Tile {
  int expert;  // -1: no tile
  int row0, rows;
  int col;
};
__device__ __forceinline__ int first_row(const ExpertRowsParams &p, int e) { return min(max(p.offsets[e], 0), p.n_rows); }
__device__ __forceinline__ int row_count(const ExpertRowsParams &p, int e) { return max(min(p.offsets[e + 1], p.n_rows) - first_row(p, e), 0); }
__device__ __forceinline__ int wave_total(int v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  return uniform(v);
}

// An expert's rows are cut into the fewest parts of at most `blocks` 32-row blocks, all of nearly the same size.  `blocks` is
// the size from 4 to 8 for which the launch's rounds of one tile a workgroup take the least time: a tile costs its rows and, for
// the weights that have to come in whatever its rows are, about 64 more.
struct TilePlan {
  int blocks, total;
};
__device__ __forceinline__ TilePlan plan_tiles(const ExpertRowsParams &p, int n_cols, int workgroups) {
  const int lane = threadIdx.x & 63;
  int n[5] = {};
  for (int e = lane; e < p.n_experts; e += 64) {
    const int c = row_count(p, e);
#pragma unroll
    for (int i = 0; i < 5; ++i) n[i] += (c + (4 + i) * 32 - 1) / ((4 + i) * 32);
  }
  TilePlan best{8, 0};
  int64_t least = INT64_MAX;
#pragma unroll
  for (int i = 4; i >= 0; --i) {
    const int total = wave_total(n[i]) * n_cols;
    const int64_t cost = (int64_t)((total + workgroups - 1) / workgroups) * ((4 + i) * 32 + 64);
    if (cost < least) {
      least = cost;
      best.blocks = 4 + i;
      best.total = total;
    }
  }
  return best;
}
// Tiles in the order expert, column, row, so that the workgroups that share weights are neighbours; the list is dealt to the
// eight XCDs in eight parts, since workgroups go to them in turn and each has an L2 of its own.
__device__ __forceinline__ Tile find_tile(const ExpertRowsParams &p, const TilePlan &plan, int n_cols, int in_part, int xcd) {
  const int lane = threadIdx.x & 63;
  Tile r{-1, 0, 0, 0};
  const int part = (plan.total + 7) / 8, want = xcd * part + in_part;
  if (in_part >= part || want >= plan.total) return r;
  int before = 0;
  const int most = plan.blocks * 32;
  for (int e0 = 0; e0 < p.n_experts; e0 += 64) {
    const int e = e0 + lane, c = e < p.n_experts ? row_count(p, e) : 0;
    const int parts = (c + most - 1) / most, t = parts * n_cols;
    int upto = t;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o);
      if (lane >= o) upto += y;
    }
    const uint64_t past = __ballot(before + upto > want);
    if (past != 0) {
      const int l = uniform(__ffsll((unsigned long long)past) - 1);
      const int left = want - before - uniform(__shfl(upto - t, l)), count = uniform(__shfl(c, l)), of = uniform(__shfl(parts, l));
      r.expert = e0 + l;
      r.col = left / of;
      const int each = ((count + of - 1) / of + 15) / 16 * 16, at = (left - r.col * of) * each;
      r.row0 = first_row(p, r.expert) + at;
      r.rows = max(min(each, count - at), 0);
      return r;
    }
    before += uniform(__shfl(upto, 63));
  }
  return r;
}

// (in scalar registers: a tile makes buffer resources and decides what is done)
__device__ __forceinline__ Tile uniform_tile(const Tile &t) { return Tile{uniform(t.expert), uniform(t.row0), uniform(t.rows), uniform(t.col)}; }

// ---- LDS images -------------------------------------------------------------------------------------------
// Side by side: 256 rows of 128 bytes, eight 16-byte chunks, the first four for the stage's first step.  Chunk c of row r lies at
// c ^ f(r).  A fragment's lanes read 16 bytes of 16 rows each, in four turns; a turn takes four lanes each of four groups: rows
// 0-3 and 12-15 at one chunk and rows 4-11 at its neighbour, or the other way round.  f spreads both kinds over all banks, where a
// fragment has 16 rows in a row and where it has 4 of each 8.
__device__ __forceinline__ int swap_rows(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int swap_fours(int r) { return ((r >> 1) & 1) | ((r >> 2) & 6); }
// Transposed, 16-bit: 64 rows (the summed index) of 256 columns, 512 bytes.  Where a fragment has 16 columns in a row, their 32
// bytes (group g) lie at g ^ swap16(k); where it has 4 of each 8, 64 bytes (group g) lie at g ^ k % 4.
__device__ __forceinline__ int swap16(int k) { return (k & 3) | ((k >> 1) & 4); }
// Results: register i of a lane is column (lane / 16) * 4 + i of a fragment.  With PAIRED fragments j and j + 1 have 4 columns
// of each 8 in turn, so that a lane has 8 columns in a row and stores 16 bytes.
__device__ __forceinline__ i32x4 transposed(const uint8_t *at) {  // 8 summed values of the lane's column: rows of `at` and + 4
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + 4 * 512));
  return __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// 8 codes q + 128 as bf16 (whole numbers up to 128: the lower halves of the floats are zero)
__device__ __forceinline__ i32x4 widen(i32x2 q) {
  i32x4 v;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int u = q[w] ^ (int)0x80808080;
    const float f0 = (float)(int8_t)u, f1 = (float)(int8_t)(u >> 8), f2 = (float)(int8_t)(u >> 16), f3 = (float)(u >> 24);
    v[2 * w] = (int)__builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302);
    v[2 * w + 1] = (int)__builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302);
  }
  return v;
}

// Results go through buffer resources too: rows that the tile does not have lie behind their end and are dropped, so that no
// lane branches (a branch that differs between lanes would take the loops around it out of scalar control).
constexpr uint32_t kNowhere = 0xf8000000u;
__device__ __forceinline__ void store8(Buffer p, uint32_t off, const float (&v)[8]) {
  rows_u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
  __builtin_amdgcn_raw_buffer_store_b128(w, p, off, 0, 0);
}
__device__ __forceinline__ void store8_f32(Buffer p, uint32_t off, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    rows_u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[4 * h + i]);
    __builtin_amdgcn_raw_buffer_store_b128(w, p, off + 16 * h, 0, 0);
  }
}
__device__ __forceinline__ void load8_f32(Buffer p, uint32_t off, float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const rows_u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(p, off + 16 * h, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * h + i] = __uint_as_float(w[i]);
  }
}
__device__ __forceinline__ void store4(Buffer p, uint32_t off, const float (&v)[4]) {
  rows_u32x2 w;
  w[0] = pack_bf16(v[0], v[1]);
  w[1] = pack_bf16(v[2], v[3]);
  __builtin_amdgcn_raw_buffer_store_b64(w, p, off, 0, 0);
}
__device__ __forceinline__ float half_lo(uint32_t v) { return (float)__builtin_bit_cast(_Float16, (uint16_t)v); }
__device__ __forceinline__ float half_hi(uint32_t v) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(v >> 16)); }
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }

// ---- one tile ---------------------------------------------------------------------------------------------
template <int FORM, bool INT8>
struct Product {
  static constexpr int EL = INT8 ? 1 : 2;
  static constexpr bool NARROW = FORM == kColumns && INT8;       // the weights' stage is of bytes: half as long
  static constexpr int A_LOADS = 4, B_LOADS = NARROW ? 2 : 4;  // of a wavefront for a stage
  using Acc = std::conditional_t<INT8 && FORM == kUp, i32x4, f32x4>;

  const ProductArgs g;  // (a copy: through a reference the arguments would not be known to be the same in every lane)
  uint8_t *lds;
  int lane, wave, wm, wn, pitch;
  uint32_t row_bytes;
  // the tile whose loads are being issued
  Buffer a, b;
  // the lane's place in loads 0 and 1; 2 and 3 are a_more, b_more behind them (side by side the weights' are exchanged otherwise)
  static constexpr bool SIDE = FORM == kUp || FORM == kDgu;
  uint32_t a_off[2], b_off[SIDE ? 4 : 2];
  uint32_t a_more, b_more;
  int stages;
  // the stages that are requested next: their places and where their operands are
  uint32_t a_put, b_put, a_at, b_at;
  int section_left;                              // kColumns: stages of the first section to come
  const uint8_t *a_base, *b_base;                // kWeights
  uint32_t a_row, b_row, a_skip, b_skip;
  int a_rows_left, b_rows_left;

  __device__ __forceinline__ Product(const ProductArgs &args, uint8_t *l) : g(args), lds(l) {
    lane = threadIdx.x & 63;
    wave = uniform(threadIdx.x >> 6);
    wm = wave >> 2;
    wn = wave & 3;
    pitch = expert_rows_pitch(g.p.inter);
    row_bytes = (uint32_t)g.p.hidden * EL;
  }

  __device__ __forceinline__ void open(const Tile &t) {
    const ExpertRowsParams &p = g.p;
    a_put = a_at = b_at = 0;
    b_put = kWeightBase;
    if constexpr (FORM == kWeights) {
      // t.col: columns of the gradient; t.row0, t.rows: its rows, 2 * pitch of gate and up, then pitch of down
      const bool down = t.row0 >= 2 * pitch;
      const int m0 = down ? t.row0 - 2 * pitch : t.row0, row0 = uniform(first_row(p, t.expert));
      a_rows_left = b_rows_left = uniform(row_count(p, t.expert));
      stages = (a_rows_left + 63) / 64;
      a_row = (down ? pitch : 2 * pitch) * 2;
      b_row = row_bytes;
      a_skip = m0 * 2;
      b_skip = t.col * kCols * 2;
      a_base = (down ? g.a2 : g.a) + (int64_t)row0 * a_row + a_skip;
      b_base = (down ? g.b2 : g.b) + (int64_t)row0 * b_row + b_skip;
      a_more = 4 * a_row;
      b_more = 4 * b_row;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = (wave * 4 + i) * 2 + lane / 32, pos = lane & 31;
        a_off[i] = k * a_row + (pos ^ (swap16(k) << 1)) * 16;
        b_off[i] = k * b_row + (pos ^ ((k & 3) << 2)) * 16;
      }
    } else {
      const uint32_t rec_bytes = 3 * row_bytes, a_bytes = FORM == kColumns ? (uint32_t)g.a_pitch * 2 : row_bytes;
      a = buffer_of(g.a + (int64_t)t.row0 * a_bytes, t.rows * a_bytes);
      b = buffer_of(p.blobs + t.expert * p.blob_stride, (uint32_t)p.inter * rec_bytes);
      a_more = 16 * a_bytes;
      b_more = 4 * rec_bytes;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = (wave * 4 + i) * 8 + lane / 8;
        a_off[i] = (uint32_t)r * a_bytes + ((lane & 7) ^ swap_rows(r)) * 16;
        if constexpr (NARROW) {
          const int k = (wave * 2 + i) * 4 + lane / 16;
          b_off[i] = (uint32_t)k * rec_bytes + t.col * kCols + ((lane & 15) ^ (k & 15)) * 16;
        } else if constexpr (FORM == kColumns) {
          const int k = (wave * 4 + i) * 2 + lane / 32;
          b_off[i] = (uint32_t)k * rec_bytes + t.col * kCols * 2 + ((lane & 31) ^ (swap16(k) << 1)) * 16;
        }
      }
      if constexpr (SIDE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // kUp: of each 64 rows the first 32 are gate rows, the others the same records' up rows.  (A record that is not there
          // lies behind the end of the resource.)
          const int r = (wave * 4 + i) * 8 + lane / 8;
          const int rec = FORM == kUp ? t.col * 128 + (r >> 6) * 32 + (r & 31) : t.col * kCols + r, which = FORM == kUp ? (r >> 5) & 1 : 2;
          b_off[i] = (uint32_t)(rec * 3 + which) * row_bytes + ((lane & 7) ^ swap_fours(r)) * 16;
        }
      }
      if constexpr (FORM == kColumns) b_at = g.first * row_bytes;
      section_left = pitch / 64;
      stages = FORM == kColumns ? section_left * g.sections : row_bytes / 128;
    }
  }

  // Requests the next stage of a side (behind a tile's last one: what comes next in memory, or zeros).
  __device__ __forceinline__ void request_rows() {
    uint8_t *at = lds + a_put + wave * 4096;
    if constexpr (FORM == kWeights) {
      const int n = max(min(64, a_rows_left), 0);
      a = buffer_of(a_base, n > 0 ? n * a_row - a_skip : 0);
    }
#pragma unroll
    for (int i = 0; i < A_LOADS; ++i) to_lds(a, a_off[i & 1], (FORM == kWeights ? 0 : a_at) + (i >> 1) * a_more, at + i * 1024);
    next_rows();
  }
  __device__ __forceinline__ void request_weights() {
    uint8_t *at = lds + b_put + wave * (NARROW ? 2048 : 4096);
    if constexpr (FORM == kWeights) {
      const int n = max(min(64, b_rows_left), 0);
      b = buffer_of(b_base, n > 0 ? n * b_row - b_skip : 0);
    }
#pragma unroll
    for (int i = 0; i < B_LOADS; ++i) to_lds(b, b_off[SIDE ? i : i & 1], (FORM == kWeights ? 0 : b_at) + (SIDE ? 0 : (i >> 1) * b_more), at + i * 1024);
    next_weights();
  }
  __device__ __forceinline__ void next_rows() {
    a_put = next_row_stage(a_put);
    if constexpr (FORM == kWeights) {
      a_rows_left -= 64;
      a_base += 64 * a_row;
    } else {
      a_at += 128;
    }
  }
  __device__ __forceinline__ void next_weights() {
    b_put = next_weight_stage(b_put);
    if constexpr (FORM == kWeights) {
      b_rows_left -= 64;
      b_base += 64 * b_row;
    } else if constexpr (FORM == kColumns) {
      // (behind the last record: outside of the resource)
      b_at += 64 * 3 * row_bytes;
      if (--section_left == 0) b_at = (g.first + 1) * row_bytes;
    } else {
      b_at += 128;
    }
  }
  static __device__ __forceinline__ uint32_t next_row_stage(uint32_t at) { return kStageBytes - at; }
  static __device__ __forceinline__ uint32_t next_weight_stage(uint32_t at) { return at == kLdsBytes - kStageBytes ? kWeightBase : at + kStageBytes; }
  // the first stages of a tile; nobody reads LDS any more
  __device__ __forceinline__ void request_first() {
    request_rows();
    request_weights();
    request_rows();
    request_weights();
    request_weights();
  }
  // as request_first leaves it, for the tile that it was called for
  __device__ __forceinline__ void skip_first() {
    next_rows();
    next_rows();
    next_weights();
    next_weights();
    next_weights();
  }

  // Where the lane's fragments lie in a stage: of the weights for each j, of the rows for block 0; of the stage's first step.
  __device__ __forceinline__ void fragment_offsets(uint32_t (&w_at)[4], uint32_t &x_at) const {
    const int l = lane & 15, q = lane >> 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (FORM == kWeights) {
        const int k = q * 8 + (l >> 2), chunk = wn * 8 + (j >> 1) * 4 + (l & 3);
        w_at[j] = k * 512 + ((chunk ^ ((k & 3) << 2)) * 16) + (j & 1) * 8;
      } else if constexpr (NARROW) {
        const int k = q * 8 + (l >> 1);
        w_at[j] = k * 256 + (((wn * 4 + j) ^ (k & 15)) * 16) + (l & 1) * 8;
      } else if constexpr (FORM == kColumns) {
        const int k = q * 8 + (l >> 2);
        w_at[j] = k * 512 + (((wn * 4 + j) ^ swap16(k)) * 32) + (l & 3) * 8;
      } else {
        // kUp: fragments 0, 2 are gate rows, 1, 3 up rows
        const int four = FORM == kUp ? j >> 1 : j & 1, half = FORM == kUp ? j & 1 : j >> 1;
        const int r = wn * 64 + half * 32 + (l >> 2) * 8 + four * 4 + (l & 3);
        w_at[j] = r * 128 + ((q ^ swap_fours(r)) * 16);
      }
    }
    if constexpr (FORM == kWeights) {
      const int k = q * 8 + (l >> 2);
      x_at = k * 512 + ((wm ^ swap16(k)) * 32) + (l & 3) * 8;
    } else {
      const int r = wm * 16 + l;
      x_at = r * 128 + ((q ^ swap_rows(r)) * 16);
    }
  }
  // second: of the stage's second step
  __device__ __forceinline__ i32x4 read_w(uint32_t w_at, uint32_t stage, bool second) const {
    if constexpr (NARROW) {
      return widen(__builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(i32x2, lds + stage + w_at + (second ? 32 * 256 : 0))));
    } else if constexpr (FORM == kWeights || FORM == kColumns) {
      return transposed(lds + stage + w_at + (second ? 32 * 512 : 0));
    } else {
      i32x4 w = *reinterpret_cast<const i32x4 *>(lds + stage + (w_at ^ (second ? 64 : 0)));
      if constexpr (INT8) w ^= (int)0x80808080;
      return w;
    }
  }
  // block m (transposed, the block is part of what was exchanged: see swap16)
  __device__ __forceinline__ i32x4 read_x(uint32_t x_at, uint32_t stage, bool second, int m) const {
    if constexpr (FORM == kWeights) return transposed(lds + stage + (x_at ^ (m * 64)) + (second ? 32 * 512 : 0));
    else return *reinterpret_cast<const i32x4 *>(lds + stage + (x_at ^ (second ? 64 : 0)) + m * 4096);
  }

  // the product of the tile that is open; then `next` opens the next one, and the results are stored
  template <typename Next>
  __device__ __forceinline__ void run(const Tile &t, Next next) {
    const int blocks = (t.rows + 31) / 32;  // of 32 rows; a wavefront has half of each
    Acc acc[kMaxBlocks][4];
#pragma unroll
    for (int m = 0; m < kMaxBlocks; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[m][j] = Acc{};
    i32x4 x[kMaxBlocks], w0[4], w1[4];
    uint32_t w_at[4], x_at, rows_stage = 0, weights_stage = kWeightBase;  // the stages whose fragments are read
    fragment_offsets(w_at, x_at);
    // A step reads the fragments of the next one, a block's once the block of this step has gone to the matrix cores.  Blocks that
    // the tile does not have are jumped over.
    const auto step = [&](i32x4 (&now)[4], i32x4 (&then)[4], bool second) MOE_ROWS_INLINE {
#pragma unroll
      for (int j = 0; j < 4; ++j) then[j] = read_w(w_at[j], weights_stage, second);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < kMaxBlocks; ++m) {
        if (m > 0 && m >= blocks) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][j] = mma(now[j], x[m], acc[m][j]);
        x[m] = read_x(x_at, rows_stage, second, m);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (stages > 0) {
      landed_but<A_LOADS + 2 * B_LOADS>();
#pragma unroll
      for (int j = 0; j < 4; ++j) w0[j] = read_w(w_at[j], weights_stage, false);
#pragma unroll
      for (int m = 0; m < kMaxBlocks; ++m) x[m] = read_x(x_at, rows_stage, false, m);
      for (int left = stages; left > 0; --left) {
        step(w0, w1, true);
        // Everybody has read all of this stage: its places are free.  The next one has landed when no more than the weights of
        // the one behind it are outstanding.  (Behind the last stage what is requested and read is not used.)
        landed_but<B_LOADS>();
        request_rows();
        request_weights();
        rows_stage = next_row_stage(rows_stage);
        weights_stage = next_weight_stage(weights_stage);
        step(w1, w0, false);
      }
    }
    everybody_has_read();
    next();
    store(t, acc, blocks);
  }

  // lane: row lane % 16 of each block of 16 rows; columns as said at the LDS images
  __device__ __forceinline__ void store(const Tile &t, const Acc (&acc)[kMaxBlocks][4], int blocks) const {
    const ExpertRowsParams &p = g.p;
    const int q = lane >> 4, r0 = wm * 16 + (lane & 15);
    const uint8_t *blob = p.blobs + t.expert * p.blob_stride;
    const int64_t tail = (int64_t)p.inter * 3 * row_bytes;
    if constexpr (FORM == kUp) {
      const int rec = t.col * 128 + wn * 32 + q * 8;
      const Buffer h = buffer_of(g.out + (int64_t)t.row0 * pitch, t.rows * pitch * 2);
      const Buffer both = buffer_of(g.gu_out + (int64_t)t.row0 * 2 * pitch, g.gu_out ? t.rows * 2 * pitch * 4 : 0);
      float sg[8], su[8];
      if constexpr (INT8) {
        const Buffer scales = buffer_of(blob + tail, p.inter * 4);
        const rows_u32x4 vg = __builtin_amdgcn_raw_buffer_load_b128(scales, rec < p.inter ? rec * 2 : kNowhere, 0, 0),
                         vu = __builtin_amdgcn_raw_buffer_load_b128(scales, rec < p.inter ? (p.inter + rec) * 2 : kNowhere, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sg[2 * i] = half_lo(vg[i]);
          sg[2 * i + 1] = half_hi(vg[i]);
          su[2 * i] = half_lo(vu[i]);
          su[2 * i + 1] = half_hi(vu[i]);
        }
      }
      const Buffer row_scale = buffer_of(g.scale + t.row0, INT8 ? t.rows * 4 : 0);
#pragma unroll
      for (int m = 0; m < kMaxBlocks; ++m) {
        if (m > 0 && m >= blocks) break;
        const uint32_t r = r0 + m * 32;
        const float sx = INT8 ? __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(row_scale, r * 4, 0, 0)) : 1.f;
        float v[8], gate[8], up[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          gate[i] = (float)acc[m][(i >> 2) * 2][i & 3];
          up[i] = (float)acc[m][(i >> 2) * 2 + 1][i & 3];
          if constexpr (INT8) {
            gate[i] *= sx * sg[i];
            up[i] *= sx * su[i];
          }
          v[i] = gate[i] * sigmoid(gate[i]) * up[i];
        }
        store8(h, rec < pitch ? (r * pitch + rec) * 2 : kNowhere, v);
        if (g.gu_out) {
          const uint32_t at = rec < pitch ? (r * 2 * pitch + rec) * 4 : kNowhere;
          store8_f32(both, at, gate);
          store8_f32(both, at + pitch * 4, up);
        }
      }
    } else if constexpr (FORM == kDgu) {
      const Buffer in = buffer_of(g.gu_in + (int64_t)t.row0 * 2 * pitch, t.rows * 2 * pitch * 4),
                   out = buffer_of(g.out + (int64_t)t.row0 * 2 * pitch, t.rows * 2 * pitch * 2);
#pragma unroll
      for (int m = 0; m < kMaxBlocks; ++m) {
        if (m > 0 && m >= blocks) break;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int rec = t.col * kCols + wn * 64 + h * 32 + q * 8;
          const uint32_t at = rec < pitch ? (r0 + m * 32) * 2 * pitch + rec : kNowhere / 4;
          float gate[8], up[8];
          load8_f32(in, at * 4, gate);
          load8_f32(in, (at + pitch) * 4, up);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float s = sigmoid(gate[i]), dh = acc[m][h * 2 + (i >> 2)][i & 3], x = gate[i];
            gate[i] = dh * up[i] * (s * (1.f + x * (1.f - s)));
            up[i] = dh * (x * s);
          }
          // (behind the last record: both resources end before kNowhere / 2)
          store8(out, at * 2, gate);
          store8(out, (at + pitch) * 2, up);
        }
      }
    } else if constexpr (FORM == kColumns) {
      const Buffer out = buffer_of(g.out + (int64_t)t.row0 * p.hidden, t.rows * p.hidden * 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = t.col * kCols + wn * 64 + j * 16 + q * 4;
        float sd[4];
        if constexpr (INT8) {
          const rows_u32x2 w = *reinterpret_cast<const rows_u32x2 *>(blob + tail + (int64_t)p.inter * 4 + col * 2);
          sd[0] = half_lo(w[0]);
          sd[1] = half_hi(w[0]);
          sd[2] = half_lo(w[1]);
          sd[3] = half_hi(w[1]);
        }
#pragma unroll
        for (int m = 0; m < kMaxBlocks; ++m) {
          if (m > 0 && m >= blocks) break;
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = INT8 ? acc[m][j][i] * sd[i] : acc[m][j][i];
          store4(out, ((r0 + m * 32) * p.hidden + col) * 2, v);
        }
      }
    } else {
      const Buffer out = buffer_of(g.dblobs + t.expert * p.blob_stride, (uint32_t)tail);
#pragma unroll
      for (int m = 0; m < kMaxBlocks; ++m) {
        if (m > 0 && m >= blocks) break;
        const int r = r0 + m * 32, at = t.row0 + r, which = at >= 2 * pitch ? 2 : at >= pitch ? 1 : 0, rec = at - which * pitch;
        // (a record that is not there lies behind the end)
        const uint32_t to = r < t.rows ? ((rec * 3 + which) * p.hidden + t.col * kCols + wn * 64 + q * 8) * 2 : kNowhere;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = acc[m][h * 2 + (i >> 2)][i & 3];
          store8(out, to + h * 64, v);
        }
      }
    }
  }
};

template <int FORM, bool INT8>
__global__ __launch_bounds__(kBlock, 2) void product_kernel(const ProductArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes];
  Product<FORM, INT8> f(g, lds);
  const ExpertRowsParams &p = g.p;
  const int workgroups = gridDim.x, per_xcd = workgroups / 8, xcd = blockIdx.x & 7;
  const int n_cols = FORM == kUp ? (f.pitch + 127) / 128 : FORM == kDgu ? (f.pitch + kCols - 1) / kCols : p.hidden / kCols;
  // kWeights: 2 * pitch rows of gate and up gradients, then pitch of down
  const int m_both = (2 * f.pitch + 255) / 256, m_tiles = m_both + (f.pitch + 255) / 256;
  TilePlan plan{8, p.n_experts * m_tiles * n_cols};
  if constexpr (FORM != kWeights) plan = plan_tiles(p, n_cols, workgroups);
  const auto tile = [&](int i) MOE_ROWS_INLINE {
    if constexpr (FORM == kWeights) {
      Tile r{-1, 0, 0, 0};
      const int part = (plan.total + 7) / 8, want = xcd * part + i;
      if (i >= part || want >= plan.total) return r;
      r.col = want % n_cols;
      const int m = want / n_cols, at = m % m_tiles;
      r.expert = m / m_tiles;
      r.row0 = at < m_both ? at * 256 : 2 * f.pitch + (at - m_both) * 256;
      r.rows = min(256, (at < m_both ? 2 : 3) * f.pitch - r.row0);
      return r;
    } else {
      return find_tile(p, plan, n_cols, i, xcd);
    }
  };
  int i = blockIdx.x >> 3;
  Tile now = uniform_tile(tile(i));
  if (now.expert >= 0) {
    f.open(now);
    f.request_first();
  }
  if constexpr (FORM == kColumns) {  // rows of nobody
    const int used = uniform(min(max(p.offsets[p.n_experts], 0), p.n_rows));
    for (int64_t r = used + blockIdx.x; r < p.n_rows; r += workgroups)
      for (int c = threadIdx.x * 8; c < p.hidden; c += kBlock * 8) *reinterpret_cast<rows_u32x4 *>(g.out + r * p.hidden + c) = rows_u32x4{};
  }
  while (now.expert >= 0) {
    // (once more: carried over from the end of the last turn, the buffers would not be known to be the same in every lane)
    f.open(now);
    f.skip_first();
    i += per_xcd;
    const Tile next = uniform_tile(tile(i));
    const auto open_next = [&]() MOE_ROWS_INLINE {
      if (next.expert < 0) return;
      f.open(next);
      f.request_first();
    };
    f.run(now, open_next);
    now = uniform_tile(next);
  }
}

template <int FORM, bool INT8>
hipError_t launch_product(const ProductArgs &g, int n_cus, hipStream_t s) {
  // one workgroup a compute unit, in whole eights
  hipLaunchKernelGGL((product_kernel<FORM, INT8>), dim3(n_cus / 8 * 8), dim3(kBlock), 0, s, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_experts_up(const ExpertRowsParams &p, int weight_fmt, const void *xs, const float *scale, uint16_t *h, float *gu, int n_cus,
                             hipStream_t s) {
  ProductArgs g{};
  g.p = p;
  g.a = static_cast<const uint8_t *>(xs);
  g.scale = scale;
  g.out = h;
  g.gu_out = gu;
  return weight_fmt == MOE_W_INT8_PC ? launch_product<kUp, true>(g, n_cus, s) : launch_product<kUp, false>(g, n_cus, s);
}
hipError_t launch_experts_down(const ExpertRowsParams &p, int weight_fmt, const uint16_t *h, uint16_t *ys, int n_cus, hipStream_t s) {
  ProductArgs g{};
  g.p = p;
  g.a = reinterpret_cast<const uint8_t *>(h);
  g.a_pitch = expert_rows_pitch(p.inter);
  g.sections = 1;
  g.first = 2;
  g.out = ys;
  return weight_fmt == MOE_W_INT8_PC ? launch_product<kColumns, true>(g, n_cus, s) : launch_product<kColumns, false>(g, n_cus, s);
}
hipError_t launch_experts_dgu(const ExpertRowsParams &p, const uint16_t *dys, const float *gu, uint16_t *dgu, int n_cus, hipStream_t s) {
  ProductArgs g{};
  g.p = p;
  g.a = reinterpret_cast<const uint8_t *>(dys);
  g.gu_in = gu;
  g.out = dgu;
  return launch_product<kDgu, false>(g, n_cus, s);
}
hipError_t launch_experts_dx(const ExpertRowsParams &p, const uint16_t *dgu, uint16_t *dxs, int n_cus, hipStream_t s) {
  ProductArgs g{};
  g.p = p;
  g.a = reinterpret_cast<const uint8_t *>(dgu);
  g.a_pitch = 2 * expert_rows_pitch(p.inter);
  g.sections = 2;
  g.first = 0;
  g.out = dxs;
  return launch_product<kColumns, false>(g, n_cus, s);
}
hipError_t launch_experts_dw(const ExpertRowsParams &p, const uint16_t *xs, const uint16_t *dys, const uint16_t *h, const uint16_t *dgu,
                             uint8_t *dblobs, int n_cus, hipStream_t s) {
  ProductArgs g{};
  g.p = p;
  g.a = reinterpret_cast<const uint8_t *>(dgu);
  g.b = reinterpret_cast<const uint8_t *>(xs);
  g.a2 = reinterpret_cast<const uint8_t *>(h);
  g.b2 = reinterpret_cast<const uint8_t *>(dys);
  g.dblobs = dblobs;
  return launch_product<kWeights, false>(g, n_cus, s);
}

}  // namespace moe
