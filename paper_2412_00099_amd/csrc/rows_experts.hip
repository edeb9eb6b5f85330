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
// H and the gradients of G and U pass through memory rounded to bf16, as the rows do: the matrix cores take bf16, and H in
// two or (as the prompt path through the cache has it) three parts of bf16 would double or triple the products over the records and
// the bytes of H.  It makes an error of 0.0023 of the results' size where 32-bit H leaves 0.0017, the rounding of the results
// themselves (8 to 16384 rows).  G and U are kept for the backward in 32 bits (rounded to bf16 they were the largest part of the
// gradients' error).  With 8-bit weights the rows of the
// first product are 8-bit codes too (whole-number sums, exact), H stays bf16 and the weights of down are widened to bf16, which
// holds every code exactly.
//
// A workgroup of eight wavefronts has a compute unit to itself and walks over tiles of up to 256 x 256, a wavefront 128 x 64 of
// it; where experts have fewer rows two workgroups share a compute unit and tiles are 128 x 128 or 64 x 128 (launch_product).  The
// summed index goes through LDS in stages of 64 (8-bit: 128) values, whole 128-byte lines, filled by loads that bypass the
// registers: two stages of the rows' side, which other workgroups of the XCD read too, and three of the weights' side, which
// comes from memory.  A stage is two steps of the matrix cores; the fragments of the next step are read while they work on this
// one's, and there is one barrier a stage.  Both rings run on from tile to tile.
//
// Measured: 8192 rows on 8 experts of 4096 x 14336 in 8 bits, kUp 832 us (2.31 POP/s), kColumns 991 (0.97 PFLOP/s), bound by the matrix
// cores; 16384 uneven rows on 60 experts of 2048 x 1408, kUp with its sums kept 254 us, kColumns 137 (down) and 249 (gradients of the
// rows, 0.74 PFLOP/s), kDgu 187, kWeights 458, bound by workgroups that end early and, where much is stored, by stores; 8 rows on
// 8 of them, 17 + 12 us, 138 MB at 4.8 TB/s, bound by the 176 and 128 tiles that 256 compute units have there.
//
// Which expert and which of its rows a tile has is worked out from `offsets` on the device.  All loads go through buffer
// resources that end where the expert's rows or records end: what lies beyond arrives as zeros.
#include "row_range.h"
#include "rows.h"
#include "tiles.h"

namespace moe {
namespace {

constexpr int kWavesWg = 8, kBlock = kWavesWg * 64;

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

// ---- tiles ------------------------------------------------------------------------------------------------
// kWeights: row0, rows are the expert's, col = tile of the gradient's columns * m_tiles + tile of its rows (the other way round 502 us
// for 482)
struct Tile {
  int expert;  // -1: no tile
  int row0, rows, col;
};
__device__ __forceinline__ int first_row(const ExpertRowsParams &p, int e) { return row_within(p.offsets[e], p.n_rows); }
__device__ __forceinline__ int row_count(const ExpertRowsParams &p, int e) { return row_range(p.offsets[e], p.offsets[e + 1], p.n_rows).count; }

// What an expert's tiles are.  Its rows are cut into the fewest parts of at most MOST, all but the last of the same size, which is
// whole blocks: they are computed whole.  cost: of a tile, in rows; that the weights have to come in costs about as much as 128 rows
// do.  kWeights: the rows in whole stages and 128 for the stores (16384 rows in 60 uneven experts: 541 us, with 64 for them 569,
// with 16 559).
struct ExpertTiles {
  int parts, each, n, cost;
};
template <int FORM, int MOST>
__device__ __forceinline__ ExpertTiles expert_tiles(int count, int n_cols, int m_tiles) {
  ExpertTiles t;
  t.parts = (count + MOST - 1) / MOST;
  t.each = t.parts > 0 ? ((count + t.parts - 1) / t.parts + 31) / 32 * 32 : 0;
  t.n = FORM == kWeights ? m_tiles * n_cols : t.parts * n_cols;
  t.cost = FORM == kWeights ? (count + 63) / 64 * 64 + 128 : t.each + 128;
  return t;
}
// Tiles in the order expert, column, row, so that the workgroups that share weights are neighbours.  The list is cut into eight
// parts of the same cost, one for each XCD: workgroups go to the XCDs in turn and each XCD has an L2 of its own.  Within a part the
// XCD's workgroups take tiles in turn.  The last large tiles, too few for all of them, are cut into pieces of their rows, up to
// one for each workgroup (16384 rows, 60 uneven experts, both products: 448 us, uncut 475; 8192 rows, 8 experts, 8-bit down 1225 and
// 1290).
template <int FORM, int MOST>
constexpr bool in_pieces() {
  return MOST == 256 && FORM != kWeights;
}
struct TileList {
  int next, end, step;  // the workgroup's tiles: next, next + step, .. below end
  int whole, pieces;    // from `whole` on a tile counts as so many, of a part of its rows each
};
// lane i: of expert e0 + i (behind the last one: no tiles)
template <int FORM, int MOST>
__device__ __forceinline__ ExpertTiles lane_expert(const ExpertRowsParams &p, int e0, int n_cols, int m_tiles) {
  const int e = e0 + (threadIdx.x & 63);
  ExpertTiles t = expert_tiles<FORM, MOST>(e < p.n_experts ? row_count(p, e) : 0, n_cols, m_tiles);
  if (e >= p.n_experts) t.n = 0;  // (kWeights has tiles for experts without rows)
  return t;
}
template <int FORM, int MOST>
__device__ __forceinline__ TileList deal_tiles(const ExpertRowsParams &p, int n_cols, int m_tiles) {
  const int xcd = blockIdx.x & 7;
  ExpertTiles t = lane_expert<FORM, MOST>(p, 0, n_cols, m_tiles);
  int64_t upto = sum_upto((int64_t)t.n * t.cost), total = of_lane(upto, 63);  // the cost, up to the lane's expert and of all
  for (int e0 = 64; e0 < p.n_experts; e0 += 64) {
    const ExpertTiles more = lane_expert<FORM, MOST>(p, e0, n_cols, m_tiles);
    total += of_lane(sum_upto((int64_t)more.n * more.cost), 63);
  }
  int begin = -1, end = -1, tiles = 0;
  int64_t before = 0;
  for (int e0 = 0;;) {
    const int past = tiles + sum_upto(t.n);
    // the tile before which a share of the cost is spent, if one of these experts has it
    const auto cut = [&](int64_t share, int &tile) MOE_ROWS_INLINE {
      const uint64_t there = __ballot(share < upto);
      if (share < before || there == 0) return;
      const int l = __builtin_ctzll(there), cost = of_lane(t.cost, l), n = of_lane(t.n, l);
      tile = of_lane(past, l) - n + (int)ceil((double)(share - (of_lane(upto, l) - (int64_t)n * cost)) / (double)cost);
    };
    cut(total * xcd / 8, begin);
    cut(total * (xcd + 1) / 8, end);
    tiles = of_lane(past, 63);
    before = of_lane(upto, 63);
    e0 += 64;
    if (e0 >= p.n_experts) break;
    t = lane_expert<FORM, MOST>(p, e0, n_cols, m_tiles);
    upto = before + sum_upto((int64_t)t.n * t.cost);
  }
  TileList r;
  begin = uniform(begin < 0 ? tiles : begin);
  r.end = uniform(end < 0 ? tiles : end);
  r.step = gridDim.x / 8;
  r.next = begin + (blockIdx.x >> 3);
  r.whole = r.end;
  r.pieces = 1;
  if constexpr (in_pieces<FORM, MOST>()) {
    const int over = max(r.end - begin, 0) % r.step;
    r.whole -= over;
    r.pieces = over > 0 ? r.step / over : 1;
    r.end = r.whole + over * r.pieces;
  }
  return r;
}
// Lane i: tile list.next + i * list.step
template <int FORM, int MOST>
__device__ __forceinline__ Tile lane_tile(const ExpertRowsParams &p, const TileList &list, int n_cols, int m_tiles) {
  const int lane = threadIdx.x & 63;
  const int64_t at = list.next + (int64_t)lane * list.step;
  int want = at < list.end ? (int)at : -1, piece = 0;
  if constexpr (in_pieces<FORM, MOST>()) {
    piece = max(want - list.whole, 0);
    want = min(want, list.whole) + piece / list.pieces;
    piece %= list.pieces;
  }
  Tile r{-1, 0, 0, 0};
  int before = 0;
  for (int e0 = 0; e0 < p.n_experts; e0 += 64) {
    const int e = e0 + lane, row0 = e < p.n_experts ? first_row(p, e) : 0, count = e < p.n_experts ? row_count(p, e) : 0;
    const ExpertTiles t = e < p.n_experts ? expert_tiles<FORM, MOST>(count, n_cols, m_tiles) : ExpertTiles{0, 0, 0, 0};
    const int past = before + sum_upto(t.n);
    // the first expert whose tiles end behind `want`
    int l = 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl(past, l + o - 1) <= want ? o : 0;
    const int of = __shfl(t.parts, l), each = __shfl(t.each, l), rows = __shfl(count, l), from = __shfl(row0, l);
    const int left = want - __shfl(past - t.n, l);
    const int all = of_lane(past, 63);
    if (want >= before && want < all) {
      r.expert = e0 + l;
      if constexpr (FORM == kWeights) {
        r.row0 = from;
        r.rows = rows;
        r.col = left;
      } else {
        r.col = left / of;
        const int at_row = (left - r.col * of) * each;
        r.row0 = from + at_row;
        r.rows = min(each, rows - at_row);
        if constexpr (in_pieces<FORM, MOST>()) {
          if (want >= list.whole) {
            const int part = ((r.rows + list.pieces - 1) / list.pieces + 31) / 32 * 32, skip = part * piece;
            r.row0 += skip;
            r.rows = min(part, r.rows - skip);
            if (r.rows <= 0) r.expert = -1;  // (nothing comes after it)
          }
        }
      }
    }
    before = all;
  }
  return r;
}

// ---- LDS images -------------------------------------------------------------------------------------------
// Side by side: 256 rows of 128 bytes, eight 16-byte chunks, the first four for the stage's first step.  Chunk c of row r lies at
// c ^ f(r).  A fragment's lanes read 16 bytes of 16 rows each, in four turns; a turn takes four lanes each of four groups: rows
// 0-3 and 12-15 at one chunk and rows 4-11 at its neighbour, or the other way round.  f spreads both kinds over all banks, where a
// fragment has 16 rows in a row and where it has 4 of each 8.
__device__ __forceinline__ int swap_rows(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int swap_fours(int r) { return ((r >> 1) & 1) | ((r >> 2) & 6); }
// Transposed, 16-bit: 64 rows (the summed index) of 256 columns, 512 bytes.  kWeights' rows: a fragment has 16 columns in a row,
// their 32 bytes (group g) lie at g ^ swap16(k).  Weights: it has 4 of each 8, 64 bytes (group g) lie at g ^ k % 4.
__device__ __forceinline__ int swap16(int k) { return (k & 3) | ((k >> 1) & 4); }
// Results: register i of a lane is column (lane / 16) * 4 + i of a fragment.  With PAIRED fragments j and j + 1 have 4 columns
// of each 8 in turn, so that a lane has 8 columns in a row and stores 16 bytes.
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
// lane branches (a branch that differs between lanes would take the loops around it out of scalar control).  Bytes within a blob, its
// gradient and a tile's kept sums pass 2^31: they are counted in unsigned 32 bits, elements in signed ones.
constexpr uint32_t kNowhere = 0xf8000000u;
template <int N>
__device__ __forceinline__ void store_bf16(Buffer p, uint32_t off, const float (&v)[N]) {
  if constexpr (N == 8) {
    rows_u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    __builtin_amdgcn_raw_buffer_store_b128(w, p, off, 0, 0);
  } else {
    rows_u32x2 w;
    w[0] = pack_bf16(v[0], v[1]);
    w[1] = pack_bf16(v[2], v[3]);
    __builtin_amdgcn_raw_buffer_store_b64(w, p, off, 0, 0);
  }
}
// Whole lines.  Before: a lane of row l (of 16) has 16 bytes in a, and 16 bytes further on or in the line's second half in b.  After:
// the lanes l and l ^ 8 have both of row l & 7 in a and both of row (l & 7) + 8 in b, lane l the part l / 8.  A store then
// writes eight rows of 128 bytes rather than sixteen of 64 (alone, 1 GB of gradients: 221 us in halves, 175 in whole lines).
__device__ __forceinline__ void swap_halves(rows_u32x4 &a, rows_u32x4 &b) {
  const bool low = (threadIdx.x & 8) == 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t got = __builtin_amdgcn_update_dpp(0, low ? b[i] : a[i], 0x128, 0xf, 0xf, true);  // (of lane l ^ 8)
    a[i] = low ? a[i] : got;
    b[i] = low ? got : b[i];
  }
}
// (past the caches, which the loads need: gradients of the weights 655 us without, 629 with)
__device__ __forceinline__ void store16(Buffer p, uint32_t off, rows_u32x4 v) { __builtin_amdgcn_raw_buffer_store_b128(v, p, off, 0, 2); }
// `off`: of row l & 7; row (l & 7) + 8 lies `eight_rows` bytes on
__device__ __forceinline__ void store_lines(Buffer p, uint32_t off, uint32_t eight_rows, rows_u32x4 a, rows_u32x4 b) {
  swap_halves(a, b);
  store16(p, off, a);
  store16(p, off + eight_rows, b);
}
__device__ __forceinline__ rows_u32x4 four_f32(const float *v) {
  rows_u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
  return w;
}
template <typename Get>
__device__ __forceinline__ rows_u32x4 eight_bf16(Get v) {
  rows_u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16(v(2 * i), v(2 * i + 1));
  return w;
}
__device__ __forceinline__ void load8_f32(Buffer p, uint32_t off, float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const rows_u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(p, off + 16 * h, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * h + i] = __uint_as_float(w[i]);
  }
}
__device__ __forceinline__ float half_lo(uint32_t v) { return (float)__builtin_bit_cast(_Float16, (uint16_t)v); }
__device__ __forceinline__ float half_hi(uint32_t v) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(v >> 16)); }
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }

// ---- one tile ---------------------------------------------------------------------------------------------
// NJ: fragments of 16 weight rows or columns a wavefront has.  MB: 32-row blocks of a tile at most.
// RS, WS: stages of the rows' ring and of the weights'.
template <int FORM, bool INT8, int NJ, int MB, int RS, int WS>
struct Product {
  static constexpr int EL = INT8 ? 1 : 2;
  static constexpr int ROWS = MB * 32, COLS = NJ * 64, OF_WAVE = NJ * 16;  // of a tile; of a wavefront
  static constexpr int RECS = COLS / 2;                                   // kUp: records of a tile, each has two products
  static constexpr bool NARROW = FORM == kColumns && INT8;       // the weights' stage is of bytes: half as long
  static constexpr uint32_t ROW_STAGE = ROWS * 128, WEIGHT_STAGE = COLS * (NARROW ? 64 : 128), WEIGHT_BASE = RS * ROW_STAGE;
  static constexpr uint32_t LDS_BYTES = WEIGHT_BASE + WS * WEIGHT_STAGE;
  static constexpr int A_LOADS = MB / 2, B_LOADS = NARROW ? NJ / 2 : NJ;  // of a wavefront for a stage
  static constexpr bool FOURS = FORM == kDgu || (FORM == kUp && NJ == 4);  // side by side: fragments of 4 rows of each 8
  static constexpr int T_BYTES = NARROW ? COLS : COLS * 2, T_LANES = T_BYTES / 16, T_ROWS = 64 / T_LANES;  // transposed: a row, its lanes in a load, rows of a load
  using Acc = std::conditional_t<INT8 && FORM == kUp, i32x4, f32x4>;

  const ProductArgs g;  // (a copy: through a reference the arguments would not be known to be the same in every lane)
  uint8_t *lds;
  int lane, wave, wm, wn, pitch;
  uint32_t row_bytes;
  int n_cols, m_both, m_tiles;  // tiles over the columns; kWeights: over 2 * pitch rows of gate and up gradients, then pitch of down
  // Of the workgroup's tiles: lane i has tile listed + i.  (Requests are at most as many tiles ahead as there are stages.)
  static constexpr int LIST = 64 - 2 * WS;
  TileList deal;
  Tile list;
  int listed;
  // What is requested next, of the rows and of the weights: the tile, how many of its stages are left, the place in the ring and
  // where the operand is; the lane's place in loads 0 and 1 (2 and 3 are a_more, b_more behind; side by side see b_xor)
  static constexpr bool SIDE = FORM == kUp || FORM == kDgu;
  i32x4 a, b;  // resources
  int a_tile, b_tile, a_left, b_left;
  uint32_t a_put, b_put, a_at, b_at, a_more, b_more;
  uint32_t a_off[2], b_off[SIDE ? 1 : 2];
  int section_left;                              // kColumns: stages of the first section to come
  const uint8_t *a_base, *b_base;                // kWeights
  uint32_t a_row, a_skip, b_skip;
  int a_rows_left, b_rows_left;

  __device__ __forceinline__ Product(const ProductArgs &args, uint8_t *l) : g(args), lds(l) {
    lane = threadIdx.x & 63;
    wave = uniform(threadIdx.x >> 6);
    wm = wave >> 2;
    wn = wave & 3;
    pitch = expert_rows_pitch(g.p.inter);
    row_bytes = (uint32_t)g.p.hidden * EL;
    n_cols = FORM == kUp ? (pitch + RECS - 1) / RECS : FORM == kDgu ? (pitch + COLS - 1) / COLS : g.p.hidden / COLS;
    m_both = (2 * pitch + 255) / 256;
    m_tiles = m_both + (pitch + 255) / 256;
    deal = deal_tiles<FORM, ROWS>(g.p, n_cols, m_tiles);
    listed = 0;
    list = lane_tile<FORM, ROWS>(g.p, deal, n_cols, m_tiles);
    a_put = 0;
    b_put = WEIGHT_BASE;
    a_tile = b_tile = 0;
    open_rows();
    open_weights();
  }
  // tile i of the workgroup, the same in every lane
  __device__ __forceinline__ Tile tile(int i) const {
    const int l = i - listed;
    return Tile{of_lane(list.expert, l), of_lane(list.row0, l), of_lane(list.rows, l), of_lane(list.col, l)};
  }
  // kWeights: the tile's rows of the gradient: first of the 3 * pitch, how many
  __device__ __forceinline__ int gradient_row(const Tile &t) const {
    const int m = t.col % m_tiles;
    return m < m_both ? m * 256 : 2 * pitch + (m - m_both) * 256;
  }
  __device__ __forceinline__ int gradient_rows(int first) const { return min(256, (first < 2 * pitch ? 2 : 3) * pitch - first); }
  __device__ __forceinline__ int stages_of(const Tile &t) const {
    // (an expert without rows has a stage of zeros: its gradients)
    return FORM == kWeights ? max((t.rows + 63) / 64, 1) : FORM == kColumns ? pitch / 64 * g.sections : row_bytes / 128;
  }

  // a_tile, b_tile: from its first stage on.  Behind the last tile nothing is loaded (a resource without bytes).
  __device__ __forceinline__ void open_rows() {
    const Tile t = tile(a_tile);
    const bool any = t.expert >= 0;
    a_left = any ? stages_of(t) : INT32_MAX;
    a_at = 0;
    if constexpr (FORM == kWeights) {
      const int m = gradient_row(t);
      const bool down = m >= 2 * pitch;
      a_rows_left = any ? t.rows : 0;
      a_row = (down ? pitch : 2 * pitch) * 2;
      a_skip = (down ? m - 2 * pitch : m) * 2;
      a_base = (down ? g.a2 : g.a) + (int64_t)t.row0 * a_row + a_skip;
      a_more = 4 * a_row;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = (wave * 4 + i) * 2 + lane / 32;
        a_off[i] = k * a_row + ((lane & 31) ^ (swap16(k) << 1)) * 16;
      }
    } else {
      const uint32_t a_bytes = FORM == kColumns ? (uint32_t)g.a_pitch * 2 : row_bytes;
      a = words_of(g.a + (int64_t)t.row0 * a_bytes, any ? t.rows * a_bytes : 0);
      a_more = 16 * a_bytes;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = (wave * A_LOADS + i) * 8 + lane / 8;
        a_off[i] = (uint32_t)r * a_bytes + ((lane & 7) ^ swap_rows(r)) * 16;
      }
    }
  }
  __device__ __forceinline__ void open_weights() {
    const Tile t = tile(b_tile);
    const bool any = t.expert >= 0;
    b_left = any ? stages_of(t) : INT32_MAX;
    if constexpr (FORM == kWeights) {
      const bool down = gradient_row(t) >= 2 * pitch;
      b_at = 0;
      b_rows_left = any ? t.rows : 0;
      b_skip = t.col / m_tiles * COLS * 2;
      b_base = (down ? g.b2 : g.b) + (int64_t)t.row0 * row_bytes + b_skip;
      b_more = 4 * row_bytes;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = (wave * 4 + i) * 2 + lane / 32;
        b_off[i] = k * row_bytes + ((lane & 31) ^ ((k & 3) << 2)) * 16;
      }
    } else {
      const uint32_t rec_bytes = 3 * row_bytes;
      b = words_of(g.p.blobs + (int64_t)max(t.expert, 0) * g.p.blob_stride, any ? (uint32_t)g.p.inter * rec_bytes : 0);
      section_left = pitch / 64;
      if constexpr (SIDE) {
        // kUp: of a wavefront's rows of the image the first half are gate rows, the others the same records' up rows.  (A record
        // that is not there lies behind the end of the resource.)  Load i has the records 8 * i further on, its chunks are
        // exchanged with another number: see swap_rows, swap_fours.
        const int r = wave * (B_LOADS * 8) + lane / 8, half = OF_WAVE / 2;
        const int rec = FORM == kUp ? t.col * RECS + r / OF_WAVE * half + r % half : t.col * COLS + r, which = FORM == kUp ? r / half & 1 : 2;
        b_off[0] = (uint32_t)(rec * 3 + which) * row_bytes + ((lane & 7) ^ (FOURS ? swap_fours(r) : swap_rows(r))) * 16;
        b_more = 8 * rec_bytes;
        b_at = 0;
      } else {
        b_at = g.first * row_bytes;
        b_more = 4 * rec_bytes;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int k = (wave * B_LOADS + i) * T_ROWS + lane / T_LANES, pos = lane % T_LANES;
          const int chunk = NARROW ? pos ^ (k & (T_LANES - 1)) : pos ^ ((k & 3) << 2);
          b_off[i] = (uint32_t)k * rec_bytes + t.col * COLS * EL + chunk * 16;
        }
      }
    }
  }

  // Requests load i of the next stage of a side; behind the last load the side is at the stage after it, of the next tile if this
  // one has no more.
  __device__ __forceinline__ void request_rows(int i) {
    uint8_t *at = lds + a_put + wave * (A_LOADS * 1024);
    if constexpr (FORM == kWeights) {
      const int n = max(min(64, a_rows_left), 0);
      a = words_of(a_base, n > 0 ? n * a_row - a_skip : 0);
    }
    to_lds(a, a_off[i & 1], a_at + (i >> 1) * a_more, at + i * 1024);
    if (i + 1 < A_LOADS) return;
    if constexpr (FORM == kWeights) {
      a_rows_left -= 64;
      a_base += 64 * a_row;
    } else {
      a_at += 128;
    }
    a_put = next_row_stage(a_put);
    if (--a_left == 0) {
      ++a_tile;
      open_rows();
    }
  }
  __device__ __forceinline__ void request_weights(int i) {
    uint8_t *at = lds + b_put + wave * (B_LOADS * 1024);
    if constexpr (FORM == kWeights) {
      const int n = max(min(64, b_rows_left), 0);
      b = words_of(b_base, n > 0 ? n * row_bytes - b_skip : 0);
    }
    if constexpr (SIDE) to_lds(b, b_off[0] ^ (i * (FOURS ? 32 : 64)), b_at + i * b_more, at + i * 1024);
    else to_lds(b, b_off[i & 1], b_at + (i >> 1) * b_more, at + i * 1024);
    if (i + 1 < B_LOADS) return;
    if constexpr (FORM == kWeights) {
      b_rows_left -= 64;
      b_base += 64 * row_bytes;
    } else if constexpr (SIDE) {
      b_at += 128;
    } else if constexpr (FORM == kColumns) {
      // (behind the last record: outside of the resource)
      b_at += 64 * 3 * row_bytes;
      if (--section_left == 0) b_at = (g.first + 1) * row_bytes;
    }
    b_put = next_weight_stage(b_put);
    if (--b_left == 0) {
      ++b_tile;
      open_weights();
    }
  }
  __device__ __forceinline__ void request_rows() {
#pragma unroll
    for (int i = 0; i < A_LOADS; ++i) request_rows(i);
  }
  __device__ __forceinline__ void request_weights() {
#pragma unroll
    for (int i = 0; i < B_LOADS; ++i) request_weights(i);
  }
  static __device__ __forceinline__ uint32_t next_row_stage(uint32_t at) { return RS == 2 ? ROW_STAGE - at : at == WEIGHT_BASE - ROW_STAGE ? 0 : at + ROW_STAGE; }
  static __device__ __forceinline__ uint32_t next_weight_stage(uint32_t at) { return at == LDS_BYTES - WEIGHT_STAGE ? WEIGHT_BASE : at + WEIGHT_STAGE; }

  // Where the lane's fragments lie in a stage: of the weights for each j, of the rows for block 0; of the stage's first step.
  __device__ __forceinline__ void fragment_offsets(uint32_t (&w_at)[NJ], uint32_t &x_at) const {
    const int l = lane & 15, q = lane >> 4;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if constexpr (NARROW) {
        const int k = q * 8 + (l >> 1);
        w_at[j] = k * T_BYTES + (((wn * NJ + j) ^ (k & (T_LANES - 1))) * 16) + (l & 1) * 8;
      } else if constexpr (!SIDE) {
        const int k = q * 8 + (l >> 2), chunk = wn * NJ * 2 + (j >> 1) * 4 + (l & 3);
        w_at[j] = k * T_BYTES + ((chunk ^ ((k & 3) << 2)) * 16) + (j & 1) * 8;
      } else if constexpr (FOURS) {
        // kUp: fragments 0, 2 are gate rows, 1, 3 up rows
        const int four = FORM == kUp ? j >> 1 : j & 1, half = FORM == kUp ? j & 1 : j >> 1;
        const int r = wn * OF_WAVE + half * 32 + (l >> 2) * 8 + four * 4 + (l & 3);
        w_at[j] = r * 128 + ((q ^ swap_fours(r)) * 16);
      } else {
        const int r = wn * OF_WAVE + j * 16 + l;  // gate rows, up rows
        w_at[j] = r * 128 + ((q ^ swap_rows(r)) * 16);
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
      return widen(__builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(i32x2, lds + stage + w_at + (second ? 32 * T_BYTES : 0))));
    } else if constexpr (FORM == kWeights || FORM == kColumns) {
      return transposed<T_BYTES>(lds + stage + w_at + (second ? 32 * T_BYTES : 0));
    } else {
      i32x4 w = *reinterpret_cast<const i32x4 *>(lds + stage + (w_at ^ (second ? 64 : 0)));
      if constexpr (INT8) w ^= (int)0x80808080;
      return w;
    }
  }
  // block m (transposed, the block is part of what was exchanged: see swap16)
  __device__ __forceinline__ i32x4 read_x(uint32_t x_at, uint32_t stage, bool second, int m) const {
    if constexpr (FORM == kWeights) return transposed<512>(lds + stage + (x_at ^ (m * 64)) + (second ? 32 * 512 : 0));
    else return *reinterpret_cast<const i32x4 *>(lds + stage + (x_at ^ (second ? 64 : 0)) + m * 4096);
  }

  __device__ __forceinline__ void run() {
    Tile t = tile(0);
    if (t.expert < 0) return;
    i32x4 x[MB], w0[NJ], w1[NJ];
    uint32_t w_at[NJ], x_at, rows_stage = 0, weights_stage = WEIGHT_BASE;  // the stages whose fragments are read
    fragment_offsets(w_at, x_at);
#pragma unroll
    for (int i = 0; i < WS; ++i) {
      if (i < RS) request_rows();
      request_weights();
    }
    landed_but<(RS - 1) * A_LOADS + (WS - 1) * B_LOADS>();
#pragma unroll
    for (int j = 0; j < NJ; ++j) w0[j] = read_w(w_at[j], weights_stage, false);
#pragma unroll
    for (int m = 0; m < MB; ++m) x[m] = read_x(x_at, rows_stage, false, m);
    int stores = 0;  // that this wavefront has issued behind its last request, at least
    for (int i = 0; t.expert >= 0;) {
      const int m0 = FORM == kWeights ? gradient_row(t) : 0;
      const int blocks = ((FORM == kWeights ? gradient_rows(m0) : t.rows) + 31) / 32;  // of 32 rows; a wavefront has half of each
      Acc acc[MB][NJ];
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[m][j] = Acc{};
      // A step reads the fragments of the next one, a block's once the block of this step has gone to the matrix cores.  Blocks that
      // the tile does not have are jumped over.
      const auto step = [&](i32x4 (&now)[NJ], i32x4 (&then)[NJ], bool second) MOE_ROWS_INLINE {
#pragma unroll
        for (int j = 0; j < NJ; ++j) then[j] = read_w(w_at[j], weights_stage, second);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          if (m == 0 || m < blocks) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[m][j] = mma(now[j], x[m], acc[m][j]);
            x[m] = read_x(x_at, rows_stage, second, m);
          }
          // (load by load in between: all at once they would hold up the matrix cores)
          if (!second) {
            if (m < A_LOADS) request_rows(m);
            else if (m < A_LOADS + B_LOADS) request_weights(m - A_LOADS);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (!second) {
#pragma unroll
          for (int m = MB; m < A_LOADS + B_LOADS; ++m) {
            if (m < A_LOADS) request_rows(m);
            else request_weights(m - A_LOADS);
          }
        }
      };
      for (int left = stages_of(t); left > 0; --left) {
        step(w0, w1, true);
        // Everybody has read all of this stage: its places are free.  The next one has landed when no more is outstanding than what
        // was requested behind it, and the stores of the tile before, which came behind that.
        constexpr int BEHIND = (WS > RS ? B_LOADS : 0) + (RS - 2) * (A_LOADS + B_LOADS);
        if (stores >= 24) landed_but<BEHIND + 24>();
        else if (stores >= 12) landed_but<BEHIND + 12>();
        else landed_but<BEHIND>();
        stores = 0;
        rows_stage = next_row_stage(rows_stage);
        weights_stage = next_weight_stage(weights_stage);
        step(w1, w0, false);
      }
      // the next tile's blocks that this one did not have
#pragma unroll
      for (int m = 1; m < MB; ++m)
        if (m >= blocks) x[m] = read_x(x_at, rows_stage, false, m);
      store(t, m0, acc, blocks);
      stores = blocks * (FORM == kUp ? 1 : FORM == kColumns && INT8 ? NJ : FORM == kColumns || FORM == kWeights ? NJ / 2 : 0);
      if (++i - listed == LIST) {
        listed += LIST;
        deal.next += LIST * deal.step;
        list = lane_tile<FORM, ROWS>(g.p, deal, n_cols, m_tiles);
      }
      t = tile(i);
    }
  }

  // lane: row lane % 16 of each block of 16 rows; columns as said at the LDS images
  // m0: kWeights, the tile's first row of the gradient's 3 * pitch
  __device__ __forceinline__ void store(const Tile &t, int m0, const Acc (&acc)[MB][NJ], int blocks) const {
    const ExpertRowsParams &p = g.p;
    const int q = lane >> 4, r0 = wm * 16 + (lane & 15);
    const uint8_t *blob = p.blobs + t.expert * p.blob_stride;
    const int64_t tail = (int64_t)p.inter * 3 * row_bytes;
    if constexpr (FORM == kUp) {
      constexpr int N = NJ * 2;  // records of a lane
      const int rec = t.col * RECS + wn * (OF_WAVE / 2) + q * N;
      const Buffer h = buffer_of(g.out + (int64_t)t.row0 * pitch, t.rows * pitch * 2);
      const Buffer both = buffer_of(g.gu_out + (int64_t)t.row0 * 2 * pitch, g.gu_out ? (uint32_t)t.rows * 2 * pitch * 4 : 0);
      float sg[N], su[N];
      if constexpr (INT8) {
        const Buffer scales = buffer_of(blob + tail, p.inter * 4);
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const rows_u32x2 vg = __builtin_amdgcn_raw_buffer_load_b64(scales, rec < p.inter ? (rec + i) * 2 : kNowhere, 0, 0),
                           vu = __builtin_amdgcn_raw_buffer_load_b64(scales, rec < p.inter ? (p.inter + rec + i) * 2 : kNowhere, 0, 0);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            sg[i + 2 * k] = half_lo(vg[k]);
            sg[i + 2 * k + 1] = half_hi(vg[k]);
            su[i + 2 * k] = half_lo(vu[k]);
            su[i + 2 * k + 1] = half_hi(vu[k]);
          }
        }
      }
      const Buffer row_scale = buffer_of(g.scale + t.row0, INT8 ? t.rows * 4 : 0);
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        if (m > 0 && m >= blocks) break;
        const uint32_t r = r0 + m * 32;
        const float sx = INT8 ? __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(row_scale, r * 4, 0, 0)) : 1.f;
        float v[N], gate[N], up[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          gate[i] = (float)acc[m][(i >> 2) * 2][i & 3];
          up[i] = (float)acc[m][(i >> 2) * 2 + 1][i & 3];
          if constexpr (INT8) {
            gate[i] *= sx * sg[i];
            up[i] *= sx * su[i];
          }
          v[i] = gate[i] * sigmoid(gate[i]) * up[i];
        }
        store_bf16(h, rec < pitch ? (r * pitch + rec) * 2 : kNowhere, v);
        if (g.gu_out) {
          if constexpr (N == 8) {
            const uint32_t at = rec < pitch ? ((m * 32 + wm * 16 + (lane & 7)) * 2 * pitch + rec + (lane & 8) / 2) * 4u : kNowhere;
            store_lines(both, at, 64 * pitch, four_f32(gate), four_f32(gate + 4));
            store_lines(both, at + pitch * 4, 64 * pitch, four_f32(up), four_f32(up + 4));
          } else {
            const uint32_t at = rec < pitch ? (r * 2 * pitch + rec) * 4 : kNowhere;
            store16(both, at, four_f32(gate));
            store16(both, at + pitch * 4, four_f32(up));
          }
        }
      }
    } else if constexpr (FORM == kDgu) {
      const Buffer in = buffer_of(g.gu_in + (int64_t)t.row0 * 2 * pitch, (uint32_t)t.rows * 2 * pitch * 4),
                   out = buffer_of(g.out + (int64_t)t.row0 * 2 * pitch, t.rows * 2 * pitch * 2);
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        if (m > 0 && m >= blocks) break;
        rows_u32x4 dg[NJ / 2], du[NJ / 2];
#pragma unroll
        for (int h = 0; h < NJ / 2; ++h) {
          const int rec = t.col * COLS + wn * OF_WAVE + h * 32 + q * 8;
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
          dg[h] = eight_bf16([&](int i) MOE_ROWS_INLINE { return gate[i]; });
          du[h] = eight_bf16([&](int i) MOE_ROWS_INLINE { return up[i]; });
        }
        // (behind the last record: the resource ends before kNowhere / 2)
        if constexpr (NJ == 4) {
          const int rec = t.col * COLS + wn * OF_WAVE + (lane & 8) * 4 + q * 8;
          const uint32_t at = rec < pitch ? (m * 32 + wm * 16 + (lane & 7)) * 2 * pitch + rec : kNowhere / 4;
          store_lines(out, at * 2, 32 * pitch, dg[0], dg[1]);
          store_lines(out, (at + pitch) * 2, 32 * pitch, du[0], du[1]);
        } else {
          const int rec = t.col * COLS + wn * OF_WAVE + q * 8;
          const uint32_t at = rec < pitch ? (r0 + m * 32) * 2 * pitch + rec : kNowhere / 4;
          store16(out, at * 2, dg[0]);
          store16(out, (at + pitch) * 2, du[0]);
        }
      }
    } else if constexpr (FORM == kColumns) {
      const Buffer out = buffer_of(g.out + (int64_t)t.row0 * p.hidden, t.rows * p.hidden * 2);
      if constexpr (INT8) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int col = t.col * COLS + wn * OF_WAVE + j * 16 + q * 4;
          const rows_u32x2 w = *reinterpret_cast<const rows_u32x2 *>(blob + tail + (int64_t)p.inter * 4 + col * 2);
          const float sd[4] = {half_lo(w[0]), half_hi(w[0]), half_lo(w[1]), half_hi(w[1])};
#pragma unroll
          for (int m = 0; m < MB; ++m) {
            if (m > 0 && m >= blocks) break;
            const float v[4] = {acc[m][j][0] * sd[0], acc[m][j][1] * sd[1], acc[m][j][2] * sd[2], acc[m][j][3] * sd[3]};
            store_bf16(out, ((r0 + m * 32) * p.hidden + col) * 2, v);
          }
        }
      } else {
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          if (m > 0 && m >= blocks) break;
          const auto half = [&](int h) MOE_ROWS_INLINE {
            return eight_bf16([&](int i) MOE_ROWS_INLINE { return acc[m][h * 2 + (i >> 2)][i & 3]; });
          };
          const int col = t.col * COLS + wn * OF_WAVE + q * 8;
          if constexpr (NJ == 4)
            store_lines(out, ((m * 32 + wm * 16 + (lane & 7)) * p.hidden + col + (lane & 8) * 4) * 2, 8 * p.hidden * 2, half(0), half(1));
          else
            __builtin_amdgcn_raw_buffer_store_b128(half(0), out, ((r0 + m * 32) * p.hidden + col) * 2, 0, 0);
        }
      }
    } else {
      const Buffer out = buffer_of(g.dblobs + t.expert * p.blob_stride, (uint32_t)tail);
      const int m_rows = gradient_rows(m0), col0 = t.col / m_tiles * COLS;
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        if (m > 0 && m >= blocks) break;
        const int r = m * 32 + wm * 16 + (lane & 7), at = m0 + r, which = at >= 2 * pitch ? 2 : at >= pitch ? 1 : 0, rec = at - which * pitch;
        // (a record that is not there lies behind the end)
        const uint32_t to = r < m_rows ? ((rec * 3 + which) * p.hidden + col0 + wn * 64 + (lane & 8) * 4 + q * 8) * 2u : kNowhere;
        const rows_u32x4 v0 = eight_bf16([&](int i) MOE_ROWS_INLINE { return acc[m][i >> 2][i & 3]; }),
                   v1 = eight_bf16([&](int i) MOE_ROWS_INLINE { return acc[m][2 + (i >> 2)][i & 3]; });
        store_lines(out, to, 8 * 3 * p.hidden * 2, v0, v1);
      }
    }
  }
};

template <int FORM, bool INT8, int NJ, int MB, int RS = 2, int WS = 3>
__global__ __launch_bounds__(kBlock, MB == 8 || RS > 2 ? 2 : FORM == kColumns && INT8 && MB == 2 ? 8 : 4) void product_kernel(const ProductArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[Product<FORM, INT8, NJ, MB, RS, WS>::LDS_BYTES];
  if constexpr (FORM == kColumns) {  // rows of nobody: ahead of the first expert (some of the experts on all of the rows), behind the last
    const ExpertRowsParams &p = g.p;
    const int first = uniform(first_row(p, 0)), end = max(uniform(min(p.offsets[p.n_experts], p.n_rows)), first);
    for (int r = blockIdx.x; r < p.n_rows - (end - first); r += gridDim.x) {
      uint16_t *row = g.out + (int64_t)(r < first ? r : r + (end - first)) * p.hidden;
      for (int c = threadIdx.x * 8; c < p.hidden; c += kBlock * 8) *reinterpret_cast<rows_u32x4 *>(row + c) = rows_u32x4{};
    }
  }
  Product<FORM, INT8, NJ, MB, RS, WS> f(g, lds);
  f.run();
}

// Which tiles, by the rows an expert has on average (the host knows no more).  Large: 256 x 256, one workgroup a compute unit.  Middle:
// 128 x 128, two workgroups, so that one computes while the other waits for weights or stores.  Small: 64 x 128, two workgroups,
// less work for rows that are not there.  Measured with 60 uneven experts of 2048 x 1408 and four a token, small | middle | large, us:
//   tokens (rows an expert)   512 (34)        768 (51)          1024 (68)         1536 (102)        2048 (137)        4096 (273)
//   kUp                       163 | 160 | 166 152 | 145 | 158   171 | 170 | 184   190 | 176 | 168   215 | 197 | 196   329 | 256 | 222
//   kColumns                  77 | 80 | 84    88 | 85 | 84      88 | 90 | 86      103 | 99 | 93     111 | 108 | 99    174 | 141 | 135
//   kUp, 8 bits               76 | 83 | 77    -                 88 | 91 | 87      102 | 97 | 95     114 | 105 | 103   173 | 139 | 128
//   kColumns, 8 bits          55 | 60 | 73    -                 63 | 71 | 81      80 | 74 | 90      90 | 94 | 98      156 | 134 | 143
//   kDgu                                                                                                              225 | 193 | 198
// and with 8192 tokens kColumns, 8 bits, 322 | 258 | 229.  (kUp in 8 bits and kDgu have the limits of kUp in bf16; in the table another
// form is ahead by up to 4 % for them there.)  Where tiles are too few for the compute units, smaller ones: 8 experts of
// 1024 x 704 and two a token, 2048 tokens 36 | 37 | 39; 16 of 2048 x 512 and two, 600 tokens 31 | 35 | 44.
//
// One small tile a compute unit at most, in bf16: nobody else keeps memory busy, so the rings have all of the LDS (kUp, 60 experts of
// 2048 x 1408 and four a token, 1 token 12.7 us, otherwise 15.8; 2 tokens 17.5 and 20; kColumns, 1 token 11.2 and 12.1).  8-bit rows
// have half the stages (11 and 11): not there.
//
// Columns of bytes take half the LDS: four workgroups a compute unit with small tiles (two, or two of 64 x 256 | four: 16 tokens 45, 36 |
// 33, 512 tokens 68, 61 | 60, 1024 tokens -, 74 | 65, 8 experts of 4096 x 4096 and 512 tokens -, 100 | 85; but 256 tokens 55, 43 | 48),
// 256 columns a middle tile (4096 tokens 136, with 128 columns 144).
template <int FORM, bool INT8>
hipError_t launch_product(const ProductArgs &g, int n_cus, hipStream_t s) {
  const int grid = n_cus / 8 * 8;  // (the XCDs are eight)
  if constexpr (FORM != kWeights) {
    // upper bounds, from what the host knows
    const int64_t n_rows = g.p.n_rows, n_experts = g.p.n_experts, with_rows = n_rows < n_experts ? n_rows : n_experts;
    const int pitch = expert_rows_pitch(g.p.inter), wide = FORM == kUp ? 2 * pitch : FORM == kDgu ? pitch : g.p.hidden;
    const auto tiles = [&](int rows, int cols) { return (n_rows / rows + with_rows) * ((wide + cols - 1) / cols); };
    constexpr bool BYTES = FORM == kColumns && INT8;
    constexpr int SMALL = BYTES ? 88 : 48, MIDDLE = BYTES ? 320 : FORM == kColumns ? SMALL : 84;
    if (n_rows <= SMALL * n_experts || tiles(128, 128) < grid) {
      constexpr bool DEEP = FORM != kDgu && !INT8;
      if (DEEP && tiles(64, 128) <= grid)
        hipLaunchKernelGGL((product_kernel<FORM, INT8, 2, 2, DEEP ? 6 : 2, DEEP ? 6 : 3>), dim3(grid), dim3(kBlock), 0, s, g);
      else
        hipLaunchKernelGGL((product_kernel<FORM, INT8, 2, 2>), dim3((BYTES ? 4 : 2) * grid), dim3(kBlock), 0, s, g);
      return hipGetLastError();
    }
    if (n_rows <= MIDDLE * n_experts || tiles(256, 256) < grid) {
      hipLaunchKernelGGL((product_kernel<FORM, INT8, BYTES ? 4 : 2, 4>), dim3(2 * grid), dim3(kBlock), 0, s, g);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((product_kernel<FORM, INT8, 4, 8>), dim3(grid), dim3(kBlock), 0, s, g);
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
