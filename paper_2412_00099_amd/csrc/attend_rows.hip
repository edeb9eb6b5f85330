// Attention of packed sequences, causal, with a window and a few first keys that stay visible; its gradients.
//
//   Z = scale Q K^T over the keys that a query sees, P = exp(Z - lse), Y = P V
//   delta = rowsum(dY Y), dP = dY V^T, dZ = P (dP - delta), dQ = scale dZ K, dK = scale dZ^T Q, dV = P^T dY
//
// Three kernels, all products on the matrix cores with sums in 32 bits: forward (Q rows), gradient of Q (Q rows; it works delta out
// too) and of K and V (K rows; the heads of a group one after the other, so that sums have one order and need no atomics).  A
// wavefront has 32 rows, which it keeps in registers as columns of every product: Z^T = K Q^T, O^T = V^T P^T, and so on.  A product's
// result goes into the next one from the registers that it is in: register i of a lane is row 8 (i / 4) + 4 (lane / 32) + i % 4, the
// next product sums over these rows in any order, and its other operand is read from LDS, transposed, in the same order.
// The other side's rows go through LDS in tiles of 64, two at a time, one computed while the next one is loaded, for all four
// wavefronts of a workgroup.
//
// P and dZ are rounded to bf16 for the matrix cores: in two parts each they would cost half as much again, and the error that they
// make (2^-9 of single terms of a sum, at random) is below that of the rounding of the results.
//
// Which sequence and which of its rows a workgroup has is worked out from the offsets on the device.  Loads go through buffer
// resources that end where the sequence ends: what lies beyond arrives as zeros.
#include <algorithm>

#include "attend.h"
#include "rows.h"
#include "tiles.h"

namespace moe {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kBlock = kWaves * 64;
constexpr int kOwn = 32 * kWaves;  // rows of a workgroup
constexpr int kTile = 64;          // rows of the other side in LDS
constexpr uint32_t kNowhere = 0xf8000000u;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ f32x16 mma(i32x4 a, i32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// A sequence: its rows of q and of k; query r is at position r + ahead
struct Sequence {
  int q0, nq, k0, nk, ahead;
};
__device__ __forceinline__ Sequence sequence_of(const AttendRowsParams &p, int s) {
  Sequence r;
  r.q0 = min(max(p.offsets[s], 0), p.n_rows);
  r.nq = max(min(p.offsets[s + 1], p.n_rows) - r.q0, 0);
  r.k0 = min(max(p.k_offsets[s], 0), p.n_k_rows);
  r.nk = max(min(p.k_offsets[s + 1], p.n_k_rows) - r.k0, 0);
  r.ahead = r.nk - r.nq;
  return r;
}
// Part `want` of the sequences' rows in parts of kOwn, a sequence's last part first (it has the most keys); no such part: sequence
// -1, and by how much it was missed
struct Part {
  int sequence, part, over;
};
template <bool KEYS>
__device__ __forceinline__ Part part_of(const AttendRowsParams &p, int want) {
  const int32_t *offsets = KEYS ? p.k_offsets : p.offsets;
  const int most = KEYS ? p.n_k_rows : p.n_rows, lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
    const int s = s0 + lane;
    int n = 0;
    if (s < p.n_seqs) {
      const int from = min(max(offsets[s], 0), most);
      n = (max(min(offsets[s + 1], most) - from, 0) + kOwn - 1) / kOwn;
    }
    const int64_t past = before + sum_upto((int64_t)n);
    const uint64_t behind = __ballot(past > want);
    if (behind != 0) {
      const int at = __builtin_ctzll(behind), in = (int)(of_lane(past, at) - want);
      return {uniform(s0 + at), KEYS ? uniform(of_lane(n, at) - in) : uniform(in - 1), 0};
    }
    before = of_lane(past, 63);
  }
  return {-1, 0, uniform((int)(want - before))};
}
// zeros for the rows of no sequence, shared by `step` workgroups
__device__ __forceinline__ void clear_rows(const int32_t *offsets, int n_seqs, int n_rows, uint16_t *to, int head, int heads, int dim, int at, int step) {
  const int first = min(max(offsets[0], 0), n_rows), last = min(max(offsets[n_seqs], first), n_rows);
  const int64_t units = (int64_t)(first + n_rows - last) * (dim / 8);
  for (int64_t u = (int64_t)at * kBlock + threadIdx.x; u < units; u += (int64_t)step * kBlock) {
    int64_t r = u / (dim / 8);
    if (r >= first) r += last - first;
    *reinterpret_cast<rows_u32x4 *>(to + (r * heads + head) * dim + u % (dim / 8) * 8) = rows_u32x4{0, 0, 0, 0};
  }
}

// Rows of DT values in LDS.  Chunk c of row r lies at c ^ f(r): both kinds of reads (16 rows at one chunk; 8 rows of four chunks,
// transposed) spread over all banks
template <int DT>
struct Tiles {
  static constexpr int ROW = DT * 2, CHUNKS = ROW / 16, ROWS_LOAD = 64 / CHUNKS;
  static constexpr int BYTES = kTile * ROW, LOADS = BYTES / 1024 / kWaves;  // of a wavefront for a tile
  static constexpr int KS = DT / 16, DS = DT / 32;                          // steps over the dims, blocks of them
  static __device__ __forceinline__ int swap(int r) { return CHUNKS == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3); }

  // where a wavefront's loads of a tile come from, per lane
  struct Source {
    uint32_t off[LOADS];
  };
  static __device__ __forceinline__ Source source(int wave, int lane, int64_t token, int dim) {
    Source s;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = (wave * LOADS + i) * ROWS_LOAD + lane / CHUNKS, c = ((lane % CHUNKS) ^ swap(r)) * 16;
      s.off[i] = c < dim * 2 ? (uint32_t)(r * (uint32_t)token * 2 + c) : kNowhere;
    }
    return s;
  }
  // the tile's rows from `from` on, `rows` of them (or fewer than none)
  static __device__ __forceinline__ void request(const Source &s, const uint16_t *from, int rows, int64_t token, int dim, int wave, uint8_t *to) {
    const i32x4 b = words_of(from, rows > 0 ? (uint32_t)((min(rows, kTile) - 1) * (uint32_t)token * 2 + dim * 2) : 0u);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) to_lds(b, s.off[i], 0, to + (wave * LOADS + i) * 1024);
  }
  // 32 rows from r0 on as rows of a product, step s over the dims
  static __device__ __forceinline__ i32x4 rows(const uint8_t *t, int r0, int s, int lane) {
    const int r = r0 + (lane & 31);
    return *reinterpret_cast<const i32x4 *>(t + r * ROW + (((s * 2 + (lane >> 5)) ^ swap(r)) * 16));
  }
  // dims d * 32 .. as rows of a product, summed over the 16 rows from r0 on
  static __device__ __forceinline__ i32x4 columns(const uint8_t *t, int r0, int d, int lane) {
    const int r = r0 + 4 * (lane >> 5) + ((lane & 15) >> 2), c = d * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), in = (lane & 1) * 8;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, t + r * ROW + ((c ^ swap(r)) * 16) + in));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, t + (r + 8) * ROW + ((c ^ swap(r + 8)) * 16) + in));
    return __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // a wavefront's own rows as columns of a product: lane's row is `at` (there: it exists)
  static __device__ __forceinline__ void own(const uint16_t *at, bool there, int dim, int lane, i32x4 (&f)[KS]) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = s * 16 + (lane >> 5) * 8;
      f[s] = i32x4{0, 0, 0, 0};
      if (there && d < dim) f[s] = *reinterpret_cast<const i32x4 *>(at + d);
    }
  }
  // the lane's column of a result, times v
  static __device__ __forceinline__ void store(uint16_t *at, bool there, int dim, int lane, const f32x16 (&o)[DS], float v) {
#pragma unroll
    for (int d = 0; d < DS; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = d * 32 + i * 8 + (lane >> 5) * 4;
        if (there && c < dim)
          *reinterpret_cast<rows_u32x2 *>(at + c) = rows_u32x2{pack_bf16(o[d][4 * i] * v, o[d][4 * i + 1] * v), pack_bf16(o[d][4 * i + 2] * v, o[d][4 * i + 3] * v)};
      }
  }
};
// rows 16 t .. of a result as the summed side of the next product
__device__ __forceinline__ i32x4 summed(const f32x16 &p, int t) {
  i32x4 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = (int)pack_bf16(p[8 * t + 2 * i], p[8 * t + 2 * i + 1]);
  return f;
}

struct Item {
  int part, head;  // behind the last one: no part
};
// Workgroups go to the XCDs in turn, and each XCD has an L2 of its own: where eight divides the heads of k, an XCD has all
// workgroups of some of them.
__device__ __forceinline__ Item item_of(int heads, int kv_heads) {
  Item r;
  const uint32_t b = (uint32_t)row_group();
  if (kv_heads % 8 == 0) {
    const uint32_t each = heads / 8, at = b >> 3;
    r.head = (b & 7) * each + at % each;
    r.part = at / each;
  } else {
    r.head = b % heads;
    r.part = b / heads;
  }
  return r;
}
dim3 grid_of(int parts, int heads) {
  const RowGrid g = row_grid((int64_t)parts * heads);
  return dim3(g.x, g.y);
}

// the tiles of keys that the queries r0 .. r1 of a sequence see, in turn
struct KeyTiles {
  int sink_tiles, first, n;
  __device__ __forceinline__ int at(int t) const { return (t < sink_tiles ? t : first + t - sink_tiles) * kTile; }
};
__device__ __forceinline__ KeyTiles key_tiles(const AttendRowsParams &p, const Sequence &s, int r0, int r1) {
  KeyTiles k;
  const int lo = p.window > 0 ? max(r0 + s.ahead - p.window + 1, 0) : 0, end = max(r1 + s.ahead + 1, 0);
  const int last = (end + kTile - 1) / kTile;
  k.first = lo / kTile;
  k.sink_tiles = min((min(p.sinks, lo) + kTile - 1) / kTile, k.first);
  k.n = k.sink_tiles + max(last - k.first, 0);
  return k;
}
// of queries at positions p0 .. p1 and keys k0 .. k1: whether all see all, whether none sees any
__device__ __forceinline__ bool see_all(const AttendRowsParams &p, int p0, int p1, int k0, int k1) {
  return k1 <= p0 && (p.window == 0 || p1 - p.window < k0 || k1 < p.sinks);
}
__device__ __forceinline__ bool see_none(const AttendRowsParams &p, int p0, int p1, int k0, int k1) {
  return k0 > p1 || (p.window > 0 && p0 - p.window >= k1 && k0 >= p.sinks);
}
__device__ __forceinline__ bool sees(const AttendRowsParams &p, int pos, int key) {
  return key <= pos && (p.window == 0 || pos - p.window < key || key < p.sinks);
}

template <int DT>
__global__ __launch_bounds__(kBlock, 2) void attend_rows_kernel(const AttendRowsParams p, const int parts) {
  using T = Tiles<DT>;
  __shared__ __align__(16) uint8_t lds[4 * T::BYTES];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Item item = item_of(p.heads, p.kv_heads);
  if (item.part >= parts) return;
  const Part part = part_of<false>(p, item.part);
  if (part.sequence < 0) {
    clear_rows(p.offsets, p.n_seqs, p.n_rows, p.y, item.head, p.heads, p.dim, part.over, parts - (item.part - part.over));
    return;
  }
  const Sequence s = sequence_of(p, part.sequence);
  const int r0 = part.part * kOwn, r1 = min(r0 + kOwn, s.nq) - 1, mine = r0 + wave * 32, row = mine + (lane & 31);
  const int p0 = mine + s.ahead, p1 = min(mine + 31, r1) + s.ahead, pos = row + s.ahead;
  const int kv = item.head / (p.heads / p.kv_heads);
  const KeyTiles tiles = key_tiles(p, s, r0, r1);
  const uint16_t *k = static_cast<const uint16_t *>(p.k.at) + s.k0 * p.k.token + kv * p.k.head;
  const uint16_t *v = static_cast<const uint16_t *>(p.v.at) + s.k0 * p.v.token + kv * p.v.head;
  const typename T::Source ks = T::source(wave, lane, p.k.token, p.dim), vs = T::source(wave, lane, p.v.token, p.dim);
  const auto request = [&](int t) MOE_ROWS_INLINE {
    const int key = tiles.at(t), rows = s.nk - key;
    uint8_t *to = lds + (t & 1) * 2 * T::BYTES;
    T::request(ks, k + key * p.k.token, rows, p.k.token, p.dim, wave, to);
    T::request(vs, v + key * p.v.token, rows, p.v.token, p.dim, wave, to + T::BYTES);
  };
  i32x4 q[T::KS];
  T::own(static_cast<const uint16_t *>(p.q.at) + (s.q0 + min(row, s.nq - 1)) * p.q.token + item.head * p.q.head, row < s.nq, p.dim, lane, q);
  f32x16 o[T::DS];
#pragma unroll
  for (int d = 0; d < T::DS; ++d) o[d] = zero16();
  float top = -INFINITY, sum = 0.f;
  const float scale = p.scale * kLog2e;
  if (tiles.n > 0) request(0);
  for (int t = 0; t < tiles.n; ++t) {
    landed_but<0>();
    if (t + 1 < tiles.n) request(t + 1);
    const uint8_t *kt = lds + (t & 1) * 2 * T::BYTES, *vt = kt + T::BYTES;
    const int key = tiles.at(t);
    if (mine > r1 || see_none(p, p0, p1, key, key + kTile - 1)) continue;
    f32x16 z[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      z[m] = zero16();
#pragma unroll
      for (int i = 0; i < T::KS; ++i) z[m] = mma(T::rows(kt, m * 32, i, lane), q[i], z[m]);
    }
    if (!see_all(p, p0, p1, key, key + kTile - 1)) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = key + m * 32 + i / 4 * 8 + (lane >> 5) * 4 + i % 4;
          z[m][i] = sees(p, pos, at) ? z[m][i] : -INFINITY;
        }
    }
    float most = -INFINITY;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, z[m][i]);
    most = fmaxf(most, __shfl_xor(most, 32)) * scale;
    // The base of the exponentials follows the largest score when that is 2^8 ahead: until then nothing is multiplied
    if (__any(most > top + 8.f)) {
      const float to = fmaxf(top, most), shrink = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - to);
      top = to;
      sum *= shrink;
#pragma unroll
      for (int d = 0; d < T::DS; ++d) o[d] *= shrink;
    }
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        z[m][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[m][i], scale, -base));
        sum += z[m][i];
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const i32x4 f = summed(z[i >> 1], i & 1);
#pragma unroll
      for (int d = 0; d < T::DS; ++d) o[d] = mma(T::columns(vt, i * 16, d, lane), f, o[d]);
    }
  }
  sum += __shfl_xor(sum, 32);
  const bool there = row < s.nq;
  T::store(p.y + ((int64_t)(s.q0 + row) * p.heads + item.head) * p.dim, there, p.dim, lane, o, sum > 0.f || sum != sum ? 1.f / sum : 0.f);
  if (p.lse && there && lane < 32) p.lse[(int64_t)item.head * p.n_rows + s.q0 + row] = top * kLn2 + __logf(sum);
}

template <int DT>
__global__ __launch_bounds__(kBlock, 2) void attend_rows_dq_kernel(const AttendRowsParams p, const int parts) {
  using T = Tiles<DT>;
  __shared__ __align__(16) uint8_t lds[4 * T::BYTES];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Item item = item_of(p.heads, p.kv_heads);
  if (item.part >= parts) return;
  const Part part = part_of<false>(p, item.part);
  if (part.sequence < 0) {
    clear_rows(p.offsets, p.n_seqs, p.n_rows, p.dq, item.head, p.heads, p.dim, part.over, parts - (item.part - part.over));
    return;
  }
  const Sequence s = sequence_of(p, part.sequence);
  const int r0 = part.part * kOwn, r1 = min(r0 + kOwn, s.nq) - 1, mine = r0 + wave * 32, row = mine + (lane & 31);
  const int p0 = mine + s.ahead, p1 = min(mine + 31, r1) + s.ahead, pos = row + s.ahead;
  const int kv = item.head / (p.heads / p.kv_heads);
  const KeyTiles tiles = key_tiles(p, s, r0, r1);
  const uint16_t *k = static_cast<const uint16_t *>(p.k.at) + s.k0 * p.k.token + kv * p.k.head;
  const uint16_t *v = static_cast<const uint16_t *>(p.v.at) + s.k0 * p.v.token + kv * p.v.head;
  const typename T::Source ks = T::source(wave, lane, p.k.token, p.dim), vs = T::source(wave, lane, p.v.token, p.dim);
  const auto request = [&](int t) MOE_ROWS_INLINE {
    const int key = tiles.at(t), rows = s.nk - key;
    uint8_t *to = lds + (t & 1) * 2 * T::BYTES;
    T::request(ks, k + key * p.k.token, rows, p.k.token, p.dim, wave, to);
    T::request(vs, v + key * p.v.token, rows, p.v.token, p.dim, wave, to + T::BYTES);
  };
  const bool there = row < s.nq;
  const int64_t at_row = s.q0 + min(row, s.nq - 1), dense = (at_row * p.heads + item.head) * p.dim;
  i32x4 q[T::KS], dy[T::KS];
  float delta = 0.f;
  {
    i32x4 y[T::KS];
    T::own(p.y + dense, there, p.dim, lane, y);
    T::own(p.dy + dense, there, p.dim, lane, dy);
#pragma unroll
    for (int i = 0; i < T::KS; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) delta += bf16_lo(y[i][w]) * bf16_lo(dy[i][w]) + bf16_hi(y[i][w]) * bf16_hi(dy[i][w]);
    delta += __shfl_xor(delta, 32);
  }
  T::own(static_cast<const uint16_t *>(p.q.at) + at_row * p.q.token + item.head * p.q.head, there, p.dim, lane, q);
  const float lse = p.lse[(int64_t)item.head * p.n_rows + at_row] * kLog2e, scale = p.scale * kLog2e;
  if (there && lane < 32) p.delta[(int64_t)item.head * p.n_rows + at_row] = delta;
  f32x16 o[T::DS];
#pragma unroll
  for (int d = 0; d < T::DS; ++d) o[d] = zero16();
  if (tiles.n > 0) request(0);
  for (int t = 0; t < tiles.n; ++t) {
    landed_but<0>();
    if (t + 1 < tiles.n) request(t + 1);
    const uint8_t *kt = lds + (t & 1) * 2 * T::BYTES, *vt = kt + T::BYTES;
    const int key = tiles.at(t);
    if (mine > r1) continue;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int key0 = key + m * 32;
      if (see_none(p, p0, p1, key0, key0 + 31)) continue;
      f32x16 z = zero16(), dp = zero16();
#pragma unroll
      for (int i = 0; i < T::KS; ++i) z = mma(T::rows(kt, m * 32, i, lane), q[i], z);
#pragma unroll
      for (int i = 0; i < T::KS; ++i) dp = mma(T::rows(vt, m * 32, i, lane), dy[i], dp);
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], scale, -lse)) * (dp[i] - delta);
      if (!see_all(p, p0, p1, key0, key0 + 31)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = sees(p, pos, key0 + i / 4 * 8 + (lane >> 5) * 4 + i % 4) ? z[i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const i32x4 f = summed(z, i);
#pragma unroll
        for (int d = 0; d < T::DS; ++d) o[d] = mma(T::columns(kt, m * 32 + i * 16, d, lane), f, o[d]);
      }
    }
  }
  T::store(p.dq + dense, there, p.dim, lane, o, p.scale);
}

template <int DT>
__global__ __launch_bounds__(kBlock, 1) void attend_rows_dkv_kernel(const AttendRowsParams p, const int parts) {
  using T = Tiles<DT>;
  __shared__ __align__(16) uint8_t lds[4 * T::BYTES + 4 * kTile * 4];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Item item = item_of(p.kv_heads, p.kv_heads);
  if (item.part >= parts) return;
  const Part part = part_of<true>(p, item.part);
  const int kv = item.head, per = p.heads / p.kv_heads;
  if (part.sequence < 0) {
    const int step = parts - (item.part - part.over);
    clear_rows(p.k_offsets, p.n_seqs, p.n_k_rows, p.dk, kv, p.kv_heads, p.dim, part.over, step);
    clear_rows(p.k_offsets, p.n_seqs, p.n_k_rows, p.dv, kv, p.kv_heads, p.dim, part.over, step);
    return;
  }
  const Sequence s = sequence_of(p, part.sequence);
  const int k0 = part.part * kOwn, k1 = min(k0 + kOwn, s.nk) - 1, mine = k0 + wave * 32, key = mine + (lane & 31);
  const bool there = key < s.nk;
  // the queries that see any of the workgroup's keys
  const int first = max(k0 - s.ahead, 0) / kTile * kTile;
  const int end = p.window > 0 && k0 >= p.sinks ? (int)min((int64_t)s.nq, (int64_t)k1 + p.window - s.ahead) : s.nq;
  const int tiles = max((end - first + kTile - 1) / kTile, 0), all = tiles * per;
  const typename T::Source qs = T::source(wave, lane, p.q.token, p.dim), ds = T::source(wave, lane, (int64_t)p.heads * p.dim, p.dim);
  uint8_t *stats = lds + 4 * T::BYTES;
  const auto request = [&](int t) MOE_ROWS_INLINE {
    const int head = kv * per + t / tiles, row = first + t % tiles * kTile, rows = s.nq - row;
    uint8_t *to = lds + (t & 1) * 2 * T::BYTES;
    T::request(qs, static_cast<const uint16_t *>(p.q.at) + (int64_t)(s.q0 + row) * p.q.token + head * p.q.head, rows, p.q.token, p.dim, wave, to);
    T::request(ds, p.dy + ((int64_t)(s.q0 + row) * p.heads + head) * p.dim, rows, (int64_t)p.heads * p.dim, p.dim, wave, to + T::BYTES);
    const int64_t at = (int64_t)head * p.n_rows + s.q0 + row;
    if (wave < 2) word_to_lds(words_of((wave == 0 ? p.lse : p.delta) + at, (uint32_t)min(rows, kTile) * 4), lane * 4, stats + ((t & 1) * 2 + wave) * kTile * 4);
  };
  i32x4 k[T::KS], v[T::KS];
  const int64_t at_key = s.k0 + min(key, s.nk - 1);
  T::own(static_cast<const uint16_t *>(p.k.at) + at_key * p.k.token + kv * p.k.head, there, p.dim, lane, k);
  T::own(static_cast<const uint16_t *>(p.v.at) + at_key * p.v.token + kv * p.v.head, there, p.dim, lane, v);
  f32x16 dk[T::DS], dv[T::DS];
#pragma unroll
  for (int d = 0; d < T::DS; ++d) dk[d] = dv[d] = zero16();
  const float scale = p.scale * kLog2e;
  if (all > 0) request(0);
  for (int t = 0; t < all; ++t) {
    landed_but<0>();
    if (t + 1 < all) request(t + 1);
    const uint8_t *qt = lds + (t & 1) * 2 * T::BYTES, *dt = qt + T::BYTES;
    const float *lse = reinterpret_cast<const float *>(stats + (t & 1) * 2 * kTile * 4), *delta = lse + kTile;
    const int row = first + t % tiles * kTile;
    if (mine > k1) continue;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int row0 = row + m * 32, p0 = row0 + s.ahead, p1 = min(row0 + 31, s.nq - 1) + s.ahead;
      if (row0 >= s.nq || see_none(p, p0, p1, mine, mine + 31)) continue;
      f32x16 z = zero16(), dp = zero16();
#pragma unroll
      for (int i = 0; i < T::KS; ++i) z = mma(T::rows(qt, m * 32, i, lane), k[i], z);
#pragma unroll
      for (int i = 0; i < T::KS; ++i) dp = mma(T::rows(dt, m * 32, i, lane), v[i], dp);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 l4 = *reinterpret_cast<const f32x4 *>(lse + m * 32 + i * 8 + (lane >> 5) * 4);
        const f32x4 d4 = *reinterpret_cast<const f32x4 *>(delta + m * 32 + i * 8 + (lane >> 5) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          z[4 * i + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[4 * i + j], scale, -l4[j] * kLog2e));
          dp[4 * i + j] -= d4[j];
        }
      }
      if (!see_all(p, p0, p1, mine, mine + 31)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = sees(p, p0 + i / 4 * 8 + (lane >> 5) * 4 + i % 4, key) ? z[i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] *= z[i];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const i32x4 f = summed(z, i), g = summed(dp, i);
#pragma unroll
        for (int d = 0; d < T::DS; ++d) {
          dv[d] = mma(T::columns(dt, m * 32 + i * 16, d, lane), f, dv[d]);
          dk[d] = mma(T::columns(qt, m * 32 + i * 16, d, lane), g, dk[d]);
        }
      }
    }
  }
  const int64_t to = (at_key * p.kv_heads + kv) * p.dim;
  T::store(p.dk + to, there, p.dim, lane, dk, p.scale);
  T::store(p.dv + to, there, p.dim, lane, dv, 1.f);
}

// parts of kOwn rows that the sequences have at most, and one at least that is none's: it clears the rows of no sequence
int parts_of(int n_rows, int n_seqs) { return n_rows / kOwn + n_seqs + 1; }

}  // namespace

hipError_t launch_attend_rows(const AttendRowsParams &p, hipStream_t s) {
  const int parts = parts_of(p.n_rows, p.n_seqs);
  const dim3 grid = grid_of(parts, p.heads);
  if (p.dim <= 64) attend_rows_kernel<64><<<grid, kBlock, 0, s>>>(p, parts);
  else attend_rows_kernel<128><<<grid, kBlock, 0, s>>>(p, parts);
  return hipGetLastError();
}

hipError_t launch_attend_rows_backward(const AttendRowsParams &p, hipStream_t s) {
  const int parts = parts_of(p.n_rows, p.n_seqs), k_parts = parts_of(p.n_k_rows, p.n_seqs);
  if (p.dim <= 64) attend_rows_dq_kernel<64><<<grid_of(parts, p.heads), kBlock, 0, s>>>(p, parts);
  else attend_rows_dq_kernel<128><<<grid_of(parts, p.heads), kBlock, 0, s>>>(p, parts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.dim <= 64) attend_rows_dkv_kernel<64><<<grid_of(k_parts, p.kv_heads), kBlock, 0, s>>>(p, k_parts);
  else attend_rows_dkv_kernel<128><<<grid_of(k_parts, p.kv_heads), kBlock, 0, s>>>(p, k_parts);
  return hipGetLastError();
}

}  // namespace moe
