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
// P and dZ are rounded to bf16 for the matrix cores.  The error that this makes is as large as that of the results' own rounding
// (dK and dV 0.0023 of their size together, 0.0017 for the results' alone).  For dQ dZ is taken in two parts: the errors of one part
// are added up with keys that have much in common, their share of the query's direction, while the dZ themselves cancel (0.0024 to 0.0027;
// two parts are a third of the products more, 386 to 403 us of 8192 tokens, all in all).  For dK, where they would not fit into the registers,
// only where queries do not see all keys of a tile: all of a short sequence.  delta is the same for all keys of
// a query, and with Y as it is rounded it would be the next largest part of the error: the forward keeps what the rounding of Y leaves,
// in bf16.
//
// Which sequence and which of its rows a workgroup has is worked out from the offsets on the device.  Loads go through buffer
// resources that end where the sequence ends: what lies beyond arrives as zeros.
//
// Measured: 16384 tokens, 32 heads of 128, 8 of k: 2080 to 2200 us, from card to card (1.06 to 1.00 PFLOP/s).  With gradients, on the slower of
// these, 8192 tokens in five sequences, 16 heads of 128: 107 + 149 + 181 + 6 us (0.61, 0.88, 0.73 PFLOP/s of the products that each makes);
// 20001 tokens in nine, 16 heads of 80, 2 of k, window 1000 and three first keys: 191 + 240 + 264 + 16.  16384 tokens: the matrix cores work 42 % of the time and the vector units as much again,
// with two wavefronts a SIMD (what the registers allow).  Tried for the forward, of 2115 us: the same without the two steps 2120; matrix
// instructions at a higher wave priority the same; 64 queries a wavefront and one of them a SIMD, half the reads of LDS, 2490.
#include <algorithm>
#include <type_traits>

#include "attend.h"
#include "row_range.h"
#include "rows.h"
#include "tiles.h"

namespace moe {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kBlock = kWaves * 64;
constexpr int kOwn = 32 * kWaves;  // rows of a workgroup
constexpr int kTile = 64;          // rows of the other side in LDS
constexpr uint32_t kNowhere = 0xc0000000u;  // behind every tile, and with what is added to it still within 32 bits
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
  const RowRange q = row_range(p.offsets[s], p.offsets[s + 1], p.n_rows), k = row_range(p.k_offsets[s], p.k_offsets[s + 1], p.n_k_rows);
  return {q.first, q.count, k.first, k.count, k.count - q.count};
}
// Part `want` of the sequences' rows in parts of OWN, later parts of the sequences first: they have more keys, and a workgroup with
// much to do must not be the last to begin.  No such part: sequence -1, and how far behind the last one it is (-1: it is not).
struct Part {
  int sequence, part, over;
  Sequence s;
};
template <int OWN = kOwn>
__device__ __forceinline__ Part part_of(const AttendRowsParams &p, int want) {
  const int lane = threadIdx.x & 63;
  if (p.n_seqs <= 64) {
    const Sequence mine = lane < p.n_seqs ? sequence_of(p, lane) : Sequence{0, 0, 0, 0, 0};
    const int n = (mine.nq + OWN - 1) / OWN;
    const auto from_on = [&](int part) { return of_lane(sum_upto(max(n - part, 0)), 63); };  // parts `part` .. of all sequences
    const int all = from_on(0);
    if (want >= all) return {-1, 0, want - all, {}};
    int at = 0, step = 1;  // the last part with `want` or fewer ahead of it and its like
    while (from_on(step) > want) step *= 2;
    for (; step > 0; step /= 2) at += from_on(at + step) > want ? step : 0;
    const int ahead = from_on(at + 1), upto = sum_upto(n > at ? 1 : 0);
    const int l = uniform(__builtin_ctzll(__ballot(upto > want - ahead)));
    return {l, uniform(at), 0, {of_lane(mine.q0, l), of_lane(mine.nq, l), of_lane(mine.k0, l), of_lane(mine.nk, l), of_lane(mine.ahead, l)}};
  }
  // More sequences: nobody adds up what is ahead of each.  Sequence s has the numbers from offsets[s] / OWN + s on, of which it needs no
  // more than there are up to the next sequence's first; the others stay idle.  The sequence is found 64 at a time.  (1000 sequences of
  // 10000 rows in all, 16 heads of 128 over 8: 168 us, 244 with the sequences' parts added up 64
  // at a time; with the gradients 581, 736.)
  const auto first_of = [&](int s) { return row_within(p.offsets[s], p.n_rows) / OWN + s; };
  int from = 0, to = p.n_seqs;  // the last one whose numbers begin at `want` or ahead of it is among these
  while (from < to) {
    const int step = (to - from + 63) / 64, s = from + (lane + 1) * step;
    const int n = __popcll(__ballot(s <= to && first_of(min(s, to)) <= want));
    from += n * step;
    to = min(from + step - 1, to);
  }
  from = uniform(from);
  const int over = uniform(want - first_of(from));
  if (from == p.n_seqs) return {-1, 0, over, {}};
  const Sequence s = sequence_of(p, from);
  const int n = (s.nq + OWN - 1) / OWN;
  if (over < 0 || over >= n) return {-1, 0, -1, {}};
  return {from, n - 1 - over, 0, s};
}
// zeros for the rows of no sequence, shared by `step` workgroups
__device__ __forceinline__ void clear_rows(const int32_t *offsets, int n_seqs, int n_rows, uint16_t *to, int head, int heads, int dim, int at, int step) {
  const int first = row_within(offsets[0], n_rows), last = max(row_within(offsets[n_seqs], n_rows), first);
  const int64_t units = (int64_t)(first + n_rows - last) * (dim / 8);
  for (int64_t u = (int64_t)at * kBlock + threadIdx.x; u < units; u += (int64_t)step * kBlock) {
    int64_t r = u / (dim / 8);
    if (r >= first) r += last - first;
    *reinterpret_cast<rows_u32x4 *>(to + (r * heads + head) * dim + u % (dim / 8) * 8) = rows_u32x4{0, 0, 0, 0};
  }
}

__device__ __forceinline__ uint32_t lds_at(const uint8_t *p) { return (uint32_t)reinterpret_cast<uintptr_t>(LDS_PTR(void, p)); }
// Rows of up to KS * 16 values in LDS, 128 or 256 bytes each.  Chunk c of row r lies at c ^ f(r): both kinds of reads (16 rows at one chunk; 8 rows of four chunks,
// transposed) spread over all banks
template <int STEPS>
struct Tiles {
  static constexpr int KS = STEPS, DS = (KS + 1) / 2;  // steps of 16 over the dims, blocks of 32 of them
  static constexpr int ROW = KS <= 4 ? 128 : 256, CHUNKS = ROW / 16, ROWS_LOAD = 64 / CHUNKS;
  static constexpr int BYTES = kTile * ROW, LOADS = BYTES / 1024 / kWaves;  // of a wavefront for a tile
  static __device__ __forceinline__ int swap(int r) { return CHUNKS == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3); }

  // Where the lane's first load of a tile comes from: the row and the chunk in bytes.  Load i is ROWS_LOAD rows further on, its
  // chunk exchanged with another number.
  struct Source {
    uint32_t row, chunk;
  };
  static __device__ __forceinline__ Source source(int wave, int lane, int64_t token) {
    const int r = wave * LOADS * ROWS_LOAD + lane / CHUNKS;
    return {(uint32_t)r * (uint32_t)token * 2, (uint32_t)((lane % CHUNKS) ^ swap(r)) * 16};
  }
  // the tile's rows from `from` on, `rows` of them (or fewer than none)
  static __device__ __forceinline__ void request(Source s, const uint16_t *from, int rows, int64_t token, int dim, int wave, uint8_t *to) {
    const i32x4 b = words_of(from, rows > 0 ? (uint32_t)((min(rows, kTile) - 1) * (uint32_t)token * 2 + dim * 2) : 0u);
    asm("" : "+v"(s.row), "+v"(s.chunk));  // (hidden, see Reader)
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t c = s.chunk ^ (i * (ROW == 256 ? 16 : 32));
      to_lds(b, c < (uint32_t)dim * 2 ? s.row + c : kNowhere, (uint32_t)i * ROWS_LOAD * (uint32_t)token * 2, to + (wave * LOADS + i) * 1024);
    }
  }
  // 32 rows by one wavefront alone; s: source of wavefront 0
  static constexpr int LOADS32 = 32 / ROWS_LOAD;
  static __device__ __forceinline__ void request32(const Source &s, const uint16_t *from, int rows, int64_t token, int dim, uint8_t *to) {
    const i32x4 b = words_of(from, rows > 0 ? (uint32_t)((min(rows, 32) - 1) * (uint32_t)token * 2 + dim * 2) : 0u);
#pragma unroll
    for (int i = 0; i < LOADS32; ++i) {
      const uint32_t c = s.chunk ^ (ROW == 256 ? (i & 3) * 16 : (i & 1) * 32);
      to_lds(b, c < (uint32_t)dim * 2 ? s.row + c : kNowhere, (uint32_t)i * ROWS_LOAD * (uint32_t)token * 2, to + i * 1024);
    }
  }
  // Where the lane reads in a tile: of 32 rows at one chunk (step s over the dims: at ^ s * 32), transposed of 4 rows of four
  // chunks (block d of the dims: at ^ d * 64; the rows 8 further on: at ^ 32).  What is read follows from these with one operation.
  // hide: from the compiler, which would hold all of them in registers where there are none left.
  struct Reader {
    uint32_t rows, columns;
    __device__ __forceinline__ Reader(uint32_t tile, const Reader &lane, bool hide) : rows(tile + lane.rows), columns(tile + lane.columns) {
      if (hide) asm("" : "+v"(rows), "+v"(columns));
    }
    __device__ __forceinline__ Reader(int lane) {
      rows = (lane & 31) * ROW + (((lane >> 5) ^ swap(lane & 31)) * 16);
      const int r = 4 * (lane >> 5) + ((lane & 15) >> 2), c = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
      columns = r * ROW + ((c ^ swap(r)) * 16) + (lane & 1) * 8;
    }
  };
  // rows r0 .. r0 + 31 as rows of a product, step s over the dims; `in` bytes behind the tile
  static __device__ __forceinline__ i32x4 rows(const Reader &a, uint32_t in, int r0, int s) {
    return *(LDS_PTR(i32x4, (uintptr_t)((a.rows ^ (s * 32)) + in + r0 * ROW)));
  }
  // dims d * 32 .. as rows of a product, summed over the 16 rows from r0 on
  static __device__ __forceinline__ i32x4 columns(const Reader &a, uint32_t in, int r0, int d) {
    const uint32_t at = a.columns ^ (d * 64);
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, (uintptr_t)(at + in + r0 * ROW)));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, (uintptr_t)((at ^ 32) + in + (r0 + 8) * ROW)));
    return __builtin_bit_cast(i32x4, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
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
  // the lane's column of a result, times v; low: and what its rounding leaves, unless nullptr
  static __device__ __forceinline__ void store(uint16_t *at, uint16_t *low, bool there, int dim, int lane, const f32x16 (&o)[DS], float v) {
    // Of 16 dims a lane has four, then four 8 further on; its other half has those in between.  They exchange four: 16 bytes each.
    const auto put = [&](uint16_t *to, int d, int i, const uint32_t (&w)[4]) MOE_ROWS_INLINE {
      const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
      const int c = d * 32 + i * 16 + (lane >> 5) * 8;
      if (there && c < dim) *reinterpret_cast<rows_u32x4 *>(to + c) = rows_u32x4{a[0], b[0], a[1], b[1]};
    };
#pragma unroll
    for (int d = 0; d < DS; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t w[4], l[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x = o[d][8 * i + 2 * k] * v, y = o[d][8 * i + 2 * k + 1] * v;
          w[k] = pack_bf16(x, y);
          l[k] = pack_bf16(x - bf16_lo(w[k]), y - bf16_hi(w[k]));
        }
        put(at, d, i, w);
        if (low) put(low, d, i, l);
      }
  }
  // ... in 32 bits
  static __device__ __forceinline__ void store_sums(float *at, bool there, int dim, int lane, const f32x16 (&o)[DS]) {
#pragma unroll
    for (int d = 0; d < DS; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = d * 32 + i * 8 + (lane >> 5) * 4;
        if (there && c < dim) *reinterpret_cast<f32x4 *>(at + c) = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
      }
  }
};
__device__ __forceinline__ float largest(const f32x16 &z) {
  float m = z[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = fmaxf(m, z[i]);
  return m;
}
// rows 16 t .. of a result as the summed side of the next product
__device__ __forceinline__ i32x4 summed(const f32x16 &p, int t) {
  i32x4 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = (int)pack_bf16(p[8 * t + 2 * i], p[8 * t + 2 * i + 1]);
  return f;
}

// what the rounding of rows 16 t .. of it leaves
__device__ __forceinline__ i32x4 left_over(const f32x16 &p, int t) {
  i32x4 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = p[8 * t + 2 * i], b = p[8 * t + 2 * i + 1];
    const uint32_t r = pack_bf16(a, b);
    f[i] = (int)pack_bf16(a - bf16_lo(r), b - bf16_hi(r));
  }
  return f;
}
// Where some queries do not see a key, its exponential is 0, but a product with an infinity or NaN would not be: the forward looks for
// such values wherever something is masked, and adds them apart.  (The backward does not: its kernels have no registers left for it.)
enum { kPlusInf = 0, kMinusInf = 1, kNotANumber = 2 };
template <typename F>
__device__ __forceinline__ i32x4 each_bf16(const i32x4 &c, F f) {  // f of each value's bits
  i32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = c[i];
    r[i] = (int)(f(two & 0xffffu) | f(two >> 16) << 16);
  }
  return r;
}
__device__ __forceinline__ i32x4 finite_of(const i32x4 &c) {
  return each_bf16(c, [](uint32_t v) { return (v & 0x7f80u) == 0x7f80u ? 0u : v; });
}
__device__ __forceinline__ i32x4 ones_where(const i32x4 &c, int kind) {
  return each_bf16(c, [kind](uint32_t v) {
    const bool is = kind == kPlusInf ? v == 0x7f80u : kind == kMinusInf ? v == 0xff80u : (v & 0x7fffu) > 0x7f80u;
    return is ? 0x3f80u : 0u;
  });
}
// whether any of 32 rows of a tile holds an infinity or NaN
template <typename T>
__device__ __forceinline__ bool odd_rows(const typename T::Reader &at, uint32_t in) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 most = {0, 0};
#pragma unroll
  for (int s = 0; s < T::KS; ++s) {
    const i32x4 x = T::rows(at, in, 0, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = x[i] & 0x7fff7fff;
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, two));
    }
  }
  return __any(max(most[0], most[1]) >= 0x7f80);
}
// rows 16 t .. of what `seen` has a bit for, as 1 and 0
__device__ __forceinline__ i32x4 ones_of(uint32_t seen, int t) {
  i32x4 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = (int)((seen >> (8 * t + 2 * i) & 1) * 0x3f80u | (seen >> (8 * t + 2 * i + 1) & 1) * 0x3f800000u);
  return f;
}
// o + the product of 32 rows' columns with f, in which a row that holds an infinity or NaN counts where `seen` has a bit (register i of
// the lane: bit i).
template <typename T>
__device__ __forceinline__ void add_apart(const typename T::Reader &at, uint32_t in, const i32x4 (&f)[2], uint32_t seen, f32x16 (&o)[T::DS]) {
#pragma unroll
  for (int d = 0; d < T::DS; ++d) {
    o[d] += mma(finite_of(T::columns(at, in, 16, d)), f[1], mma(finite_of(T::columns(at, in, 0, d)), f[0], zero16()));
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
      const f32x16 n = mma(ones_where(T::columns(at, in, 16, d), kind), ones_of(seen, 1), mma(ones_where(T::columns(at, in, 0, d), kind), ones_of(seen, 0), zero16()));
      const float value = kind == kNotANumber ? NAN : kind == kPlusInf ? INFINITY : -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] += n[i] > 0.f ? value : 0.f;
    }
  }
}
// sum + the values of f, as they are rounded
__device__ __forceinline__ float add_up(float sum, const i32x4 &f) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int two = f[i];  // (a bit cast of f[i] itself takes element 0 of f, whatever i is)
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3f803f80), sum, false);
  }
  return sum;
}

struct Item {
  int part, head;  // behind the last one: no part
};
// Workgroups go to the XCDs in turn, and each XCD has an L2 of its own: where eight divides the heads of k, an XCD has all
// workgroups of some of them.  (One of these heads after the other, so that fewer are in the L2 at a time, makes the workgroups end less
// evenly: 8192 tokens, 16 heads of 128, with gradients 395 us, that way 415.)
__device__ __forceinline__ Item item_of(int heads, int kv_heads, int lead = 0) {
  Item r;
  const uint32_t b = (uint32_t)row_group() - lead;
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
dim3 grid_of(int64_t parts, int heads, int lead = 0) {
  const RowGrid g = row_grid(parts * heads + lead);
  return dim3(g.x, g.y);
}

// the tiles of keys that the queries r0 .. r1 of a sequence see, in turn
struct KeyTiles {
  int sink_tiles, first, n;
  int begin;  // a share's first one
  __device__ __forceinline__ int at(int t) const { return (t + begin < sink_tiles ? t + begin : first + t + begin - sink_tiles) * kTile; }
  __device__ __forceinline__ void cut(int share, int of) {
    const int all = n;
    begin = uniform((int)((int64_t)all * share / of));
    n = uniform((int)((int64_t)all * (share + 1) / of)) - begin;
  }
};
__device__ __forceinline__ KeyTiles key_tiles(const AttendRowsParams &p, const Sequence &s, int r0, int r1) {
  KeyTiles k;
  const int lo = p.window > 0 ? max(r0 + s.ahead - p.window + 1, 0) : 0, end = max(r1 + s.ahead + 1, 0);
  const int last = (end + kTile - 1) / kTile;
  k.first = lo / kTile;
  k.sink_tiles = min((min(p.sinks, lo) + kTile - 1) / kTile, k.first);
  k.n = k.sink_tiles + max(last - k.first, 0);
  k.begin = 0;
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

// What a wavefront has of its 32 queries.  Y is divided by the sum of the exponentials as they are rounded, so that the rounding of
// one that outweighs the others cancels (the error of Y 0.0022 of its size otherwise); KEEP: lse is of the sum in 32 bits, since the
// backward takes the exponentials anew.
template <int KS, bool KEEP>
struct Queries {
  using T = Tiles<KS>;
  i32x4 q[T::KS];
  f32x16 o[T::DS];
  float top, most, sum, rounded, scale;  // most: the largest score that is new, of the lane's own keys; the others to the base 2

  __device__ __forceinline__ void begin(float s) {
#pragma unroll
    for (int d = 0; d < T::DS; ++d) o[d] = zero16();
    top = most = -INFINITY;
    sum = rounded = 0.f;
    scale = s;
  }
  // The base of the exponentials follows the largest score (of the query's two lanes) when that is `slack` ahead (to the base 2): until
  // then nothing is multiplied and no lane asks the other one.  No slack: the largest exponential is 1, which has no rounding, and
  // that counts for queries that see few keys.
  __device__ __forceinline__ void rebase(float slack) {
    if (__any(most * scale > top + slack)) {
      const float to = fmaxf(top, fmaxf(most, __shfl_xor(most, 32)) * scale), shrink = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - to);
      top = to;
      if (KEEP) sum *= shrink;
      rounded *= shrink;
#pragma unroll
      for (int d = 0; d < T::DS; ++d) o[d] *= shrink;
    }
  }
  // 32 keys from `key` on by themselves; the queries are at positions p0 .. p1, the lane's at pos
  __device__ __forceinline__ void add(const AttendRowsParams &p, const typename T::Reader &keys, const typename T::Reader &values, int p0, int p1, int pos, int key, int lane) {
    f32x16 z = zero16();
#pragma unroll
    for (int i = 0; i < T::KS; ++i) z = mma(T::rows(keys, 0, 0, i), q[i], z);
    bool odd = false;
    uint32_t seen = 0;
    if (!see_all(p, p0, p1, key, key + 31)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool is = sees(p, pos, key + i / 4 * 8 + (lane >> 5) * 4 + i % 4);
        seen |= is ? 1u << i : 0u;
        z[i] = is ? z[i] : -INFINITY;
      }
      odd = odd_rows<T>(values, 0);
    }
    most = largest(z);
    rebase(0.f);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      z[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], scale, -base));
      if (KEEP) sum += z[i];
    }
    const i32x4 f[2] = {summed(z, 0), summed(z, 1)};
    rounded = add_up(add_up(rounded, f[0]), f[1]);
    if (odd) {
      add_apart<T>(values, 0, f, seen, o);
      return;
    }
#pragma unroll
    for (int i = 0; i < 2 * T::DS; ++i) o[i % T::DS] = mma(T::columns(values, 0, i / T::DS * 16, i % T::DS), f[i / T::DS], o[i % T::DS]);
  }
  // z: the scores of 32 keys that all see, `most` the largest.  next: those of the 32 keys at `keys`.
  __device__ __forceinline__ void step(f32x16 &z, f32x16 &next, const typename T::Reader &keys, const typename T::Reader &values) {
    rebase(8.f);
    const float base = top == -INFINITY ? 0.f : top;  // (all scores so far -infinity: their exponentials are 0)
    constexpr int EACH = (16 + T::KS - 1) / T::KS, PVS = 2 * T::DS, AHEAD = 3;
    i32x4 a[AHEAD + 1], c[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) a[i] = T::rows(keys, 0, 0, i);
    next = zero16();
#pragma unroll
    for (int i = 0; i < T::KS; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i + AHEAD < T::KS) a[(i + AHEAD) % (AHEAD + 1)] = T::rows(keys, 0, 0, i + AHEAD);
      else c[i + AHEAD - T::KS] = T::columns(values, 0, (i + AHEAD - T::KS) / T::DS * 16, (i + AHEAD - T::KS) % T::DS);
      next = mma(a[i % (AHEAD + 1)], q[i], next);
#pragma unroll
      for (int e = i * EACH; e < (i + 1) * EACH && e < 16; ++e) {
        z[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[e], scale, -base));
        if (KEEP) sum += z[e];
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    const i32x4 f[2] = {summed(z, 0), summed(z, 1)};
    most = -INFINITY;
#pragma unroll
    for (int i = 0; i < PVS; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i + AHEAD < PVS) c[(i + AHEAD) % (AHEAD + 1)] = T::columns(values, 0, (i + AHEAD) / T::DS * 16, (i + AHEAD) % T::DS);
      o[i % T::DS] = mma(c[i % (AHEAD + 1)], f[i / T::DS], o[i % T::DS]);
      if (i < 2) rounded = add_up(rounded, f[i]);
      if (i >= PVS - 4) {
#pragma unroll
        for (int e = (i - PVS + 4) * 4; e < (i - PVS + 5) * 4; ++e) most = fmaxf(most, next[e]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
};

// Tiles that all of a workgroup's queries see go in two steps per 32 keys, in which matrix instructions and others do not wait for
// each other: the scores of the next 32 keys while the exponentials of these are taken, and the product with the values while the
// largest of the next scores is found.  The other tiles (the diagonal, a window's edge, first keys) are computed one by one and masked.
// Tiles are requested two ahead; there is one barrier for each, in its middle or at its end, and values have three places in LDS.
// SPLIT: few queries, many keys.  The tiles are cut into p.splits shares, each a workgroup's, and what it has goes to the workspace.
// (32 heads of 128, 8 of k: 100 queries behind 8000 tokens 36 us, with 32 queries a workgroup and no shares 72; 512 behind 8000: 63, 88, where the
// products alone take 46; four times 4 behind up to 9000: 60, 150.  8 heads, 2000 tokens: 33, 46.  Below some 1500 keys it
// does not pay: 8 heads, 1000 tokens 24.5, 20.6; 300 queries with a window of 1000: 20.8, 15.2.)
template <int KS, bool KEEP, bool SPLIT>
__global__ __launch_bounds__(kBlock, 2) void attend_rows_kernel(const AttendRowsParams p, const int parts) {
  using T = Tiles<KS>;
  __shared__ __align__(256) uint8_t lds[5 * T::BYTES];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  Item item = item_of(p.heads, p.kv_heads);
  const int place = item.part, share = SPLIT ? uniform(place % p.splits) : 0;
  if (SPLIT) item.part = uniform(place / p.splits);
  if (item.part >= parts) return;
  const Part part = part_of(p, item.part);
  if (part.sequence < 0) {
    if (part.over >= 0 && share == 0)
      clear_rows(p.offsets, p.n_seqs, p.n_rows, p.y, item.head, p.heads, p.dim, part.over, parts - (item.part - part.over));
    return;
  }
  const Sequence s = part.s;
  const int r0 = part.part * kOwn, r1 = min(r0 + kOwn, s.nq) - 1, mine = r0 + wave * 32, row = mine + (lane & 31);
  const int p0 = mine + s.ahead, p1 = min(mine + 31, r1) + s.ahead, pos = row + s.ahead;
  const int kv = item.head / (p.heads / p.kv_heads);
  KeyTiles tiles = key_tiles(p, s, r0, r1);
  if (SPLIT) tiles.cut(share, p.splits);
  const uint16_t *k = static_cast<const uint16_t *>(p.k.at) + s.k0 * p.k.token + kv * p.k.head;
  const uint16_t *v = static_cast<const uint16_t *>(p.v.at) + s.k0 * p.v.token + kv * p.v.head;
  const typename T::Source ks = T::source(wave, lane, p.k.token), vs = T::source(wave, lane, p.v.token);
  const uint32_t lds0 = lds_at(lds);
  uint32_t v_put = 2 * T::BYTES, v_at = lds0 + 2 * T::BYTES;
  const auto request = [&](int t) MOE_ROWS_INLINE {
    const int key = tiles.at(t), rows = s.nk - key;
    T::request(ks, k + key * p.k.token, rows, p.k.token, p.dim, wave, lds + (t & 1) * T::BYTES);
    T::request(vs, v + key * p.v.token, rows, p.v.token, p.dim, wave, lds + v_put);
    v_put = v_put == 4 * T::BYTES ? 2 * T::BYTES : v_put + T::BYTES;
  };
  Queries<KS, KEEP> w;
  T::own(static_cast<const uint16_t *>(p.q.at) + (s.q0 + min(row, s.nq - 1)) * p.q.token + item.head * p.q.head, row < s.nq, p.dim, lane, w.q);
  w.begin(p.scale * kLog2e);
  const typename T::Reader reader(lane);
  const auto at = [&](uint32_t tile) MOE_ROWS_INLINE { return typename T::Reader(tile, reader, false); };
  const auto next_tile = [&](int t) MOE_ROWS_INLINE {
    if (t + 1 < tiles.n) {
      landed_but<0>();
      if (t + 2 < tiles.n) request(t + 2);
    }
  };
  const auto next_values = [&] { v_at = v_at == lds0 + 4 * T::BYTES ? lds0 + 2 * T::BYTES : v_at + T::BYTES; };
  const auto tile_alone = [&](int t) MOE_ROWS_INLINE {
#pragma unroll 1
    for (int m = 0; m < 2; ++m) {
      const int key = tiles.at(t) + 32 * m;
      if (mine > r1 || see_none(p, p0, p1, key, key + 31)) continue;
      w.add(p, at(lds0 + (t & 1) * T::BYTES + 32 * m * T::ROW), at(v_at + 32 * m * T::ROW), p0, p1, pos, key, lane);
    }
    next_tile(t);
    next_values();
  };

  if (tiles.n > 0) {
    request(0);
    if (tiles.n > 1) {
      request(1);
      landed_but<2 * T::LOADS>();
    } else {
      landed_but<0>();
    }
    // tiles from..to - 1 are seen by all
    const int w0 = r0 + s.ahead, w1 = r1 + s.ahead;
    const int to = min(max(tiles.sink_tiles + (w0 + 1) / kTile - tiles.first - tiles.begin, 0), tiles.n);
    const int from = p.window > 0 ? min(max(tiles.sink_tiles + max((max(w1 - p.window + 1, 0) + kTile - 1) / kTile - tiles.first, 0) - tiles.begin, 0), to) : 0;
    const int fast = min(to, tiles.n - 1);  // (the last one looks ahead in vain, unless there is nothing behind it)
    int t = 0;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {
      for (const int end = round == 0 && from < fast ? from : tiles.n; t < end; ++t) tile_alone(t);
      if (t >= fast) continue;
      f32x16 za = zero16(), zb;
      const typename T::Reader keys = at(lds0 + (t & 1) * T::BYTES);
#pragma unroll
      for (int i = 0; i < T::KS; ++i) za = mma(T::rows(keys, 0, 0, i), w.q[i], za);
      w.most = largest(za);
      for (; t < fast; ++t) {
        w.step(za, zb, at(lds0 + (t & 1) * T::BYTES + 32 * T::ROW), at(v_at));
        next_tile(t);
        w.step(zb, za, at(lds0 + (~t & 1) * T::BYTES), at(v_at + 32 * T::ROW));
        next_values();
      }
    }
  }
  const bool there = row < s.nq;
  const float total = w.rounded + __shfl_xor(w.rounded, 32);
  if (SPLIT) {
    w.sum += __shfl_xor(w.sum, 32);
    const int64_t at = ((int64_t)place * p.heads + item.head) * kOwn + wave * 32 + (lane & 31);
    T::store_sums(p.sums + at * p.dim, there, p.dim, lane, w.o);
    if (there && lane < 32) *reinterpret_cast<f32x4 *>(p.stats + at * 4) = f32x4{w.top, total, w.sum, 0.f};
    return;
  }
  const int64_t dense = ((int64_t)(s.q0 + row) * p.heads + item.head) * p.dim;
  T::store(p.y + dense, p.low ? p.low + dense : nullptr, there, p.dim, lane, w.o, total > 0.f || total != total ? 1.f / total : 0.f);
  if (KEEP) w.sum += __shfl_xor(w.sum, 32);
  if (KEEP && there && lane < 32) p.lse[(int64_t)item.head * p.n_rows + s.q0 + row] = w.top * kLn2 + __logf(w.sum);
}

// What the shares of the keys have; a workgroup has kJoinRows of the queries of a part, a thread eight dims of one of them.
constexpr int kJoinRows = 16;
__global__ __launch_bounds__(kBlock) void join_rows_kernel(const AttendRowsParams p, const int parts) {
  const int b = blockIdx.x, row0 = b % (kOwn / kJoinRows) * kJoinRows, head = b / (kOwn / kJoinRows) % p.heads, at = b / (kOwn / kJoinRows) / p.heads;
  const Part part = part_of(p, at);
  if (at >= parts || part.sequence < 0) return;
  const int first = part.part * kOwn + row0, rows = min(kJoinRows, part.s.nq - first), chunks = p.dim / 8;
  for (int u = threadIdx.x; u < rows * chunks; u += kBlock) {
    const int r = u / chunks, c = u % chunks * 8;
    const int64_t from = ((int64_t)at * p.splits * p.heads + head) * kOwn + row0 + r, step = (int64_t)p.heads * kOwn;
    float top = -INFINITY, total = 0.f, sum = 0.f;
    f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    constexpr int AT_ONCE = 4;  // shares whose loads are under way together
    for (int i0 = 0; i0 < p.splits; i0 += AT_ONCE) {
      f32x4 of[AT_ONCE], y[AT_ONCE][2];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const int64_t share = from + min(i0 + i, p.splits - 1) * step;
        of[i] = *reinterpret_cast<const f32x4 *>(p.stats + share * 4);
        if (i0 + i >= p.splits) of[i] = f32x4{-INFINITY, 0.f, 0.f, 0.f};
        y[i][0] = *reinterpret_cast<const f32x4 *>(p.sums + share * p.dim + c);
        y[i][1] = *reinterpret_cast<const f32x4 *>(p.sums + share * p.dim + c + 4);
      }
      float to = top;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) to = fmaxf(to, of[i][0]);
      const float base = to == -INFINITY ? 0.f : to, shrink = __builtin_amdgcn_exp2f(top - base);
      top = to;
      total *= shrink;
      sum *= shrink;
      x[0] *= shrink;
      x[1] *= shrink;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        // (Nothing of it is seen, or all scores are -infinity.  If they are NaN the largest is -infinity, too, but the sum is NaN.)
        if (of[i][0] == -INFINITY && of[i][1] == 0.f) continue;
        const float weight = __builtin_amdgcn_exp2f(of[i][0] - base);
        total += weight * of[i][1];
        sum += weight * of[i][2];
        x[0] += weight * y[i][0];
        x[1] += weight * y[i][1];
      }
    }
    const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
    const int64_t dense = ((int64_t)(part.s.q0 + first + r) * p.heads + head) * p.dim + c;
    rows_u32x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v0 = x[i / 2][i % 2 * 2] * inv, v1 = x[i / 2][i % 2 * 2 + 1] * inv;
      hi[i] = pack_bf16(v0, v1);
      lo[i] = pack_bf16(v0 - bf16_lo(hi[i]), v1 - bf16_hi(hi[i]));
    }
    *reinterpret_cast<rows_u32x4 *>(p.y + dense) = hi;
    if (p.low) *reinterpret_cast<rows_u32x4 *>(p.low + dense) = lo;
    if (p.lse && c == 0) p.lse[(int64_t)head * p.n_rows + part.s.q0 + first + r] = top * kLn2 + __logf(sum);
  }
}

// Few queries: a workgroup has 32, and each of its wavefronts a quarter of the keys, 32 at a time in turn, in a ring of its own; what
// they have is joined through LDS.
template <int KS, bool KEEP>
__global__ __launch_bounds__(kBlock, 1) void attend_few_rows_kernel(const AttendRowsParams p, const int parts) {
  using T = Tiles<KS>;
  constexpr int HALF = 32 * T::ROW, PITCH = T::ROW / 2 + 4;  // bytes of 32 rows; floats of a query's sums
  static_assert(kWaves * 32 * (PITCH + 4) * 4 <= kWaves * 4 * HALF, "the sums go where the rings were");
  __shared__ __align__(256) uint8_t lds[kWaves * 4 * HALF];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Item item = item_of(p.heads, p.kv_heads);
  if (item.part >= parts) return;
  const Part part = part_of<32>(p, item.part);
  if (part.sequence < 0) {
    if (part.over >= 0)
      clear_rows(p.offsets, p.n_seqs, p.n_rows, p.y, item.head, p.heads, p.dim, part.over, parts - (item.part - part.over));
    return;
  }
  const Sequence s = part.s;
  const int r0 = part.part * 32, r1 = min(r0 + 32, s.nq) - 1, row = r0 + (lane & 31), p0 = r0 + s.ahead, p1 = r1 + s.ahead, pos = row + s.ahead;
  const int kv = item.head / (p.heads / p.kv_heads);
  const KeyTiles tiles = key_tiles(p, s, r0, r1);
  const uint16_t *k = static_cast<const uint16_t *>(p.k.at) + s.k0 * p.k.token + kv * p.k.head;
  const uint16_t *v = static_cast<const uint16_t *>(p.v.at) + s.k0 * p.v.token + kv * p.v.head;
  const typename T::Source ks = T::source(0, lane, p.k.token), vs = T::source(0, lane, p.v.token);
  uint8_t *mine = lds + wave * 4 * HALF;
  const auto key_of = [&](int u) { return tiles.at(u >> 1) + (u & 1) * 32; };
  const auto request = [&](int u, int place) MOE_ROWS_INLINE {  // (behind the last one: nothing, which arrives as zeros)
    const int key = u < 2 * tiles.n ? key_of(u) : 0, rows = u < 2 * tiles.n ? s.nk - key : 0;
    T::request32(ks, k + key * p.k.token, rows, p.k.token, p.dim, mine + place * 2 * HALF);
    T::request32(vs, v + key * p.v.token, rows, p.v.token, p.dim, mine + place * 2 * HALF + HALF);
  };
  Queries<KS, KEEP> w;
  T::own(static_cast<const uint16_t *>(p.q.at) + (s.q0 + min(row, s.nq - 1)) * p.q.token + item.head * p.q.head, row < s.nq, p.dim, lane, w.q);
  w.begin(p.scale * kLog2e);
  const typename T::Reader reader(lane);
  request(wave, 0);
  request(wave + kWaves, 1);
  int place = 0;
  for (int u = wave; u < 2 * tiles.n; u += kWaves, place ^= 1) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * T::LOADS32) : "memory");
    const int key = key_of(u);
    if (!see_none(p, p0, p1, key, key + 31)) {
      const uint32_t at = lds_at(mine) + place * 2 * HALF;
      w.add(p, typename T::Reader(at, reader, false), typename T::Reader(at + HALF, reader, false), p0, p1, pos, key, lane);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    request(u + 2 * kWaves, place);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  w.rounded += __shfl_xor(w.rounded, 32);
  if (KEEP) w.sum += __shfl_xor(w.sum, 32);
  float *sums = reinterpret_cast<float *>(lds), *stats = sums + kWaves * 32 * PITCH;  // [wave][query][dim], [wave][query][3]
#pragma unroll
  for (int d = 0; d < T::DS; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = d * 32 + i * 8 + (lane >> 5) * 4;
      *reinterpret_cast<f32x4 *>(sums + (wave * 32 + (lane & 31)) * PITCH + c) = f32x4{w.o[d][4 * i], w.o[d][4 * i + 1], w.o[d][4 * i + 2], w.o[d][4 * i + 3]};
    }
  if (lane < 32) {
    float *at = stats + (wave * 32 + lane) * 3;
    at[0] = w.top;
    at[1] = w.rounded;
    at[2] = w.sum;
  }
  __syncthreads();
  // eight threads a query
  const int r = threadIdx.x >> 3, place8 = threadIdx.x & 7;
  if (r0 + r >= s.nq) return;
  float top = -INFINITY, total = 0.f, sum = 0.f, weight[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) top = fmaxf(top, stats[(i * 32 + r) * 3]);
  const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    weight[i] = __builtin_amdgcn_exp2f(stats[(i * 32 + r) * 3] - base);
    total += weight[i] * stats[(i * 32 + r) * 3 + 1];
    sum += weight[i] * stats[(i * 32 + r) * 3 + 2];
  }
  const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
  const int64_t dense = ((int64_t)(s.q0 + r0 + r) * p.heads + item.head) * p.dim;
  for (int c = place8 * 8; c < p.dim; c += 64) {
    rows_u32x4 hi, lo;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) x += weight[i] * *reinterpret_cast<const f32x4 *>(sums + (i * 32 + r) * PITCH + c + 4 * h);
      x *= inv;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t two = pack_bf16(x[2 * i], x[2 * i + 1]);
        hi[2 * h + i] = two;
        lo[2 * h + i] = pack_bf16(x[2 * i] - bf16_lo(two), x[2 * i + 1] - bf16_hi(two));
      }
    }
    *reinterpret_cast<rows_u32x4 *>(p.y + dense + c) = hi;
    if (p.low) *reinterpret_cast<rows_u32x4 *>(p.low + dense + c) = lo;
  }
  if (KEEP && place8 == 0) p.lse[(int64_t)item.head * p.n_rows + s.q0 + r0 + r] = top * kLn2 + __logf(sum);
}

// ---- the gradients of k and v: how their work is cut ------------------------------------------------------------
// The queries that see any of kOwn keys, tile by tile, and that for each head of the group, are a list.  Lists are long and few
// where few heads of k serve many of q, or where first keys stay visible: a list of more than half as many tiles again as a
// workgroup's equal share is cut into pieces of about a share, whose sums, in 32 bits, are added up in order by a launch of its own.
// (A piece costs as much as some eight tiles, 128 rows of sums to memory and back, but where few lists leave compute units idle, a
// list's tiles one after the other take longer: 1193 tokens, 4 heads of 112 for 1, with all else: shares of 16 tiles at least 115 us, 8 77, 4 61,
// 2 63; 2005 tokens, 16 heads of 64: 54, 54, 50, 52.)  There are 512 shares of wide heads, as many as the
// GPU holds workgroups at once, and more of narrow heads, whose sums are smaller (16384 tokens, 4 heads of 64 for 16, with all else: 512
// shares 538, 768 499, 1024 481 us; 8192 tokens, 16 heads of 128: 401, 404, 441; 20001 tokens, 2 heads of 80 for 16, window: 669, 663, 659).
inline int shares_of(int dim) { return std::min(std::max(65536 / dim, 512), 1024); }
constexpr int kLeast = 4;     // tiles of a share at least
constexpr int kLead = 8;       // workgroups ahead of those with rows in the launch that plans: one plans, and each XCD has one
struct List {
  int first, end, tiles;  // query rows of the sequence, from a tile's first row on; tiles of one head
};
__device__ __forceinline__ List list_of(const AttendRowsParams &p, const Sequence &s, int part) {
  const int k0 = part * kOwn, k1 = min(k0 + kOwn, s.nk) - 1;
  List l;
  l.first = max(k0 - s.ahead, 0) / kTile * kTile;
  l.end = p.window > 0 && k0 >= p.sinks ? (int)min((int64_t)s.nq, (int64_t)k1 + p.window - s.ahead) : s.nq;
  l.tiles = max((l.end - l.first + kTile - 1) / kTile, 0);
  return l;
}
// of the threads of the workgroup up to this one, and of all
template <typename V>
__device__ __forceinline__ V block_upto(V v, V *waves, V &all) {
  const V upto = sum_upto(v);
  if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = upto;
  __syncthreads();
  V before = 0;
  all = 0;
  for (int w = 0; w < kWaves; ++w) {
    before += w < (int)(threadIdx.x >> 6) ? waves[w] : 0;
    all += waves[w];
  }
  __syncthreads();
  return before + upto;
}
// The pieces, long ones first (in kSizes classes).  Three passes over the parts of the keys: their tiles, how many pieces of each size,
// where each goes.
constexpr int kSizes = 64;
__device__ __forceinline__ void plan_pieces(const AttendRowsParams &p, uint8_t *lds) {
  int64_t *waves = reinterpret_cast<int64_t *>(lds);
  int64_t *past = waves + kWaves;                              // parts of the chunk's sequences up to and with each
  int *sizes = reinterpret_cast<int *>(past + kBlock);         // pieces of a size, then where the next one of it goes
  const int per = p.heads / p.kv_heads, tid = threadIdx.x;
  int64_t total = 0, share = 0, all;
  if (tid < kSizes) sizes[tid] = 0;
  for (int pass = 0; pass < 3; ++pass) {
    int64_t slots = 0, left = p.max_pieces;
    for (int s0 = 0; s0 < p.n_seqs; s0 += kBlock) {
      const int64_t n = s0 + tid < p.n_seqs ? (sequence_of(p, s0 + tid).nk + kOwn - 1) / kOwn : 0;
      int64_t parts;
      past[tid] = block_upto(n, waves, parts);
      parts = min(parts, left);  // (all of them, unless sequences overlap)
      left -= parts;
      __syncthreads();
      for (int64_t u0 = 0; u0 < parts; u0 += kBlock) {
        const int64_t u = u0 + tid;
        int at = 0, part = 0, tiles = 0;
        if (u < parts) {
#pragma unroll
          for (int o = kBlock / 2; o > 0; o >>= 1) at += past[at + o - 1] <= u ? o : 0;
          part = (int)(u - (at > 0 ? past[at - 1] : 0));
          tiles = list_of(p, sequence_of(p, s0 + at), part).tiles * per;
        }
        if (pass == 0) {
          total += tiles;
          continue;
        }
        int n = u < parts ? 1 : 0;
        if (2 * (int64_t)tiles > 3 * share) n = (int)((tiles + share - 1) / share);
        const int64_t slot = slots + block_upto((int64_t)(n > 1 ? n : 0), waves, all) - n;
        slots += all;
        if (n > 1 && slot + n > p.max_slots) n = 1;  // (only where sequences overlap)
        if (n == 0) continue;
        const int size = kSizes - 1 - (int)min((int64_t)tiles / n * kSizes / (3 * share / 2 + 1), (int64_t)kSizes - 1);
        const int piece = atomicAdd(&sizes[size], n);  // (the order of equals changes no result)
        if (pass == 1) continue;
        for (int i = 0; i < n; ++i) {
          const int from = (int)((int64_t)tiles * i / n), to = (int)((int64_t)tiles * (i + 1) / n);
          if (piece + i < p.max_pieces) p.pieces[piece + i] = KeyPiece{s0 + at, part, from, to - from, i, n, (int)slot};
        }
      }
      __syncthreads();
    }
    if (pass == 0) {
      block_upto(total, waves, all);
      share = max((all * p.kv_heads + p.shares - 1) / p.shares, (int64_t)kLeast);
    } else if (pass == 1 && tid < 64) {
      const int n = sizes[tid], upto = sum_upto(n);
      sizes[tid] = upto - n;
      if (tid == kSizes - 1) *p.n_pieces = min(upto, p.max_pieces);
    }
    __syncthreads();
  }
}

// Products of the backward.  What they read of LDS is requested AHEAD steps before its use, in this order; left to
// itself the compiler reads right ahead of each use and waits (gradients of k and v, dims of 80: 300 us, so 262; with dims of 128 they have
// no registers left for it: 165, with what then goes to memory 318).
// z + 32 rows with x, dp + the 32 rows of the tile behind it with y
template <typename T, int AHEAD>
__device__ __forceinline__ void two_products(const typename T::Reader &at, const i32x4 (&x)[T::KS], const i32x4 (&y)[T::KS], f32x16 &z, f32x16 &dp) {
  i32x4 a[AHEAD + 1], b[AHEAD + 1];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    a[i] = T::rows(at, 0, 0, i);
    b[i] = T::rows(at, T::BYTES, 0, i);
  }
#pragma unroll
  for (int i = 0; i < T::KS; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < T::KS) {
      a[(i + AHEAD) % (AHEAD + 1)] = T::rows(at, 0, 0, i + AHEAD);
      b[(i + AHEAD) % (AHEAD + 1)] = T::rows(at, T::BYTES, 0, i + AHEAD);
    }
    z = mma(a[i % (AHEAD + 1)], x[i], z);
    dp = mma(b[i % (AHEAD + 1)], y[i], dp);
  }
  __builtin_amdgcn_sched_barrier(0);
}
// o + 32 rows' columns with f
template <typename T, int AHEAD>
__device__ __forceinline__ void add_columns(const typename T::Reader &at, uint32_t in, const i32x4 (&f)[2], f32x16 (&o)[T::DS]) {
  i32x4 c[AHEAD + 1];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) c[i] = T::columns(at, in, i / T::DS * 16, i % T::DS);
#pragma unroll
  for (int i = 0; i < 2 * T::DS; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < 2 * T::DS) c[(i + AHEAD) % (AHEAD + 1)] = T::columns(at, in, (i + AHEAD) / T::DS * 16, (i + AHEAD) % T::DS);
    o[i % T::DS] = mma(c[i % (AHEAD + 1)], f[i / T::DS], o[i % T::DS]);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// ... and with g
template <typename T, int AHEAD>
__device__ __forceinline__ void add_columns_twice(const typename T::Reader &at, uint32_t in, const i32x4 (&f)[2], const i32x4 (&g)[2], f32x16 (&o)[T::DS]) {
  i32x4 c[AHEAD + 1];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) c[i] = T::columns(at, in, i / T::DS * 16, i % T::DS);
#pragma unroll
  for (int i = 0; i < 2 * T::DS; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < 2 * T::DS) c[(i + AHEAD) % (AHEAD + 1)] = T::columns(at, in, (i + AHEAD) / T::DS * 16, (i + AHEAD) % T::DS);
    o[i % T::DS] = mma(c[i % (AHEAD + 1)], f[i / T::DS], o[i % T::DS]);
    o[i % T::DS] = mma(c[i % (AHEAD + 1)], g[i / T::DS], o[i % T::DS]);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// SPLIT: few queries, many keys, as in the forward; the sums of a share's keys go to the workspace.  (With all else: 2000 tokens, 8 heads of 128
// for 2, 133 us, without shares 161; 1000 of 8 heads 80, 94; 400 54, 59; 3529 behind up to 12135, 2 heads: 244, 466.)
template <int KS, bool SPLIT>
__global__ __launch_bounds__(kBlock, 2) void attend_rows_dq_kernel(const AttendRowsParams p, const int parts) {
  using T = Tiles<KS>;
  __shared__ __align__(256) uint8_t lds[4 * T::BYTES];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  if (row_group() < kLead) {
    if (row_group() == 0) plan_pieces(p, lds);
    return;
  }
  Item item = item_of(p.heads, p.kv_heads, kLead);
  const int place = item.part, share = SPLIT ? uniform(place % p.splits) : 0;
  if (SPLIT) item.part = uniform(place / p.splits);
  if (item.part >= parts) return;
  const Part part = part_of(p, item.part);
  if (part.sequence < 0) {
    if (part.over >= 0 && share == 0)
      clear_rows(p.offsets, p.n_seqs, p.n_rows, p.dq, item.head, p.heads, p.dim, part.over, parts - (item.part - part.over));
    return;
  }
  const Sequence s = part.s;
  const int r0 = part.part * kOwn, r1 = min(r0 + kOwn, s.nq) - 1, mine = r0 + wave * 32, row = mine + (lane & 31);
  const int p0 = mine + s.ahead, p1 = min(mine + 31, r1) + s.ahead, pos = row + s.ahead;
  const int kv = item.head / (p.heads / p.kv_heads);
  KeyTiles tiles = key_tiles(p, s, r0, r1);
  if (SPLIT) tiles.cut(share, p.splits);
  const uint16_t *k = static_cast<const uint16_t *>(p.k.at) + s.k0 * p.k.token + kv * p.k.head;
  const uint16_t *v = static_cast<const uint16_t *>(p.v.at) + s.k0 * p.v.token + kv * p.v.head;
  const typename T::Source ks = T::source(wave, lane, p.k.token), vs = T::source(wave, lane, p.v.token);
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
    if (p.low) {
      T::own(p.low + dense, there, p.dim, lane, y);
#pragma unroll
      for (int i = 0; i < T::KS; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) delta += bf16_lo(y[i][w]) * bf16_lo(dy[i][w]) + bf16_hi(y[i][w]) * bf16_hi(dy[i][w]);
    }
    delta += __shfl_xor(delta, 32);
  }
  T::own(static_cast<const uint16_t *>(p.q.at) + at_row * p.q.token + item.head * p.q.head, there, p.dim, lane, q);
  const float lse = p.lse[(int64_t)item.head * p.n_rows + at_row] * kLog2e, scale = p.scale * kLog2e;
  if (there && lane < 32 && share == 0) {
    p.stats[(int64_t)item.head * p.n_rows + at_row] = -lse;
    p.stats[(int64_t)(p.heads + item.head) * p.n_rows + at_row] = -delta;
  }
  f32x16 less_delta;  // what dP begins with
#pragma unroll
  for (int i = 0; i < 16; ++i) less_delta[i] = -delta;
  f32x16 o[T::DS];
#pragma unroll
  for (int d = 0; d < T::DS; ++d) o[d] = zero16();
  const typename T::Reader reader(lane);
  if (tiles.n > 0) request(0);
  for (int t = 0; t < tiles.n; ++t) {
    landed_but<0>();
    if (t + 1 < tiles.n) request(t + 1);
    const int key = tiles.at(t);
    if (mine > r1) continue;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int key0 = key + m * 32;
      if (see_none(p, p0, p1, key0, key0 + 31)) continue;
      const typename T::Reader at(lds_at(lds) + (t & 1) * 2 * T::BYTES + m * 32 * T::ROW, reader, false);
      f32x16 z = zero16(), dp = less_delta;
      two_products<T, 2>(at, q, dy, z, dp);
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], scale, -lse)) * dp[i];
      if (!see_all(p, p0, p1, key0, key0 + 31)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = sees(p, pos, key0 + i / 4 * 8 + (lane >> 5) * 4 + i % 4) ? z[i] : 0.f;
      }
      const i32x4 f[2] = {summed(z, 0), summed(z, 1)}, low[2] = {left_over(z, 0), left_over(z, 1)};
      add_columns_twice<T, 3>(at, 0, f, low, o);
    }
  }
  if (SPLIT) {
    T::store_sums(p.q_sums + (((int64_t)place * p.heads + item.head) * kOwn + wave * 32 + (lane & 31)) * p.dim, there, p.dim, lane, o);
    return;
  }
  T::store(p.dq + dense, nullptr, there, p.dim, lane, o, p.scale);
}

template <int KS>
__global__ __launch_bounds__(kBlock, 2) void attend_rows_dkv_kernel(const AttendRowsParams p, const int parts) {
  using T = Tiles<KS>;
  __shared__ __align__(256) uint8_t lds[4 * T::BYTES + 4 * kTile * 4];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Item item = item_of(p.kv_heads, p.kv_heads);
  if (item.part >= parts) return;
  const int kv = item.head, per = p.heads / p.kv_heads, n_pieces = *p.n_pieces;
  if (item.part >= n_pieces) {
    clear_rows(p.k_offsets, p.n_seqs, p.n_k_rows, p.dk, kv, p.kv_heads, p.dim, item.part - n_pieces, parts - n_pieces);
    clear_rows(p.k_offsets, p.n_seqs, p.n_k_rows, p.dv, kv, p.kv_heads, p.dim, item.part - n_pieces, parts - n_pieces);
    return;
  }
  const KeyPiece piece = p.pieces[item.part];
  const Sequence s = sequence_of(p, piece.sequence);
  const int k0 = piece.part * kOwn, k1 = min(k0 + kOwn, s.nk) - 1, mine = k0 + wave * 32, key = mine + (lane & 31);
  const bool there = key < s.nk;
  const List list = list_of(p, s, piece.part);
  const int first = list.first, end = list.end, all = piece.count;
  const typename T::Source qs = T::source(wave, lane, p.q.token), ds = T::source(wave, lane, (int64_t)p.heads * p.dim);
  uint8_t *stats = lds + 4 * T::BYTES;
  // the heads one after the other, their tiles in turn
  int next_head = kv * per + (all > 0 ? piece.first / list.tiles : 0), next_row = first + (all > 0 ? piece.first % list.tiles * kTile : 0);
  const auto request = [&](int t) MOE_ROWS_INLINE {
    const int head = next_head, row = next_row, rows = s.nq - row;
    next_row += kTile;
    if (next_row >= end) {
      next_row = first;
      ++next_head;
    }
    uint8_t *to = lds + (t & 1) * 2 * T::BYTES;
    T::request(qs, static_cast<const uint16_t *>(p.q.at) + (int64_t)(s.q0 + row) * p.q.token + head * p.q.head, rows, p.q.token, p.dim, wave, to);
    T::request(ds, p.dy + ((int64_t)(s.q0 + row) * p.heads + head) * p.dim, rows, (int64_t)p.heads * p.dim, p.dim, wave, to + T::BYTES);
    const int64_t at = (int64_t)head * p.n_rows + s.q0 + row;
    if (wave < 2) word_to_lds(words_of(p.stats + (wave == 0 ? at : at + (int64_t)p.heads * p.n_rows), (uint32_t)min(rows, kTile) * 4), lane * 4, stats + ((t & 1) * 2 + wave) * kTile * 4);
  };
  i32x4 k[T::KS], v[T::KS];
  const int64_t at_key = s.k0 + min(key, s.nk - 1);
  T::own(static_cast<const uint16_t *>(p.k.at) + at_key * p.k.token + kv * p.k.head, there, p.dim, lane, k);
  T::own(static_cast<const uint16_t *>(p.v.at) + at_key * p.v.token + kv * p.v.head, there, p.dim, lane, v);
  f32x16 dk[T::DS], dv[T::DS];
#pragma unroll
  for (int d = 0; d < T::DS; ++d) dk[d] = dv[d] = zero16();
  const float scale = p.scale * kLog2e;
  const typename T::Reader reader(lane);
  int row = next_row;
  if (all > 0) request(0);
  for (int t = 0; t < all; ++t, row = row + kTile < end ? row + kTile : first) {
    landed_but<0>();
    if (t + 1 < all) request(t + 1);
    const float *less_lse = reinterpret_cast<const float *>(stats + (t & 1) * 2 * kTile * 4), *less_delta = less_lse + kTile;
    if (mine > k1) continue;
#pragma unroll 1
    for (int m = 0; m < 2; ++m) {
      const int row0 = row + m * 32, p0 = row0 + s.ahead, p1 = min(row0 + 31, s.nq - 1) + s.ahead;
      if (row0 >= s.nq || see_none(p, p0, p1, mine, mine + 31)) continue;
      const typename T::Reader at(lds_at(lds) + (t & 1) * 2 * T::BYTES + m * 32 * T::ROW, reader, true);
      f32x16 z = zero16(), dp;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 d4 = *reinterpret_cast<const f32x4 *>(less_delta + m * 32 + i * 8 + (lane >> 5) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) dp[4 * i + j] = d4[j];
      }
      if constexpr (KS < 8) {
        two_products<T, 2>(at, k, v, z, dp);
      } else {
#pragma unroll
        for (int i = 0; i < T::KS; ++i) {
          z = mma(T::rows(at, 0, 0, i), k[i], z);
          dp = mma(T::rows(at, T::BYTES, 0, i), v[i], dp);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 l4 = *reinterpret_cast<const f32x4 *>(less_lse + m * 32 + i * 8 + (lane >> 5) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[4 * i + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[4 * i + j], scale, l4[j]));
      }
      bool again = !see_all(p, p0, p1, mine, mine + 31);
      if (again) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = sees(p, p0 + i / 4 * 8 + (lane >> 5) * 4 + i % 4, key) ? z[i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] *= z[i];
      const i32x4 f[2] = {summed(z, 0), summed(z, 1)};
      if constexpr (KS < 8) {
        add_columns<T, 3>(at, T::BYTES, f, dv);
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int d = 0; d < T::DS; ++d) dv[d] = mma(T::columns(at, T::BYTES, i * 16, d), f[i], dv[d]);
      }
      i32x4 g[2] = {summed(dp, 0), summed(dp, 1)}, low[2];
      if (again) {
        low[0] = left_over(dp, 0);
        low[1] = left_over(dp, 1);
      }
#pragma unroll 1
      for (;; again = false) {
        if constexpr (KS < 8) {
          add_columns<T, 3>(at, 0, g, dk);
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int d = 0; d < T::DS; ++d) dk[d] = mma(T::columns(at, 0, i * 16, d), g[i], dk[d]);
        }
        if (!again) break;
        g[0] = low[0];
        g[1] = low[1];
      }
    }
  }
  if (piece.of > 1) {
    float *sums = p.sums + (((int64_t)(piece.slot + piece.index) * p.kv_heads + kv) * kOwn + key - k0) * 2 * p.dim;
    T::store_sums(sums, there, p.dim, lane, dk);
    T::store_sums(sums + p.dim, there, p.dim, lane, dv);
    return;
  }
  const int64_t to = (at_key * p.kv_heads + kv) * p.dim;
  T::store(p.dk + to, nullptr, there, p.dim, lane, dk, p.scale);
  T::store(p.dv + to, nullptr, there, p.dim, lane, dv, 1.f);
}

// The sums of the pieces of a list, in order; a workgroup has kJoinRows of its keys.  The first `ahead` workgroups: the shares of the
// gradients of q, kJoinRows queries each.
__global__ __launch_bounds__(kBlock) void join_pieces_kernel(const AttendRowsParams p, const int ahead) {
  uint32_t b = (uint32_t)row_group();
  if ((int)b < ahead) {
    const int strip = b % (kOwn / kJoinRows), head = b / (kOwn / kJoinRows) % p.heads, at = b / (kOwn / kJoinRows) / p.heads;
    const Part part = part_of(p, at);
    if (part.sequence < 0) return;
    const int first = part.part * kOwn + strip * kJoinRows, rows = min(kJoinRows, part.s.nq - first), quads = p.dim / 4;
    const int64_t step = (int64_t)p.heads * kOwn * p.dim;
    for (int u = threadIdx.x; u < rows * quads; u += kBlock) {
      const int r = u / quads, c = u % quads * 4;
      const float *from = p.q_sums + (((int64_t)at * p.splits * p.heads + head) * kOwn + strip * kJoinRows + r) * p.dim + c;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      for (int i = 0; i < p.splits; ++i) v += *reinterpret_cast<const f32x4 *>(from + i * step);
      v *= p.scale;
      *reinterpret_cast<rows_u32x2 *>(p.dq + ((int64_t)(part.s.q0 + first + r) * p.heads + head) * p.dim + c) = rows_u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
    return;
  }
  b -= ahead;
  const int strip = b % (kOwn / kJoinRows), kv = b / (kOwn / kJoinRows) % p.kv_heads, at = b / (kOwn / kJoinRows) / p.kv_heads;
  if (at >= *p.n_pieces) return;
  const KeyPiece piece = p.pieces[at];
  if (piece.of < 2 || piece.index > 0) return;
  const Sequence s = sequence_of(p, piece.sequence);
  const int row0 = strip * kJoinRows, rows = min(kJoinRows, s.nk - piece.part * kOwn - row0), quads = p.dim / 4;
  for (int u = threadIdx.x; u < rows * 2 * quads; u += kBlock) {
    const int r = row0 + u / (2 * quads), c = u % (2 * quads);
    const float *from = p.sums + (((int64_t)piece.slot * p.kv_heads + kv) * kOwn + r) * 2 * p.dim + c * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < piece.of; ++i) v += *reinterpret_cast<const f32x4 *>(from + (int64_t)i * p.kv_heads * kOwn * 2 * p.dim);
    if (c < quads) v *= p.scale;
    const int64_t to = ((int64_t)(s.k0 + piece.part * kOwn + r) * p.kv_heads + kv) * p.dim + c % quads * 4;
    *reinterpret_cast<rows_u32x2 *>((c < quads ? p.dk : p.dv) + to) = rows_u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
}

// parts of `own` rows that the sequences have at most, and one at least that is none's: it clears the rows of no sequence
int parts_of(int n_rows, int n_seqs, int own = kOwn) { return n_rows / own + n_seqs + 1; }

// keys of a query, at most
int64_t seen_of(const AttendRowsParams &p) { return p.window > 0 ? (int64_t)p.window + p.sinks + kOwn : p.n_k_rows; }
// Into how many shares the keys of kOwn queries are cut: 1 unless a sequence has `many` keys that are seen, and then so many that there
// are as many workgroups as the GPU holds at once, with `least` keys each or more.
constexpr int kMostShares = 512;
int shares_of_keys(int n_rows, int n_k_rows, int n_seqs, int heads, int64_t seen, int least, int many) {
  if (n_seqs == 0 || n_rows == 0) return 1;
  seen = std::min<int64_t>(n_k_rows / n_seqs, seen);
  if (seen < many) return 1;
  const int64_t real = std::max<int64_t>(parts_of(n_rows, n_seqs) - 1, 1) * heads;
  return (int)std::max<int64_t>(std::min(kMostShares / real, seen / least), 1);
}

// f(steps over the dims): as many as there are, or the next more that there is a kernel for
template <typename F>
void with_steps(int dim, F f) {
  if (dim <= 64) f(std::integral_constant<int, 4>());
  else if (dim <= 80) f(std::integral_constant<int, 5>());
  else if (dim <= 96) f(std::integral_constant<int, 6>());
  else f(std::integral_constant<int, 8>());
}

}  // namespace

constexpr int kFew = 128;        // workgroups of kOwn queries up to which a wavefront takes a quarter of the keys instead
struct ForwardSpace {
  int splits;
  int64_t sums, bytes;  // where they begin
};
constexpr int kShareKeys = 256, kManyKeys = 1500;  // of a sequence: for a share of them at least; for there to be any
static ForwardSpace forward_space(int n_rows, int n_k_rows, int n_seqs, int heads, int dim, int64_t seen) {
  ForwardSpace w{shares_of_keys(n_rows, n_k_rows, n_seqs, heads, seen, kShareKeys, kManyKeys), 0, 0};
  if (w.splits == 1) return w;
  const int64_t rows = (int64_t)parts_of(n_rows, n_seqs) * w.splits * heads * kOwn;
  w.sums = rows * 16;
  w.bytes = w.sums + rows * dim * 4;
  return w;
}
size_t attend_rows_bytes(int n_rows, int n_k_rows, int n_seqs, int heads, int dim) { return forward_space(n_rows, n_k_rows, n_seqs, heads, dim, n_k_rows).bytes; }

hipError_t launch_attend_rows(const AttendRowsParams &given, uint8_t *workspace, hipStream_t s) {
  AttendRowsParams p = given;
  const int parts = parts_of(p.n_rows, p.n_seqs);
  const ForwardSpace w = forward_space(p.n_rows, p.n_k_rows, p.n_seqs, p.heads, p.dim, seen_of(p));
  if (w.splits > 1) {
    p.splits = w.splits;
    p.stats = reinterpret_cast<float *>(workspace);
    p.sums = reinterpret_cast<float *>(workspace + w.sums);
    with_steps(p.dim, [&](auto ks) {
      attend_rows_kernel<decltype(ks)::value, true, true><<<grid_of((int64_t)parts * w.splits, p.heads), kBlock, 0, s>>>(p, parts);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    join_rows_kernel<<<(parts - 1) * p.heads * (kOwn / kJoinRows), kBlock, 0, s>>>(p, parts - 1);
    return hipGetLastError();
  }
  with_steps(p.dim, [&](auto ks) {
    constexpr int KS = decltype(ks)::value;
    if ((int64_t)parts * p.heads <= kFew) {
      const int few = parts_of(p.n_rows, p.n_seqs, 32);
      if (p.lse) attend_few_rows_kernel<KS, true><<<grid_of(few, p.heads), kBlock, 0, s>>>(p, few);
      else attend_few_rows_kernel<KS, false><<<grid_of(few, p.heads), kBlock, 0, s>>>(p, few);
      return;
    }
    if (p.lse) attend_rows_kernel<KS, true, false><<<grid_of(parts, p.heads), kBlock, 0, s>>>(p, parts);
    else attend_rows_kernel<KS, false, false><<<grid_of(parts, p.heads), kBlock, 0, s>>>(p, parts);
  });
  return hipGetLastError();
}

// The workspace: what the gradients of k and v need of each query, the pieces, their sums.  A list of n tiles is cut if n > 1.5 shares, into n / share + 1 pieces at most, so that
// there are 5 / 3 pieces of lists that are cut for each of all lists' shares.
struct BackwardSpace {
  int64_t pieces, sums, q_sums, bytes;  // where they begin
  int max_pieces, max_slots, splits;
};
constexpr int kShareKeysDq = 128, kManyKeysDq = 256;
static BackwardSpace backward_space(int n_rows, int n_k_rows, int n_seqs, int heads, int kv_heads, int dim, int64_t seen) {
  BackwardSpace w;
  const int parts = parts_of(n_k_rows, n_seqs);
  const int64_t list = (int64_t)(heads / kv_heads) * ((n_rows + kTile - 1) / kTile);  // tiles, at most
  const int64_t shares = std::min<int64_t>(shares_of(dim), list * (parts - 1) * kv_heads / kLeast + 1);
  w.max_slots = 2 * list > 3 * kLeast ? (int)(5 * shares / (3 * kv_heads) + 1) : 0;
  w.max_pieces = parts + (w.max_slots > 0 ? shares_of(dim) / kv_heads + 1 : 0);
  const auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
  w.pieces = up((int64_t)n_rows * heads * 8);
  w.sums = up(w.pieces + 16 + (int64_t)w.max_pieces * sizeof(KeyPiece));
  w.q_sums = w.sums + (int64_t)w.max_slots * kv_heads * kOwn * 2 * dim * 4;
  w.splits = shares_of_keys(n_rows, n_k_rows, n_seqs, heads, seen, kShareKeysDq, kManyKeysDq);
  w.bytes = w.q_sums + (w.splits > 1 ? (int64_t)parts_of(n_rows, n_seqs) * w.splits * heads * kOwn * dim * 4 : 0);
  return w;
}
size_t attend_rows_backward_bytes(int n_rows, int n_k_rows, int n_seqs, int heads, int kv_heads, int dim) {
  return backward_space(n_rows, n_k_rows, n_seqs, heads, kv_heads, dim, n_k_rows).bytes;
}

hipError_t launch_attend_rows_backward(const AttendRowsParams &given, uint8_t *workspace, hipStream_t s) {
  AttendRowsParams p = given;
  const BackwardSpace w = backward_space(p.n_rows, p.n_k_rows, p.n_seqs, p.heads, p.kv_heads, p.dim, seen_of(p));
  p.stats = reinterpret_cast<float *>(workspace);
  p.n_pieces = reinterpret_cast<int32_t *>(workspace + w.pieces);
  p.pieces = reinterpret_cast<KeyPiece *>(workspace + w.pieces + 16);
  p.sums = reinterpret_cast<float *>(workspace + w.sums);
  p.q_sums = reinterpret_cast<float *>(workspace + w.q_sums);
  p.splits = w.splits;
  p.max_pieces = w.max_pieces;
  p.shares = shares_of(p.dim);
  p.max_slots = w.max_slots;
  const int parts = parts_of(p.n_rows, p.n_seqs), k_parts = w.max_pieces + 1;
  with_steps(p.dim, [&](auto ks) {
    constexpr int KS = decltype(ks)::value;
    if (w.splits > 1) attend_rows_dq_kernel<KS, true><<<grid_of((int64_t)parts * w.splits, p.heads, kLead), kBlock, 0, s>>>(p, parts);
    else attend_rows_dq_kernel<KS, false><<<grid_of(parts, p.heads, kLead), kBlock, 0, s>>>(p, parts);
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  with_steps(p.dim, [&](auto ks) { attend_rows_dkv_kernel<decltype(ks)::value><<<grid_of(k_parts, p.kv_heads), kBlock, 0, s>>>(p, k_parts); });
  e = hipGetLastError();
  if (e != hipSuccess || (w.max_slots == 0 && w.splits == 1)) return e;
  const int ahead = w.splits > 1 ? (parts - 1) * p.heads * (kOwn / kJoinRows) : 0, behind = w.max_slots > 0 ? w.max_pieces * (kOwn / kJoinRows) : 0;
  join_pieces_kernel<<<grid_of(behind, p.kv_heads, ahead), kBlock, 0, s>>>(p, ahead);
  return hipGetLastError();
}

}  // namespace moe
