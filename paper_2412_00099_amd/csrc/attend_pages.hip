// Attention of one new token per sequence over a cache of pages.
//
//   z_j = scale <q, k_j> over the keys that are seen, y = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m), m the largest so far
//
// Bound by memory: every key and value that is seen is read once.  The heads that share a key are up to 16 columns of a product:
// S^T = K Q^T (rows: keys), O^T = V^T P^T (rows: dims), so that a lane keeps one head throughout, its maximum and its share of the sum
// in registers, and P^T goes from the first product into the second without changing lanes: which keys stand for which summed index
// of the second product is free, as long as V^T is read in the same order.  P is split into two parts of bf16 (what is left of a
// value is 2^-16 of it at most): the second product costs nothing here.  8-bit codes are widened to bf16, which holds them exactly; their
// scales go to the scores and to P.
//
// The work of all sequences is a line of tiles of 32 keys (sequence, group of heads, tile), cut into equal shares, one for each
// wavefront of the launch, whatever the lengths are.  A wavefront keeps a ring of stages of its own in LDS, a stage the keys and
// values of a tile, filled by loads that bypass the registers, and runs from one sequence into the next; no wavefront waits
// for another.  What it has of a (sequence, group) that it does not have whole goes to the workspace: sums, maximum, sum of
// exponentials; a second launch joins these.  Where the table has few pages and there are few (sequence, group)s, a workgroup takes
// one of them whole instead, its wavefronts every eighth tile, and joins through LDS: one launch (777 tokens 10.9 us, in two 12.9).
//
// Two wavefronts a SIMD with half the ring each, rather than one: what a wavefront does with a tile takes longer than its bytes.
// Pass after pass, both launches: four sequences of up to 131072 tokens, 8 heads of 128 for 32, 1.25 GB in 227 us (5.5 TB/s; with one
// wavefront 252); 64 of up to 8192 in 8 bits, 484 MB in 103 (4.7 TB/s; 177); 96 with a window of 4096, 4 heads of 64 for 32, 358 MB in 76
// (4.7 TB/s; 100).  In a trace, each launch by itself: 224 + 7, 114 (100 at least) + 5 and 66 + 5.
#include <algorithm>

#include "attend.h"
#include "rows.h"
#include "tiles.h"

namespace moe {
namespace {

constexpr int kTile = 32;        // keys
constexpr int kWaves = 8;        // of a workgroup: two for each SIMD
constexpr int kGroups = 256;     // workgroups: one for each compute unit
constexpr int kWorkers = kGroups * kWaves;
constexpr int kCols = 16;        // heads of a product
constexpr int kWholeTiles = 64;  // up to so many a workgroup may take a (sequence, group) by itself
constexpr uint32_t kNowhere = 0xf8000000u;

// The workspace: the share of a worker, in tiles; per sequence the place of its first tile on the line; then, for each worker, what
// it has of the (sequence, group) that began ahead of it and of the one that goes on behind it: [heads][dim] and [heads][2]
struct Parts {
  int64_t *share, *start;
  float *sums, *stats;
  int rows;  // heads of a group at most
};
__host__ __device__ inline int group_rows(int heads, int kv_heads) { return heads / kv_heads < kCols ? heads / kv_heads : kCols; }
__host__ __device__ inline int64_t parts_head(int n_seqs) { return ((int64_t)n_seqs + 2) / 2 * 16; }
__device__ __forceinline__ Parts parts_of(const AttendPagesParams &p) {
  Parts r;
  r.rows = group_rows(p.heads, p.c.kv_heads);
  r.share = reinterpret_cast<int64_t *>(p.parts);
  r.start = r.share + 1;
  r.sums = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(p.parts) + parts_head(p.n_seqs));
  r.stats = r.sums + (int64_t)2 * kWorkers * r.rows * p.c.dim;
  return r;
}

typedef const __attribute__((address_space(4))) int32_t *Constant;  // read with scalar loads
__device__ __forceinline__ Constant constant(const int32_t *p) { return (Constant)(uintptr_t)p; }

// What is seen of a sequence: keys below `end` from `lo` on, and those below `sinks`
struct Seen {
  int end, lo, sink_tiles, first, tiles;  // tile t < sink_tiles is tile t of the cache, the others follow from `first` on
};
__device__ __forceinline__ Seen seen_of(const AttendPagesParams &p, int length) {
  Seen s;
  length = max(length, 0);
  s.end = (int)min((int64_t)length, (int64_t)p.table_pages << p.c.page_bits);
  s.lo = p.window > 0 ? max(length - p.window, 0) : 0;
  s.first = s.lo / kTile;
  const int last = (int)(((int64_t)s.end + kTile - 1) / kTile);
  s.sink_tiles = min(min((int)(((int64_t)min(p.sinks, s.lo) + kTile - 1) / kTile), s.first), last);
  s.tiles = s.sink_tiles + max(last - s.first, 0);
  return s;
}

template <int CACHE, int DT, bool WHOLE>
struct Attend {
  static constexpr bool INT8 = CACHE == MOE_R_INT8;
  static constexpr int EL = INT8 ? 1 : 2;
  static constexpr int ROW = DT * EL, CHUNKS = ROW / 16;              // of a key in LDS
  static constexpr int ROWS_LOAD = 64 / CHUNKS, LOADS = kTile / ROWS_LOAD;  // keys of a load, loads of a tile
  static constexpr int MATRIX = kTile * ROW, STAGE = 2 * MATRIX, RING = 16384 / STAGE;
  static constexpr int SCALES = INT8 ? 256 : 0;
  static constexpr int WAVE_LDS = RING * (STAGE + SCALES);
  static constexpr int AHEAD = (INT8 ? 1 : 0);                        // loads of a stage's scales
  static constexpr int KS = DT / 32, DS = DT / 16;                    // steps over the dims, blocks of them

  const AttendPagesParams p;
  uint8_t *lds;
  int lane, l, q, n_groups, per_kv;

  // chunk c of key r lies at c ^ f(r): reads of 16 keys at four chunks, and transposed ones, spread over all banks
  static __device__ __forceinline__ int swap(int r) { return CHUNKS == 16 ? r & 15 : CHUNKS == 8 ? (r >> 1) & 7 : (r >> 2) & 3; }

  struct Spot {
    int seq, group, tile;
    Seen s;
  };
  __device__ __forceinline__ void open(Spot &a) const {
    a.s = seen_of(p, constant(p.lengths)[a.seq]);
  }
  __device__ __forceinline__ void step(Spot &a) const {
    if constexpr (WHOLE) {
      a.tile += kWaves;
      return;
    }
    if (++a.tile < a.s.tiles) return;
    a.tile = 0;
    if (++a.group < n_groups) return;
    a.group = 0;
    do {
      if (++a.seq >= p.n_seqs) return;
      open(a);
    } while (a.s.tiles == 0);
  }
  __device__ __forceinline__ int tile_at(const Spot &a) const {
    return uniform((a.tile < a.s.sink_tiles ? a.tile : a.s.first + a.tile - a.s.sink_tiles) * kTile);
  }
  // the page of 16 keys, -1: none
  __device__ __forceinline__ int page_at(const Spot &a, int pos) const {
    if (pos >= a.s.end) return -1;
    const int id = constant(p.table)[(int64_t)a.seq * p.table_pages + (pos >> p.c.page_bits)];
    return id < p.c.n_pages ? max(id, -1) : -1;
  }

  // A tile that is requested: where its halves of 16 keys begin in the cache (keys and values alike), how many bytes they have
  struct Place {
    int pos, kv;
    bool all;  // every key that is there is seen
    int id[2];
    int64_t from[2];
    uint32_t bytes[2];
  };
  // `there` false: nothing; its loads bring zeros
  __device__ __forceinline__ Place place_of(const Spot &a, bool there) const {
    Place r;
    r.pos = there ? tile_at(a) : 0;
    r.kv = a.group / per_kv;
    r.all = r.pos >= a.s.lo;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int pos = r.pos + 16 * h, id = there ? page_at(a, pos) : -1;
      r.id[h] = id;
      r.from[h] = id < 0 ? 0 : id * p.c.page_stride + (((int64_t)r.kv << p.c.page_bits) + (pos & ((1 << p.c.page_bits) - 1))) * p.c.dim;
      r.bytes[h] = id < 0 ? 0 : min(a.s.end - pos, 16) * p.c.dim * EL;
    }
    return r;
  }
  // Requests its keys or values.  Keys that are not seen arrive as zeros: they may hold anything.
  template <bool VALUES>
  __device__ __forceinline__ void request(const Spot &a, const Place &at, int stage) const {
    uint8_t *to = lds + stage * STAGE + (VALUES ? MATRIX : 0);
    const uint8_t *base = static_cast<const uint8_t *>(VALUES ? p.c.v : p.c.k);
    const int bytes = p.c.dim * EL;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int half = i * ROWS_LOAD / 16, r = i * ROWS_LOAD + lane / CHUNKS, c = ((lane % CHUNKS) ^ swap(r)) * 16;
      uint32_t off = c < bytes ? (uint32_t)((r - half * 16) * bytes + c) : kNowhere;
      if (!at.all && at.pos + r < a.s.lo && at.pos + r >= p.sinks) off = kNowhere;
      to_lds(words_of(base + at.from[half] * EL, at.bytes[half]), off, 0, to + i * 1024);
    }
    if constexpr (INT8 && !VALUES) {
      // lanes 0 .. 31: scales of the keys, the others: of the values.  (Where there are none: any word; it is not used.)
      const int r = lane & 31, pos = at.pos + r;
      const float *from = reinterpret_cast<const float *>(p.lengths);
      if ((r < 16 ? at.bytes[0] : at.bytes[1]) != 0 && pos < a.s.end)
        from = (lane < 32 ? p.c.k_scale : p.c.v_scale) + (((int64_t)(r < 16 ? at.id[0] : at.id[1]) * p.c.kv_heads + at.kv) << p.c.page_bits) + (pos & ((1 << p.c.page_bits) - 1));
      scale_to_lds(from, lds + RING * STAGE + stage * SCALES);
    }
  }
  static __device__ __forceinline__ void scale_to_lds(const float *from, uint8_t *to) {
    const uint32_t at = uniform((uint32_t)reinterpret_cast<uintptr_t>(LDS_PTR(void, to)));
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 3\n\t"
        "global_load_lds_dword %1, off" ::"s"(at), "v"(from)
        : "memory");
  }
  template <int N>
  static __device__ __forceinline__ void landed() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  }
  static __device__ __forceinline__ i32x4 widen(i32x2 c) {  // 8 codes as bf16 (exact: the lower halves of the floats are zero)
    i32x4 v;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const int u = c[w];
      const float f0 = (float)(int8_t)u, f1 = (float)(int8_t)(u >> 8), f2 = (float)(int8_t)(u >> 16), f3 = (float)(u >> 24);
      v[2 * w] = (int)__builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302);
      v[2 * w + 1] = (int)__builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302);
    }
    return v;
  }
  // Two exponentials in two parts each.  Values of bf16 may be infinite, and a part that is 0 or of the other sign would make NaN of
  // them: the first part is cut off rather than rounded, and the second one is of 1 + 2^-22 of the exponential, so that it is above 0
  // where the exponential is (above 2^-104, to be exact).  8-bit values are finite; there the first part is rounded, which leaves half as much.
  static __device__ __forceinline__ i32x2 parts_of_p(float a, float b) {
    constexpr float ABOVE = INT8 ? 1.f : 1.f + 0x1p-22f;
    const uint32_t hi = INT8 ? pack_bf16(a, b) : __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
    return i32x2{(int)hi, (int)pack_bf16(__builtin_fmaf(a, ABOVE, -bf16_lo(hi)), __builtin_fmaf(b, ABOVE, -bf16_hi(hi)))};
  }

  __device__ __forceinline__ void run(int worker, uint8_t *mine) {
    lds = mine;
    lane = threadIdx.x & 63;
    l = lane & 15;
    q = lane >> 4;
    const int per = p.heads / p.c.kv_heads;
    per_kv = (per + kCols - 1) / kCols;
    n_groups = p.c.kv_heads * per_kv;
    Spot now{0, 0, 0, {}};
    int64_t left, begin = 0;
    const Parts parts = parts_of(p);
    if constexpr (WHOLE) {
      now.seq = uniform(blockIdx.x / n_groups);
      now.group = uniform(blockIdx.x % n_groups);
      now.tile = worker % kWaves;
      open(now);
      left = (max(now.s.tiles - now.tile, 0) + kWaves - 1) / kWaves;
    } else {
      // the line, and this worker's share of it
      int64_t all = 0;
      for (int s0 = 0; s0 < p.n_seqs; s0 += 64) all += s0 + lane < p.n_seqs ? seen_of(p, p.lengths[s0 + lane]).tiles : 0;
      all = of_lane(sum_upto(all), 63) * n_groups;
      const int64_t share = max((all + kWorkers - 1) / kWorkers, (int64_t)1);
      begin = worker * share;
      if (worker == 0 && lane == 0) *parts.share = share;
      if (begin >= all) return;
      left = min(share, all - begin);
      int64_t before = 0;
      for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
        const int tiles = s0 + lane < p.n_seqs ? seen_of(p, p.lengths[s0 + lane]).tiles : 0;
        const int64_t past = before + sum_upto((int64_t)tiles) * n_groups;
        const uint64_t behind = __ballot(past > begin);
        if (behind != 0) {
          const int at = __builtin_ctzll(behind), n = of_lane(tiles, at);
          const int64_t in = begin - (of_lane(past, at) - (int64_t)n * n_groups);
          now.seq = uniform(s0 + at);
          now.group = uniform((int)(in / n));
          now.tile = uniform((int)(in % n));
          break;
        }
        before = of_lane(past, 63);
      }
      open(now);
    }
    int64_t line = begin;
    Spot then = now;
    int64_t then_left = left;
    uint32_t halves = 0;  // two bits a stage: which halves of the tiles that are under way there are
    Place to_come;
    // a stage's requests: keys (and scales), values
    const auto look = [&]() MOE_ROWS_INLINE {
      to_come = place_of(then, then_left > 0);
      halves = halves << 2 | (to_come.bytes[0] ? 1 : 0) | (to_come.bytes[1] ? 2 : 0);
    };
    const auto next = [&]() MOE_ROWS_INLINE {
      if (then_left > 0 && --then_left > 0) step(then);
    };
    for (int i = 0; i < RING; ++i) {
      look();
      request<false>(then, to_come, i);
      request<true>(then, to_come, i);
      next();
    }
    // all requests behind those that are waited for
    constexpr int BEHIND = (2 * RING - 1) * LOADS + (RING - 1) * AHEAD, BEHIND_V = (2 * RING - 1) * LOADS + RING * AHEAD;
    f32x4 o[DS];
    i32x4 qf[KS];
    float top = -INFINITY, sum = 0.f;
    const float scale = p.scale * 1.4426950408889634f;  // exponentials to the base 2
    int head0 = 0, heads = 0, stage = 0;
    bool fresh = true, from_start = false;
    for (; left > 0; --left, ++line) {
      if (fresh) {
        const int kv = now.group / per_kv, part = now.group % per_kv;
        head0 = kv * per + part * kCols;
        heads = min(per - part * kCols, kCols);
        from_start = now.tile == 0;
        if (!WHOLE && from_start && now.group == 0 && lane == 0) parts.start[now.seq] = line;
        const uint16_t *qp = static_cast<const uint16_t *>(p.q.at) + now.seq * p.q.token + (head0 + min(l, heads - 1)) * p.q.head;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const int d = INT8 ? ((s >> 1) * 4 + q) * 16 + (s & 1) * 8 : (s * 4 + q) * 8;
          qf[s] = i32x4{0, 0, 0, 0};
          if (l < heads && d < p.c.dim) qf[s] = *reinterpret_cast<const i32x4 *>(qp + d);
        }
#pragma unroll
        for (int d = 0; d < DS; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        top = -INFINITY;
        sum = 0.f;
        fresh = false;
      }
      const uint8_t *kt = lds + stage * STAGE, *vt = kt + MATRIX;
      const float *scales = reinterpret_cast<const float *>(lds + RING * STAGE + stage * SCALES);
      landed<BEHIND>();
      f32x4 z[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        z[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int r = t * 16 + l;
        if constexpr (INT8) {
#pragma unroll
          for (int s = 0; s < KS / 2; ++s) {
            const i32x4 codes = *reinterpret_cast<const i32x4 *>(kt + r * ROW + (((s * 4 + q) ^ swap(r)) * 16));
            z[t] = mma(widen(i32x2{codes[0], codes[1]}), qf[2 * s], z[t]);
            z[t] = mma(widen(i32x2{codes[2], codes[3]}), qf[2 * s + 1], z[t]);
          }
        } else {
#pragma unroll
          for (int s = 0; s < KS; ++s) z[t] = mma(*reinterpret_cast<const i32x4 *>(kt + r * ROW + (((s * 4 + q) ^ swap(r)) * 16)), qf[s], z[t]);
        }
      }
      f32x4 ks[2], vs[2];
      if constexpr (INT8) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          ks[t] = *reinterpret_cast<const f32x4 *>(scales + t * 16 + q * 4);
          vs[t] = *reinterpret_cast<const f32x4 *>(scales + 32 + t * 16 + q * 4);
        }
      }
      const uint32_t there = halves >> (2 * (RING - 1)) & 3;
      const int pos0 = tile_at(now);
      float w[8], most = top;
      bool see[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int pos = pos0 + (i / 4) * 16 + q * 4 + i % 4;
        see[i] = (there >> (i / 4) & 1) && pos < now.s.end && (pos >= now.s.lo || pos < p.sinks);
        w[i] = z[i / 4][i % 4] * scale;
        if constexpr (INT8) w[i] *= ks[i / 4][i % 4];
        w[i] = see[i] ? w[i] : -INFINITY;
        most = fmaxf(most, w[i]);
      }
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      const float base = most == -INFINITY ? 0.f : most, shrink = __builtin_amdgcn_exp2f(top - base);
      top = most;
      sum *= shrink;
      i32x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = __builtin_amdgcn_exp2f(w[i] - base);
        sum += w[i];
        if constexpr (INT8) w[i] = see[i] ? w[i] * vs[i / 4][i % 4] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const i32x2 parts = parts_of_p(w[2 * i], w[2 * i + 1]);
        hi[i] = parts[0];
        lo[i] = parts[1];
      }
#pragma unroll
      for (int d = 0; d < DS; ++d) o[d] *= shrink;
      // (the keys have been read: the products above have waited for them)
      look();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      request<false>(then, to_come, stage);
      landed<BEHIND_V>();
#pragma unroll
      for (int d = 0; d < DS; ++d) {
        i32x4 v;
        if constexpr (INT8) {
          const int r8 = l >> 1, r = (r8 < 4 ? r8 : r8 + 12) + q * 4;
          v = widen(__builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(i32x2, vt + r * ROW + ((d ^ swap(r)) * 16) + (l & 1) * 8)));
        } else {
          const int r = q * 4 + (l >> 2), c = d * 2 + ((l & 3) >> 1), in = (l & 1) * 8;
          const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, vt + r * ROW + ((c ^ swap(r)) * 16) + in));
          const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, vt + (r + 16) * ROW + ((c ^ swap(r + 16)) * 16) + in));
          v = __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        o[d] = mma(v, hi, o[d]);
        o[d] = mma(v, lo, o[d]);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      request<true>(then, to_come, stage);
      next();
      stage = stage + 1 == RING ? 0 : stage + 1;
      const bool ends = now.tile + 1 == now.s.tiles;
      if (!WHOLE && (ends || left == 1)) {
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (from_start && ends) {
          const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
          uint16_t *y = p.y + ((int64_t)now.seq * p.heads + head0 + l) * p.c.dim;
#pragma unroll
          for (int d = 0; d < DS; ++d) {
            const int c = d * 16 + q * 4;
            if (l < heads && c < p.c.dim)
              *reinterpret_cast<rows_u32x2 *>(y + c) = rows_u32x2{pack_bf16(o[d][0] * inv, o[d][1] * inv), pack_bf16(o[d][2] * inv, o[d][3] * inv)};
          }
        } else {
          const int64_t row = ((int64_t)worker * 2 + (from_start ? 1 : 0)) * parts.rows + l;
#pragma unroll
          for (int d = 0; d < DS; ++d) {
            const int c = d * 16 + q * 4;
            if (l < heads && c < p.c.dim) *reinterpret_cast<f32x4 *>(parts.sums + row * p.c.dim + c) = o[d];
          }
          if (l < heads && q == 0) {
            parts.stats[row * 2] = top;
            parts.stats[row * 2 + 1] = sum;
          }
        }
        fresh = true;
      }
      if (left > 1) step(now);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing is under way into LDS when the workgroup ends)
    if constexpr (WHOLE) join(now, fresh, o, top, sum);
  }

  // WHOLE: what the workgroup's wavefronts have of the heads, through LDS.  none: this one has seen no tile.
  __device__ __forceinline__ void join(const Spot &now, bool none, const f32x4 (&o)[DS], float top, float sum) {
    uint8_t *all = lds - (threadIdx.x >> 6) * WAVE_LDS;
    float *sums = reinterpret_cast<float *>(all), *stats = sums + kWaves * kCols * DT;  // [wave][head][dim], [wave][head][2]
    const int wave = threadIdx.x >> 6, heads_of_kv = p.heads / p.c.kv_heads;
    __syncthreads();
    if (none) {
      top = -INFINITY;
      sum = 0.f;
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const int row = wave * kCols + l;
#pragma unroll
    for (int d = 0; d < DS; ++d) *reinterpret_cast<f32x4 *>(sums + row * DT + d * 16 + q * 4) = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[d];
    if (q == 0) {
      stats[row * 2] = top;
      stats[row * 2 + 1] = sum;
    }
    __syncthreads();
    const int h = threadIdx.x / 32, c = threadIdx.x % 32 * 4, head0 = now.group / per_kv * heads_of_kv + now.group % per_kv * kCols;
    if (h >= min(heads_of_kv - now.group % per_kv * kCols, kCols) || c >= p.c.dim) return;
    float most = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, stats[(w * kCols + h) * 2]);
    const float base = most == -INFINITY ? 0.f : most;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float weight = __builtin_amdgcn_exp2f(stats[(w * kCols + h) * 2] - base);
      total += weight * stats[(w * kCols + h) * 2 + 1];
      v += weight * *reinterpret_cast<const f32x4 *>(sums + (w * kCols + h) * DT + c);
    }
    v *= total > 0.f || total != total ? 1.f / total : 0.f;
    *reinterpret_cast<rows_u32x2 *>(p.y + ((int64_t)now.seq * p.heads + head0 + h) * p.c.dim + c) = rows_u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
};

template <int CACHE, int DT, bool WHOLE>
__global__ __launch_bounds__(kWaves * 64, 2) void attend_pages_kernel(const AttendPagesParams p) {
  using A = Attend<CACHE, DT, WHOLE>;
  static_assert(kWaves * kCols * (DT + 2) * 4 <= kWaves * A::WAVE_LDS, "the join's sums go where the rings were");
  __shared__ __align__(16) uint8_t lds[kWaves * A::WAVE_LDS];
  const int wave = uniform(threadIdx.x >> 6);
  A a{p};
  a.run(uniform(blockIdx.x * kWaves) + wave, lds + wave * A::WAVE_LDS);
}

// The parts of each (sequence, head), or zeros where nothing is seen.  A workgroup has `each` heads of a (sequence, group): one where
// few workgroups are to do; kJoinHeads where there are so many that their starts count, most of them for nothing, since the worker that
// had all of a group wrote it.  Few parts are a wavefront's work, many the workgroup's, head by head.  (All in all, 412 sequences of up to 5
// tokens, 48 heads: 21 us, with a workgroup for each head 35; 512 of up to 1000, 16 heads: 113, 120.  20 of up to 16000, 32 heads, have
// long lists of parts: one head each 109, four 114.)
constexpr int kJoinBlock = 256, kJoinWaves = kJoinBlock / 64, kJoinHeads = 4, kFewParts = 16;
constexpr int kJoinMost = 1024;  // workgroups of one head each, at most
__global__ __launch_bounds__(kJoinBlock, 4) void join_pages_kernel(const AttendPagesParams p, const int each) {
  constexpr int STRIPS = kJoinBlock / 32;
  __shared__ float weights[kWorkers], part[STRIPS][MOE_ATTEND_MAX_DIM];
  __shared__ float tops[kJoinWaves], totals[kJoinWaves];
  const Parts parts = parts_of(p);
  const int tid = threadIdx.x, per = p.heads / p.c.kv_heads, per_kv = (per + kCols - 1) / kCols, n_groups = p.c.kv_heads * per_kv;
  const int shares = (parts.rows + each - 1) / each, item = blockIdx.x / shares, seq = item / n_groups, group = item % n_groups;
  const int in0 = group % per_kv * kCols + blockIdx.x % shares * each, in1 = min(min(in0 + each, per), (group % per_kv + 1) * kCols);
  const int64_t share = *parts.share, start = parts.start[seq];
  const Seen s = seen_of(p, p.lengths[seq]);
  uint16_t *y = p.y + ((int64_t)seq * p.heads + group / per_kv * per) * p.c.dim;
  if (s.tiles == 0) {
    for (int d = in0 * p.c.dim + tid; d < in1 * p.c.dim; d += kJoinBlock) y[d] = 0;
    return;
  }
  const int64_t from = start + (int64_t)group * s.tiles;
  const int first = (int)(from / share), n = (int)((from + s.tiles - 1) / share) - first + 1;
  if (n == 1) return;  // (one worker had all of it)
  const auto row_of = [&](int i, int in) { return (uint32_t)((first + i) * 2 + (i == 0 ? 1 : 0)) * parts.rows + in % kCols; };
  if (each > 1 && n <= kFewParts) {
    const int in = in0 + (tid >> 6), lane = tid & 63, half = lane >> 5, d = lane % 32 * 4;
    if (in >= in1) return;
    f32x4 v[kFewParts / 2];
#pragma unroll
    for (int k = 0; k < kFewParts / 2; ++k) {
      const int i = 2 * k + half;
      v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i < n && d < p.c.dim) v[k] = *reinterpret_cast<const f32x4 *>(parts.sums + row_of(i, in) * p.c.dim + d);
    }
    float top = -INFINITY, total = 0.f;
    if (lane < n) {
      top = parts.stats[row_of(lane, in) * 2];
      total = parts.stats[row_of(lane, in) * 2 + 1];
    }
    float most = top;
#pragma unroll
    for (int m = 1; m < kFewParts; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    most = __shfl(most, 0);
    const float weight = __builtin_amdgcn_exp2f(top - (most == -INFINITY ? 0.f : most));
    total *= weight;
#pragma unroll
    for (int m = 1; m < kFewParts; m <<= 1) total += __shfl_xor(total, m);
    total = __shfl(total, 0);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kFewParts / 2; ++k) acc += __shfl(weight, 2 * k + half) * v[k];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      acc[i] += __shfl_xor(acc[i], 32);
      acc[i] = total > 0.f || total != total ? acc[i] / total : 0.f;
    }
    if (half == 0 && d < p.c.dim) *reinterpret_cast<rows_u32x2 *>(y + in * p.c.dim + d) = rows_u32x2{pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3])};
    return;
  }
  for (int in = in0; in < in1; ++in) {
    const int strip = tid / 32, d = tid % 32 * 4;
    // (the first sums come while the weights are worked out)
    f32x4 v[8];
    const auto load = [&](int i0) MOE_ROWS_INLINE {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + strip + k * STRIPS;
        v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (i < n && d < p.c.dim) v[k] = *reinterpret_cast<const f32x4 *>(parts.sums + row_of(i, in) * p.c.dim + d);
      }
    };
    load(0);
    float top = -INFINITY, total = 0.f;
    for (int i = tid; i < n; i += kJoinBlock) top = fmaxf(top, weights[i] = parts.stats[row_of(i, in) * 2]);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kJoinWaves; ++i) top = fmaxf(top, tops[i]);
    const float base = top == -INFINITY ? 0.f : top;
    for (int i = tid; i < n; i += kJoinBlock) {
      weights[i] = __builtin_amdgcn_exp2f(weights[i] - base);
      total += weights[i] * parts.stats[row_of(i, in) * 2 + 1];
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
    if ((tid & 63) == 0) totals[tid >> 6] = total;
    __syncthreads();
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < n; i0 += 8 * STRIPS) {
      if (i0 > 0) load(i0);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + strip + k * STRIPS;
        if (i < n) acc += weights[i] * v[k];
      }
    }
    if (d < p.c.dim) *reinterpret_cast<f32x4 *>(&part[strip][d]) = acc;
    __syncthreads();
    if (tid < p.c.dim) {
      float sum = 0.f;
      total = 0.f;
#pragma unroll
      for (int i = 0; i < STRIPS; ++i) sum += part[i][tid];
#pragma unroll
      for (int i = 0; i < kJoinWaves; ++i) total += totals[i];
      y[in * p.c.dim + tid] = (uint16_t)pack_bf16(total > 0.f || total != total ? sum / total : 0.f, 0.f);
    }
    __syncthreads();
  }
}

template <int CACHE, int DT>
hipError_t attend_with(const AttendPagesParams &p, hipStream_t s) {
  const int per = p.heads / p.c.kv_heads, groups = p.n_seqs * p.c.kv_heads * ((per + kCols - 1) / kCols);
  const int64_t width = (int64_t)p.table_pages << p.c.page_bits;  // no sequence has more
  const int64_t most = p.window > 0 ? std::min<int64_t>(width, (int64_t)p.window + p.sinks + 2 * kTile) : width;
  if (most <= kWholeTiles * kTile && groups <= kGroups) {
    attend_pages_kernel<CACHE, DT, true><<<groups, kWaves * 64, 0, s>>>(p);
    return hipGetLastError();
  }
  attend_pages_kernel<CACHE, DT, false><<<kGroups, kWaves * 64, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = group_rows(p.heads, p.c.kv_heads), each = groups * rows <= kJoinMost ? 1 : kJoinHeads;
  join_pages_kernel<<<groups * ((rows + each - 1) / each), kJoinBlock, 0, s>>>(p, each);
  return hipGetLastError();
}

}  // namespace

size_t attend_pages_bytes(int n_seqs, int heads, int kv_heads, int dim) {
  return parts_head(n_seqs) + (size_t)2 * kWorkers * group_rows(heads, kv_heads) * (dim + 2) * sizeof(float);
}

hipError_t launch_attend_pages(const AttendPagesParams &p, int cache_fmt, hipStream_t s) {
  if (cache_fmt == MOE_R_INT8) return p.c.dim <= 64 ? attend_with<MOE_R_INT8, 64>(p, s) : attend_with<MOE_R_INT8, 128>(p, s);
  return p.c.dim <= 64 ? attend_with<MOE_R_BF16, 64>(p, s) : attend_with<MOE_R_BF16, 128>(p, s);
}

}  // namespace moe
