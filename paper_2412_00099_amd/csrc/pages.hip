// Pages of a cache of keys and values: which pages and places new tokens get, and the copy of their rows into them.
//
// Plan: sums over the sequences (new tokens, pages to take) in the order of the sequences.  One launch: every workgroup goes over all
// sequences, kChunk at a time, and sums them up for itself (a few KB from the caches), then finds the sequence of each of its tokens
// and taken pages by bisection of the chunk's sums in LDS.  A token of a page that is taken in this launch finds the page in the
// list of free ones, not in the table, so that no workgroup waits for another.  Bound by latency: the sequences' numbers, two barriers,
// the entries.  Eight requests 4.3 us, 1024 with 320000 new tokens 7.6.
// Store: bound by memory; a lane has 8 values of a head, the 8-bit form takes the largest over a head's lanes.  8 tokens of 16 heads of
// 128 2.8 us; 8191 of 8 heads into 8 bits, 51 MB, 14 us (3.6 TB/s).
#include <algorithm>

#include "attend.h"
#include "rows.h"
#include "tiles.h"

namespace moe {
namespace {

constexpr int kPlanBlock = 256, kChunk = 1024, kEach = kChunk / kPlanBlock;  // a thread has kEach sequences in a row

__device__ __forceinline__ int to32(int64_t v) { return (int)min(v, (int64_t)INT32_MAX); }

__global__ __launch_bounds__(kPlanBlock) void plan_pages_kernel(const PlanPagesParams p) {
  // behind sequence i of the chunk: new tokens and taken pages so far, of all sequences (element 0: ahead of the chunk)
  __shared__ int64_t tokens[kChunk + 1], taken[kChunk + 1];
  __shared__ int64_t wave_tokens[kPlanBlock / 64], wave_taken[kPlanBlock / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t step = (int64_t)gridDim.x * kPlanBlock, mine = (int64_t)blockIdx.x * kPlanBlock + tid;
  const int64_t used = p.used ? *p.used : 0;
  int64_t all_tokens = 0, all_taken = 0;
  const auto pages_of = [&](int64_t n) { return min((n + (1 << p.page_bits) - 1) >> p.page_bits, (int64_t)p.table_pages); };
  const auto free_page = [&](int64_t i) { return i >= 0 && i < p.n_free ? p.free[i] : -1; };
  for (int s0 = 0; s0 < p.n_seqs; s0 += kChunk) {
    int64_t have[kEach], more[kEach], take[kEach], upto_tokens = 0, upto_taken = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int s = s0 + tid * kEach + i;
      have[i] = s < p.n_seqs ? max(p.have[s], 0) : 0;
      more[i] = s < p.n_seqs ? max(p.more[s], 0) : 0;
      take[i] = pages_of(have[i] + more[i]) - pages_of(have[i]);
      upto_tokens += more[i];
      upto_taken += take[i];
    }
    const int64_t t = sum_upto(upto_tokens), k = sum_upto(upto_taken);
    if (lane == 63) {
      wave_tokens[wave] = t;
      wave_taken[wave] = k;
    }
    __syncthreads();
    int64_t before_tokens = all_tokens + t - upto_tokens, before_taken = all_taken + k - upto_taken;
    for (int w = 0; w < kPlanBlock / 64; ++w) {
      before_tokens += w < wave ? wave_tokens[w] : 0;
      before_taken += w < wave ? wave_taken[w] : 0;
      all_tokens += wave_tokens[w];
      all_taken += wave_taken[w];
    }
    if (tid == 0) {
      tokens[0] = before_tokens;
      taken[0] = before_taken;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int c = tid * kEach + i, s = s0 + c;
      if (s < p.n_seqs && blockIdx.x == 0) {
        p.offsets[s] = to32(before_tokens);
        p.lengths[s] = to32(have[i] + more[i]);
      }
      tokens[c + 1] = before_tokens += more[i];
      taken[c + 1] = before_taken += take[i];
    }
    __syncthreads();
    // the sequence of the chunk that has element v of a sum
    const auto of = [&](const int64_t *sums, int64_t v) {
      int at = 0;
#pragma unroll
      for (int o = kChunk / 2; o > 0; o >>= 1) at += sums[at + o] <= v ? o : 0;
      return at;
    };
    // this workgroup's elements of a sum, up to `end`: the first one of its own from the chunk's first on
    const auto first = [&](int64_t from) { return from <= mine ? mine : mine + (from - mine + step - 1) / step * step; };
    for (int64_t v = first(taken[0]); v < taken[kChunk]; v += step) {
      const int c = of(taken, v), s = s0 + c;
      p.table[(int64_t)s * p.table_pages + pages_of(max(p.have[s], 0)) + (v - taken[c])] = free_page(used + v);
    }
    const int64_t end = min(tokens[kChunk], (int64_t)p.n_tokens);
    for (int64_t v = first(tokens[0]); v < end; v += step) {
      const int c = of(tokens, v), s = s0 + c;
      const int64_t had = max(p.have[s], 0), pos = had + (v - tokens[c]), old = pages_of(had), at = pos >> p.page_bits;
      int64_t slot = -1;
      if (at < p.table_pages) {
        const int64_t page = at < old ? p.table[(int64_t)s * p.table_pages + at] : free_page(used + taken[c] + (at - old));
        slot = page < 0 ? -1 : page << p.page_bits | (pos & ((1 << p.page_bits) - 1));
      }
      p.slots[v] = slot > INT32_MAX ? -1 : (int)slot;
      p.positions[v] = to32(pos);
    }
    __syncthreads();
  }
  for (int64_t v = all_tokens <= mine ? mine : mine + (all_tokens - mine + step - 1) / step * step; v < p.n_tokens; v += step) {
    p.slots[v] = -1;
    p.positions[v] = -1;
  }
  if (mine == 0) {
    p.offsets[p.n_seqs] = to32(all_tokens);
    *p.used_out = to32(used + all_taken);
  }
}

struct StoreArgs {
  CacheParams c;
  HeadRows k, v;
  const int32_t *slots;
  int64_t items;  // heads of all rows
};

__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
  return v;
}

// round(127 v / top) as if computed exactly.  16-bit values are often half way between two codes, or so close that 32 bits do not tell:
// there the quotient is taken in 64 (127 v and the halves are exact in them).
__device__ __forceinline__ int code_of(float v, float top, float inv) {
  const float q = v * inv;  // (three roundings: off by less than 127 * 3 * 2^-24 = 2.3e-5)
  float r = rintf(q);
  if (fabsf(fabsf(q - r) - 0.5f) < 5e-5f) r = (float)rint(127.0 * (double)v / (double)top);
  return (int)r;
}

// LANES: lanes of a head, 8 values each
template <int FMT, int CACHE, int LANES>
__global__ __launch_bounds__(256) void store_pages_kernel(const StoreArgs a) {
  const int64_t item = ((int64_t)row_group() * 256 + threadIdx.x) / LANES;
  const int l = threadIdx.x % LANES, d = l * 8;
  if (item >= a.items) return;  // (all lanes of a head)
  const int row = (int)(item / a.c.kv_heads), head = (int)(item % a.c.kv_heads);
  const int slot = a.slots[row], page = slot >> a.c.page_bits, place = slot & ((1 << a.c.page_bits) - 1);
  if (slot < 0 || page >= a.c.n_pages) return;
  const bool there = d < a.c.dim;
  float v[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[0][i] = v[1][i] = 0.f;
  if (there) {
    load_row<FMT, 8>(a.k.at, row * a.k.token + head * a.k.head + d, v[0]);
    load_row<FMT, 8>(a.v.at, row * a.v.token + head * a.v.head + d, v[1]);
  }
  const int64_t at = page * a.c.page_stride + (((int64_t)head << a.c.page_bits) + place) * a.c.dim + d;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    void *to = w == 0 ? a.c.k : a.c.v;
    if constexpr (CACHE != MOE_R_INT8) {
      if (there) store_row<CACHE, 8>(to, at, v[w]);
    } else {
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) bits = max(bits, __float_as_uint(v[w][i]) & 0x7fffffffu);
      bits = lanes_max(bits, LANES);
      const float top = __uint_as_float(bits);
      const bool finite = bits < 0x7f800000u, none = !finite || top < 1e-30f;
      const float inv = none ? 0.f : 127.f * (1.f / top);
      rows_u32x2 codes = {0, 0};
      if (!none) {
#pragma unroll
        for (int i = 0; i < 8; ++i) codes[i / 4] |= (uint32_t)(code_of(v[w][i], top, inv) & 0xff) << (i % 4 * 8);
      }
      if (there) *reinterpret_cast<rows_u32x2_codes *>(static_cast<uint8_t *>(to) + at) = codes;
      if (l == 0)
        (w == 0 ? a.c.k_scale : a.c.v_scale)[(((int64_t)page * a.c.kv_heads + head) << a.c.page_bits) + place] =
            !finite ? __uint_as_float(0x7fc00000u) : none ? 0.f : top / 127.f;
    }
  }
}

template <int FMT, int CACHE>
void store_with(const StoreArgs &a, int lanes, hipStream_t s) {
  const RowGrid g = row_grid((a.items * lanes + 255) / 256);
  const dim3 grid(g.x, g.y);
  switch (lanes) {
    case 1: store_pages_kernel<FMT, CACHE, 1><<<grid, 256, 0, s>>>(a); break;
    case 2: store_pages_kernel<FMT, CACHE, 2><<<grid, 256, 0, s>>>(a); break;
    case 4: store_pages_kernel<FMT, CACHE, 4><<<grid, 256, 0, s>>>(a); break;
    case 8: store_pages_kernel<FMT, CACHE, 8><<<grid, 256, 0, s>>>(a); break;
    default: store_pages_kernel<FMT, CACHE, 16><<<grid, 256, 0, s>>>(a); break;
  }
}

}  // namespace

hipError_t launch_plan_pages(const PlanPagesParams &p, hipStream_t s) {
  const int64_t groups = ((int64_t)p.n_tokens + kPlanBlock - 1) / kPlanBlock;
  plan_pages_kernel<<<(int)std::clamp<int64_t>(groups, 1, 512), kPlanBlock, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_store_pages(const CacheParams &c, int cache_fmt, const HeadRows &k, const HeadRows &v, int fmt, const int32_t *slots,
                              int n_rows, hipStream_t s) {
  const StoreArgs a{c, k, v, slots, (int64_t)n_rows * c.kv_heads};
  int lanes = 1;
  while (lanes * 8 < c.dim) lanes *= 2;
  if (fmt == MOE_R_FP32) {
    if (cache_fmt == MOE_R_INT8) store_with<MOE_R_FP32, MOE_R_INT8>(a, lanes, s);
    else store_with<MOE_R_FP32, MOE_R_BF16>(a, lanes, s);
  } else {
    if (cache_fmt == MOE_R_INT8) store_with<MOE_R_BF16, MOE_R_INT8>(a, lanes, s);
    else store_with<MOE_R_BF16, MOE_R_BF16>(a, lanes, s);
  }
  return hipGetLastError();
}

}  // namespace moe
