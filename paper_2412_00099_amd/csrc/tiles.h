// What kernels on the matrix cores share: buffer resources, loads that go straight into LDS, transposed reads of it, products.
#pragma once

#include "common.h"

#if defined(__HIPCC__)
namespace moe {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __amdgpu_buffer_rsrc_t Buffer;
#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T *)(p))

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ Buffer buffer_of(const void *base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}
// the same for to_lds, as the instruction takes it
__device__ __forceinline__ i32x4 words_of(const void *base, uint32_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(base);
  return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32 & 0xffff), (int)bytes, 0x00020000};
}
// 16 bytes per lane straight into LDS, lane after lane from `lds` (the same in every lane).  Written out, without results in
// registers: the compiler, which would see that LDS is written, waits for all of them ahead of every transposed read of LDS
// (16384 rows, 60 experts of 2048 x 1408: down 156, gradients of the rows 288, of the weights 600 us that way, 143, 270 and 526 so).  landed_but waits for them instead.
__device__ __forceinline__ void to_lds(i32x4 b, uint32_t off, uint32_t at, uint8_t *lds) {
  const uint32_t to = (uint32_t)reinterpret_cast<uintptr_t>(LDS_PTR(void, lds));
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"  // (five states between a write of a scalar register by the vector unit and its use)
      "buffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(b), "s"(at)
      : "memory");  // (and m0, which is reserved: the compiler sets it ahead of each use of its own, of which there are none here)
}
// the same with 4 bytes per lane
__device__ __forceinline__ void word_to_lds(i32x4 b, uint32_t off, uint8_t *lds) {
  const uint32_t to = (uint32_t)reinterpret_cast<uintptr_t>(LDS_PTR(void, lds));
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(b)
      : "memory");
}
// all but the last N loads of each wavefront of the workgroup have landed, and the reads of LDS that they have issued are done
template <int N>
__device__ __forceinline__ void landed_but() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ i32x4 mma(i32x4 a, i32x4 b, i32x4 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
template <int ROW_BYTES>
__device__ __forceinline__ i32x4 transposed(const uint8_t *at) {  // 8 summed values of the lane's column: rows of `at` and + 4
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + 4 * ROW_BYTES));
  return __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}


// of lanes 0 .. lane: within rows of 16 lanes, then over the rows
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t from_lane(int64_t v) {
  const uint32_t lo = from_lane<CTRL, ROWS>((int)v), hi = from_lane<CTRL, ROWS>((int)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
template <typename T>
__device__ __forceinline__ T sum_upto(T v) {
  v += from_lane<0x111, 0xf>(v);
  v += from_lane<0x112, 0xf>(v);
  v += from_lane<0x114, 0xf>(v);
  v += from_lane<0x118, 0xf>(v);
  v += from_lane<0x142, 0xa>(v);
  v += from_lane<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ int of_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ int64_t of_lane(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)of_lane((int)(v >> 32), lane) << 32 | (uint32_t)of_lane((int)v, lane));
}

}  // namespace moe
#endif
