// Vector access shared by the row-wise kernels (LayerNorm, dropout): VEC consecutive elements of a bf16 or fp32 row as
// floats.  VEC is the widest power of two, up to 16 bytes, that divides the row length, every row stride and every
// pointer (row_vec).  Rows that share less are read as the aligned 16-byte pieces that hold them, and moved into place in
// registers (realign), where single elements would take much longer (8192 x 2047 bf16: LayerNorm 41 us forward and 108
// backward with a residual gradient by elements, 30 and 58 by pieces; dropout into rows of 2048 76 and 33).
#pragma once
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "common.cuh"

namespace fs {

template <typename T, int VEC>
struct RowVec;

// 2, 4 or 8 elements (bf16 rows that share less are put together from pieces)
template <int VEC>
struct RowVec<bf16, VEC> {
  typedef typename std::conditional<VEC == 8, uint4, typename std::conditional<VEC == 4, uint2, uint32_t>::type>::type Raw;
  static __device__ __forceinline__ Raw zero() {
    Raw r;
    memset(&r, 0, sizeof(r));
    return r;
  }
  static __device__ __forceinline__ Raw load(const bf16* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&f)[VEC]) {
    uint32_t w[VEC / 2];
    memcpy(w, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
  }
  static __device__ __forceinline__ void store(bf16* p, const float (&f)[VEC]) {
    uint32_t w[VEC / 2];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    Raw r;
    memcpy(&r, w, sizeof(r));
    *reinterpret_cast<Raw*>(p) = r;
  }
};

template <int VEC>
struct RowVec<float, VEC> {
  typedef typename std::conditional<VEC == 4, float4, typename std::conditional<VEC == 2, float2, float>::type>::type Raw;
  static __device__ __forceinline__ Raw zero() {
    Raw r;
    memset(&r, 0, sizeof(r));
    return r;
  }
  static __device__ __forceinline__ Raw load(const float* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&f)[VEC]) { memcpy(f, &r, sizeof(r)); }
  static __device__ __forceinline__ void store(float* p, const float (&f)[VEC]) {
    Raw r;
    memcpy(&r, f, sizeof(r));
    *reinterpret_cast<Raw*>(p) = r;
  }
};

__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ void store_one(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }

// Asynchronous copies from global memory into slots of shared memory: a thread keeps the next rows' elements on their way without
// holding registers for them.  4, 8 or 16 bytes each; valid = false fills the slot with zeros and reads nothing.
template <int BYTES>
__device__ __forceinline__ void async_copy(uint32_t dst, const void* src, bool valid) {
  const int n = valid ? BYTES : 0;
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint4 load_piece(const void* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void unpack_piece(const uint4& r, float (&f)[8]) { RowVec<bf16, 8>::unpack(r, f); }
__device__ __forceinline__ void unpack_piece(const uint4& r, float (&f)[4]) {
  f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
}

// VEC elements that start `d` elements behind the 16-byte boundary at which the pieces a and b lie one after the other.  d is
// the same for a whole row.
__device__ __forceinline__ uint4 realign(const uint4& a, const uint4& b, int d, int elem) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  const int words = d * elem >> 2;
  if (words & 2) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (words & 1) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  if (elem == 2 && (d & 1)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Elements from the last 16-byte boundary at or before p.
template <typename T>
__device__ __forceinline__ int behind_boundary(const T* p) {
  return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
}

// Widest vector width for rows of h elements of `elem` bytes: h and the strides are given or-ed together, as are the
// pointers' addresses (null pointers change nothing).
inline int row_vec(uint64_t h_and_strides, uintptr_t pointers, int elem) {
  int v = 16 / elem;
  while (v > 1 && ((h_and_strides & (uint64_t)(v - 1)) != 0 || (pointers & (uintptr_t)(v * elem - 1)) != 0)) v >>= 1;
  return v;
}

}  // namespace fs
