// Dropout of a residual branch with a counter-based mask: y = resid + scale / (1 - p) * keep * x.  The mask is a function
// of (seed, site, step, element index) and is computed where it is used, in the forward and again in the backward pass;
// it is never stored.
//
//   key  = mix(mix(seed ^ (site + 1) C1) ^ step C2)      one per call
//   word = mix(key ^ (index / 4) C3)                     64 bits for four consecutive elements
//   keep = bits [16 (index % 4), +16) of word >= t,      t = round(65536 p)
//
// mix is the splitmix64 finaliser that also keys the weight initialiser.  16 bits an element put the drop rate within
// 2^-17 of p; the factor of the kept elements is 65536 / (65536 - t), the inverse of the rate really used, so the
// expectation is exact.  A word costs about 25 integer instructions for 16-24 bytes of traffic: the kernel stays bound
// by memory.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "../../include/forgestep.h"
#include "layernorm.cuh"
#include "rows.cuh"

namespace fs {
namespace {

constexpr unsigned long long kSite = 0xD1B54A32D192ED03ull, kStep = 0xA24BAED4963EE407ull, kGroup = 0x8CB92BA72F3D8DD7ull;

// f[e] <- scale * f[e] where element first + e is kept, else 0.  A chunk of 4 or 8 starts on a multiple of 4.
template <int VEC>
__device__ __forceinline__ void drop(float (&f)[VEC], unsigned long long first, unsigned long long key, uint32_t t, float scale) {
  unsigned long long word = 0;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const unsigned long long i = first + e;
    if (VEC < 4 ? (e == 0 || (i & 3) == 0) : (e & 3) == 0) word = splitmix64(key ^ ((i >> 2) * kGroup));
    const uint32_t lane = VEC < 4 ? (uint32_t)(i & 3) : (uint32_t)(e & 3);
    const uint32_t bits = (uint32_t)(word >> (16 * lane)) & 0xffffu;
    f[e] = bits >= t ? f[e] * scale : 0.f;
  }
}

// U chunks of VEC elements in flight a thread.  FLAT: rows follow one another without gaps, so the chunk index is the
// element index; the last `n % VEC` elements are handled one by one.
template <typename T, int VEC, bool FLAT, int U>
__global__ void __launch_bounds__(256)
dropout_add_kernel(const T* x, long long ldx, const T* resid, long long ldr, T* y, long long ldy, long long n, unsigned h,
                   unsigned long long base, const long long* __restrict__ step, uint32_t t, float scale) {
  using V = RowVec<T, VEC>;
  pdl_trigger();
  pdl_wait();
  const unsigned long long key = splitmix64(base ^ ((unsigned long long)(step != nullptr ? *step : 0) * kStep));
  const long long chunks = n / VEC;
  const unsigned per_row = h / VEC;
  const long long stride = (long long)gridDim.x * blockDim.x;
  for (long long c0 = (long long)blockIdx.x * blockDim.x + threadIdx.x; c0 < chunks; c0 += stride * U) {
    typename V::Raw a[U], b[U];
    long long row[U];
    unsigned col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long c = c0 + u * stride;
      if constexpr (FLAT) {
        row[u] = 0;
        col[u] = 0;
        a[u] = c < chunks ? V::load(x + c * VEC) : V::zero();
        b[u] = c < chunks && resid != nullptr ? V::load(resid + c * VEC) : V::zero();
      } else {
        row[u] = c <= 0xffffffffll ? (long long)((unsigned)c / per_row) : c / per_row;
        col[u] = (unsigned)(c - row[u] * per_row) * VEC;
        a[u] = c < chunks ? V::load(x + row[u] * ldx + col[u]) : V::zero();
        b[u] = c < chunks && resid != nullptr ? V::load(resid + row[u] * ldr + col[u]) : V::zero();
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long c = c0 + u * stride;
      if (c < chunks) {
        float f[VEC], q[VEC];
        V::unpack(a[u], f);
        V::unpack(b[u], q);
        drop<VEC>(f, (unsigned long long)c * VEC, key, t, scale);
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] += q[e];
        V::store(FLAT ? y + c * VEC : y + row[u] * ldy + col[u], f);
      }
    }
  }
  if (FLAT && VEC > 1) {
    const long long i = chunks * VEC + threadIdx.x;
    if (blockIdx.x == 0 && i < n) {
      float f[1], q[1] = {0.f};
      RowVec<T, 1>::unpack(RowVec<T, 1>::load(x + i), f);
      if (resid != nullptr) RowVec<T, 1>::unpack(RowVec<T, 1>::load(resid + i), q);
      drop<1>(f, (unsigned long long)i, key, t, scale);
      f[0] += q[0];
      RowVec<T, 1>::store(y + i, f);
    }
  }
}

template <typename T, int VEC, bool FLAT>
cudaError_t launch(const void* x, int64_t ldx, const void* resid, int64_t ldr, void* y, int64_t ldy, int rows, int h,
                   unsigned long long base, const long long* step, uint32_t t, float scale, cudaStream_t st) {
  constexpr int U = 2;
  const long long n = (long long)rows * h, chunks = n / VEC;
  const long long want = (chunks + 256 * U - 1) / (256 * U);
  const int blocks = (int)(want < 1 ? 1 : want < 148 * 16 ? want : 148 * 16);
  return launch_pdl(dropout_add_kernel<T, VEC, FLAT, U>, dim3(blocks), dim3(256), 0, st, reinterpret_cast<const T*>(x), (long long)ldx,
                    reinterpret_cast<const T*>(resid), (long long)ldr, reinterpret_cast<T*>(y), (long long)ldy, n, (unsigned)h, base,
                    step, t, scale);
}

}  // namespace

cudaError_t dropout_add(const void* x, int64_t ldx, const void* resid, int64_t ldr, void* y, int64_t ldy, int rows, int h, float p,
                        float scale, uint64_t seed, int32_t site, const long long* step, int dtype, cudaStream_t st) {
  const uint32_t t = (uint32_t)fmin(65535.0, floor((double)p * 65536.0 + 0.5));
  const float factor = (float)((double)scale * 65536.0 / (65536.0 - (double)t));
  const unsigned long long base = splitmix64(seed ^ ((unsigned long long)(long long)(site + 1ll) * kSite));
  const int elem = dtype == 0 ? 2 : 4;
  const bool flat = ldx == h && ldy == h && (resid == nullptr || ldr == h);
  const uintptr_t ptrs = (uintptr_t)x | (uintptr_t)resid | (uintptr_t)y;
  const int v = flat ? row_vec(0, ptrs, elem) : row_vec((uint64_t)h | (uint64_t)ldx | (uint64_t)ldy | (resid ? (uint64_t)ldr : 0), ptrs, elem);
#define DROP(T, V, F) launch<T, V, F>(x, ldx, resid, ldr, y, ldy, rows, h, base, step, t, factor, st)
#define DROP_T(T, F) (v == 8 ? DROP(T, (sizeof(T) == 2 ? 8 : 4), F) : v == 4 ? DROP(T, 4, F) : v == 2 ? DROP(T, 2, F) : DROP(T, 1, F))
  if (dtype == 0) return flat ? DROP_T(bf16, true) : DROP_T(bf16, false);
  return flat ? DROP_T(float, true) : DROP_T(float, false);
#undef DROP_T
#undef DROP
}

}  // namespace fs

extern "C" ft_status ft_k_dropout_add(const void* dev_x, int64_t ldx, const void* dev_resid, int64_t ldr, void* dev_y, int64_t ldy,
                                      int32_t rows, int32_t h, float p, float scale, uint64_t seed, int32_t site,
                                      const int64_t* dev_step, int32_t dtype, void* stream) {
  if (!dev_x || !dev_y || rows <= 0 || h <= 0 || (dtype != 0 && dtype != 1) || site < 0) return FT_EINVAL;
  if (!(p >= 0.f && p < 1.f) || !isfinite(scale) || ldx < h || ldy < h || (dev_resid && ldr < h)) return FT_EINVAL;
  const uintptr_t mask = dtype == 0 ? 1u : 3u;
  if (((uintptr_t)dev_x | (uintptr_t)dev_resid | (uintptr_t)dev_y) & mask || (uintptr_t)dev_step & 7u) return FT_EINVAL;
  cudaError_t e = fs::dropout_add(dev_x, ldx, dev_resid, ldr, dev_y, ldy, rows, h, p, scale, seed, site,
                                  reinterpret_cast<const long long*>(dev_step), dtype, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}
