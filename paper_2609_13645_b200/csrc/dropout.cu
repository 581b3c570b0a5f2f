// Dropout of a residual branch with a counter-based mask: y = resid + scale / (1 - p) * keep * x.  The mask is a function
// of (seed, site, step, element index) and is computed where it is used, in the forward and again in the backward pass;
// it is never stored.
//
//   key  = mix(mix(seed ^ (site + 1) C1) ^ step C2)      one per call
//   word = mix(key ^ (index / 4) C3)                     64 bits for four consecutive elements
//   keep = bits [16 (index % 4), +16) of word >= t,      t = round(65536 p)
//
// mix is the splitmix64 finaliser that also keys the weight initialiser.  16 bits an element put the drop rate within
// 2^-17 of p (within 2^-16 above 65535.5 / 65536, where t stops at 65535); the factor of the kept elements is
// 65536 / (65536 - t), the inverse of the rate really used, so the expectation is exact.  A word costs about 25 integer
// instructions for 16-24 bytes of traffic: the kernel stays bound by memory (16384 x 2048 bf16 with a residual: 33.4 us, 6.0 TB/s).
#include <math.h>

#include "../../include/forgestep.h"
#include "dropout.cuh"
#include "rows.cuh"

namespace fs {
namespace {

constexpr unsigned long long kSite = 0xD1B54A32D192ED03ull, kStep = 0xA24BAED4963EE407ull, kGroup = 0x8CB92BA72F3D8DD7ull;

// f[e] <- scale * f[e] where element first + e is kept, else 0.  ALIGNED: first is a multiple of 4.  Elements in front of the
// first one (first < 0) are nobody's.
template <int VEC, bool ALIGNED>
__device__ __forceinline__ void drop(float (&f)[VEC], long long first, unsigned long long key, uint32_t t, float scale) {
  const long long group = first >> 2;
  unsigned long long next = splitmix64(key ^ ((unsigned long long)group * kGroup));
#pragma unroll
  for (int e = 0; e < VEC; e += 4) {
    unsigned long long word = next;
    if (!ALIGNED || e + 4 < VEC) next = splitmix64(key ^ ((unsigned long long)(group + e / 4 + 1) * kGroup));
    if constexpr (!ALIGNED) {
      const int s = 16 * (int)(first & 3);
      if (s != 0) word = word >> s | next << (64 - s);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t bits = (uint32_t)(word >> (16 * k)) & 0xffffu;
      f[e + k] = bits >= t ? f[e + k] * scale : 0.f;
    }
  }
}

// VEC elements from p on, of which those at [from, to) are in the tensor [begin, end) and are read; the others may hold anything.
template <typename T, int VEC>
__device__ __forceinline__ void load_chunk(const T* p, int from, int to, const T* begin, const T* end, float (&f)[VEC]) {
  const int d = behind_boundary(p);
  const T* a = p - d;
  if (a >= begin && a + 2 * VEC <= end) {
    uint4 r = load_piece(a);
    if (d != 0) r = realign(r, load_piece(a + VEC), d, sizeof(T));
    unpack_piece(r, f);
  } else {  // at the tensor's ends
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = e >= from && e < to ? to_float(p[e]) : 0.f;
  }
}

// Rows without gaps between them, whole 16-byte pieces from the start: the chunk index is the element index; the last n % VEC
// elements are handled one by one.  U chunks in flight a thread.
template <typename T, int U>
__global__ void __launch_bounds__(256)
dropout_add_flat_kernel(const T* x, const T* resid, T* y, long long n, unsigned long long base, const long long* __restrict__ step,
                        uint32_t t, float scale) {
  constexpr int VEC = 16 / (int)sizeof(T);
  using V = RowVec<T, VEC>;
  pdl_trigger();
  pdl_wait();
  const unsigned long long key = splitmix64(base ^ ((unsigned long long)(step != nullptr ? *step : 0) * kStep));
  const long long chunks = n / VEC;
  const long long stride = (long long)gridDim.x * blockDim.x;
  for (long long c0 = (long long)blockIdx.x * blockDim.x + threadIdx.x; c0 < chunks; c0 += stride * U) {
    typename V::Raw a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long c = c0 + u * stride;
      a[u] = c < chunks ? V::load(x + c * VEC) : V::zero();
      b[u] = c < chunks && resid != nullptr ? V::load(resid + c * VEC) : V::zero();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long c = c0 + u * stride;
      if (c < chunks) {
        float f[VEC], q[VEC];
        V::unpack(a[u], f);
        V::unpack(b[u], q);
        drop<VEC, true>(f, c * VEC, key, t, scale);
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] += q[e];
        V::store(y + c * VEC, f);
      }
    }
  }
  const long long rest = chunks * VEC;
  if (blockIdx.x == 0 && threadIdx.x == 0 && rest < n) {
    float f[VEC], q[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      f[e] = rest + e < n ? to_float(x[rest + e]) : 0.f;
      q[e] = rest + e < n && resid != nullptr ? to_float(resid[rest + e]) : 0.f;
    }
    drop<VEC, true>(f, rest, key, t, scale);
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (rest + e < n) store_one(y + rest + e, f[e] + q[e]);
  }
}

// Any rows: the chunks of a row are cut at the 16-byte boundaries of its output (the first and the last are partial); a chunk of an
// input that lies otherwise is put together from the two aligned pieces that hold it, the second of which its neighbour
// reads too.
template <typename T>
__global__ void __launch_bounds__(256)
dropout_add_rows_kernel(const T* x, long long ldx, const T* resid, long long ldr, T* y, long long ldy, unsigned rows, unsigned h,
                        unsigned per_row, unsigned long long base, const long long* __restrict__ step, uint32_t t, float scale) {
  constexpr int VEC = 16 / (int)sizeof(T);
  using V = RowVec<T, VEC>;
  pdl_trigger();
  pdl_wait();
  const unsigned long long key = splitmix64(base ^ ((unsigned long long)(step != nullptr ? *step : 0) * kStep));
  const T *x_end = x + (long long)(rows - 1) * ldx + h, *r_end = resid != nullptr ? resid + (long long)(rows - 1) * ldr + h : nullptr;
  const long long chunks = (long long)rows * per_row, stride = (long long)gridDim.x * blockDim.x;
  for (long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x; c < chunks; c += stride) {
    const long long row = c <= 0xffffffffll ? (long long)((unsigned)c / per_row) : c / per_row;
    T* out = y + row * ldy;
    const long long col = (c - row * per_row) * VEC - behind_boundary(out);  // of the chunk's first element
    if (col >= (long long)h) continue;
    const int from = col < 0 ? (int)-col : 0, to = (long long)h - col < VEC ? (int)((long long)h - col) : VEC;
    float f[VEC], q[VEC];
    load_chunk<T, VEC>(x + row * ldx + col, from, to, x, x_end, f);
    if (resid != nullptr) {
      load_chunk<T, VEC>(resid + row * ldr + col, from, to, resid, r_end, q);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) q[e] = 0.f;
    }
    drop<VEC, false>(f, row * h + col, key, t, scale);
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] += q[e];
    if (from == 0 && to == VEC) {
      V::store(out + col, f);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e >= from && e < to) store_one(out + col + e, f[e]);
    }
  }
}

// Elements whose 16 bits are below it are dropped; the factor of the others.
uint32_t threshold(float p) { return (uint32_t)fmin(65535.0, floor((double)p * 65536.0 + 0.5)); }
float kept_factor(float p, float scale) { return (float)((double)scale * 65536.0 / (65536.0 - (double)threshold(p))); }

int blocks_for(long long chunks, int per_thread) {
  const long long want = (chunks + 256 * per_thread - 1) / (256 * per_thread);
  return (int)(want < 1 ? 1 : want < 148 * 16 ? want : 148 * 16);
}

template <typename T>
cudaError_t launch(const void* x, int64_t ldx, const void* resid, int64_t ldr, void* y, int64_t ldy, int rows, int h,
                   unsigned long long base, const long long* step, uint32_t t, float scale, cudaStream_t st) {
  constexpr int VEC = 16 / (int)sizeof(T), U = 2;
  const T *xp = reinterpret_cast<const T*>(x), *rp = reinterpret_cast<const T*>(resid);
  T* yp = reinterpret_cast<T*>(y);
  if (ldx == h && ldy == h && (resid == nullptr || ldr == h) && ((uintptr_t)x | (uintptr_t)resid | (uintptr_t)y) % 16 == 0) {
    const long long n = (long long)rows * h;
    return launch_pdl(dropout_add_flat_kernel<T, U>, dim3(blocks_for(n / VEC, U)), dim3(256), 0, st, xp, rp, yp, n, base, step, t, scale);
  }
  // a row has one chunk more where it may start behind a boundary
  const bool whole = ((uint64_t)ldy * sizeof(T) & 15u) == 0 && ((uintptr_t)y & 15u) == 0;
  const unsigned per_row = (unsigned)(((long long)h + (whole ? 0 : VEC - 1) + VEC - 1) / VEC);
  return launch_pdl(dropout_add_rows_kernel<T>, dim3(blocks_for((long long)rows * per_row, 1)), dim3(256), 0, st, xp, (long long)ldx, rp,
                    (long long)ldr, yp, (long long)ldy, (unsigned)rows, (unsigned)h, per_row, base, step, t, scale);
}

}  // namespace

cudaError_t dropout_add(const void* x, int64_t ldx, const void* resid, int64_t ldr, void* y, int64_t ldy, int rows, int h, float p,
                        float scale, uint64_t seed, int32_t site, const long long* step, int dtype, cudaStream_t st) {
  const uint32_t t = threshold(p);
  const float factor = kept_factor(p, scale);
  const unsigned long long base = splitmix64(seed ^ ((unsigned long long)(long long)(site + 1ll) * kSite));
  if (dtype == 0) return launch<bf16>(x, ldx, resid, ldr, y, ldy, rows, h, base, step, t, factor, st);
  return launch<float>(x, ldx, resid, ldr, y, ldy, rows, h, base, step, t, factor, st);
}

}  // namespace fs

extern "C" ft_status ft_k_dropout_add(const void* dev_x, int64_t ldx, const void* dev_resid, int64_t ldr, void* dev_y, int64_t ldy,
                                      int32_t rows, int32_t h, float p, float scale, uint64_t seed, int32_t site,
                                      const int64_t* dev_step, int32_t dtype, void* stream) {
  if (!dev_x || !dev_y || rows <= 0 || h <= 0 || (dtype != 0 && dtype != 1) || site < 0) return FT_EINVAL;
  if (!(p >= 0.f && p < 1.f) || !isfinite(scale) || !isfinite(fs::kept_factor(p, scale)) || ldx < h || ldy < h || (dev_resid && ldr < h)) return FT_EINVAL;
  if (rows > 1 && ((dev_y == dev_x && ldy != ldx) || (dev_y == dev_resid && ldy != ldr))) return FT_EINVAL;
  const uintptr_t mask = dtype == 0 ? 1u : 3u;
  if (((uintptr_t)dev_x | (uintptr_t)dev_resid | (uintptr_t)dev_y) & mask || (uintptr_t)dev_step & 7u) return FT_EINVAL;
  cudaError_t e = fs::dropout_add(dev_x, ldx, dev_resid, ldr, dev_y, ldy, rows, h, p, scale, seed, site,
                                  reinterpret_cast<const long long*>(dev_step), dtype, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}
