// Rotary positions as an operator of its own: every pair (a, b) of a head becomes (a c - b s, b c + a s) with the cosine and sine of
// its row's position and its frequency, read from fp32 tables.  Pairs are (i, i + rot / 2) or (2 i, 2 i + 1) of the first `rot`
// elements of a head; the others are passed on.  With -s it is the transpose, which is the backward pass.
//
// Bound by memory: each element is read and written once.  A thread keeps its pairs' table entries in registers and walks over
// heads of its row, up to 4 in flight, so that the tables cost one read a row and not one a head.
#include <math.h>

#include "../../include/forgestep.h"
#include "attention.cuh"
#include "rows.cuh"

namespace fs {
namespace {

// N consecutive elements (N * size at most 16 bytes, aligned to that) as floats, and back.
template <int BYTES> struct Word;
template <> struct Word<2> { typedef uint16_t type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<8> { typedef uint2 type; };
template <> struct Word<16> { typedef uint4 type; };
template <typename T, int N>
struct Piece {
  typename Word<N * (int)sizeof(T)>::type w;
  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const decltype(w)*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<decltype(w)*>(p) = w; }
  __device__ __forceinline__ void unpack(float (&f)[N]) const {
    T e[N];
    memcpy(e, &w, sizeof(w));
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_float(e[i]);
  }
  __device__ __forceinline__ void pack(const float (&f)[N]) {
    T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) store_one(e + i, f[i]);
    memcpy(&w, e, sizeof(w));
  }
};

struct RotaryShape {
  long long ldx, ldy;
  int rows, heads, d, rot, n_pos;
  int units;   // of a head: pieces of pairs, then (unless in place) pieces that are passed on
  int turned;  // the former
  int lanes;   // threads that share the heads of a unit
};

// P pairs a unit: two pieces of P elements, or one of 2 P (interleaved, P > 1); what is passed on goes in pieces of W.
template <typename T, int P, bool PAIRS>
__global__ void __launch_bounds__(256)
rotary_kernel(const T* x, T* y, const int* __restrict__ positions, const float* __restrict__ cos, const float* __restrict__ sin,
              float sign, const __grid_constant__ RotaryShape s, int* err) {
  constexpr bool WHOLE = PAIRS && P > 1;
  constexpr int W = WHOLE ? 2 * P : P, U = 4;
  pdl_trigger();
  pdl_wait();
  const int per_row = s.units * s.lanes, half = s.rot / 2;
  // a block takes whole rows where they are small, else a row is walked over
  const int rows_a_block = per_row < 256 ? 256 / per_row : 1;
  const int mine = per_row < 256 ? (int)threadIdx.x / per_row : 0;
  if (mine >= rows_a_block) return;
  for (long long row = (long long)blockIdx.x * rows_a_block + mine; row < s.rows; row += (long long)gridDim.x * rows_a_block) {
    const int pos = positions != nullptr ? __ldg(positions + row) : (int)row;
    if (pos < 0 || pos >= s.n_pos) {
      atomicCAS(err, (int)ERR_NONE, (int)ERR_BAD_INDEX);
      continue;
    }
    for (int i = (int)threadIdx.x - mine * per_row; i < per_row; i += 256) {
      const int u = i % s.units, lane = i / s.units;
      const T* in = x + row * s.ldx;
      T* out = y + row * s.ldy;
      if (u >= s.turned) {
        const int at = s.rot + (u - s.turned) * W;
        for (int h = lane; h < s.heads; h += s.lanes) {
          Piece<T, W> v;
          v.load(in + (long long)h * s.d + at);
          v.store(out + (long long)h * s.d + at);
        }
        continue;
      }
      float c[P], n[P];
      const float *cr = cos + (long long)pos * half + u * P, *sr = sin + (long long)pos * half + u * P;
#pragma unroll
      for (int e = 0; e < P; e += (P < 4 ? P : 4)) {
        Piece<float, (P < 4 ? P : 4)> a, b;
        a.load(cr + e);
        b.load(sr + e);
        float fa[P < 4 ? P : 4], fb[P < 4 ? P : 4];
        a.unpack(fa);
        b.unpack(fb);
#pragma unroll
        for (int k = 0; k < (P < 4 ? P : 4); ++k) { c[e + k] = fa[k]; n[e + k] = sign * fb[k]; }
      }
      const int first = PAIRS ? u * 2 * P : u * P, partner = PAIRS ? 1 : half;
      for (int h0 = lane; h0 < s.heads; h0 += U * s.lanes) {
        if constexpr (WHOLE) {
          Piece<T, 2 * P> v[U];
#pragma unroll
          for (int k = 0; k < U; ++k)
            if (h0 + k * s.lanes < s.heads) v[k].load(in + (long long)(h0 + k * s.lanes) * s.d + first);
#pragma unroll
          for (int k = 0; k < U; ++k) {
            if (h0 + k * s.lanes >= s.heads) break;
            float f[2 * P], r[2 * P];
            v[k].unpack(f);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              r[2 * e] = f[2 * e] * c[e] - f[2 * e + 1] * n[e];
              r[2 * e + 1] = f[2 * e + 1] * c[e] + f[2 * e] * n[e];
            }
            v[k].pack(r);
            v[k].store(out + (long long)(h0 + k * s.lanes) * s.d + first);
          }
        } else {
          Piece<T, P> va[U], vb[U];
#pragma unroll
          for (int k = 0; k < U; ++k)
            if (h0 + k * s.lanes < s.heads) {
              const T* p = in + (long long)(h0 + k * s.lanes) * s.d + first;
              va[k].load(p);
              vb[k].load(p + partner);
            }
#pragma unroll
          for (int k = 0; k < U; ++k) {
            if (h0 + k * s.lanes >= s.heads) break;
            float a[P], b[P], ra[P], rb[P];
            va[k].unpack(a);
            vb[k].unpack(b);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              ra[e] = a[e] * c[e] - b[e] * n[e];
              rb[e] = b[e] * c[e] + a[e] * n[e];
            }
            va[k].pack(ra);
            vb[k].pack(rb);
            T* p = out + (long long)(h0 + k * s.lanes) * s.d + first;
            va[k].store(p);
            vb[k].store(p + partner);
          }
        }
      }
    }
  }
}

// Tables of position p and frequency i: angle = p theta^(-2 i / rot) / factor_i, cos and sin times mscale.  The angle is formed in
// turns in 64 bits and reduced to half a turn there; what is left goes through the fp32 functions of pi x, so that far
// positions lose nothing.
__global__ void __launch_bounds__(256)
rotary_tables_kernel(float* __restrict__ cos, float* __restrict__ sin, const float* __restrict__ factors, int n_pos, int half,
                     double log2_step, float mscale) {
  pdl_trigger();
  pdl_wait();
  extern __shared__ double turns[];  // a position's step in each frequency
  for (int i = threadIdx.x; i < half; i += 256)
    turns[i] = exp2(i * log2_step) * 0.15915494309189533577 / (factors != nullptr ? (double)__ldg(factors + i) : 1.0);
  __syncthreads();
  const long long n = (long long)n_pos * half, stride = (long long)gridDim.x * 256;
  for (long long k = (long long)blockIdx.x * 256 + threadIdx.x; k < n; k += stride) {
    const int p = n <= 0xffffffffll ? (int)((unsigned)k / (unsigned)half) : (int)(k / half);
    const double t = p * turns[k - (long long)p * half];
    const float x = 2.0f * (float)(t - rint(t));
    float s, c;
    sincospif(x, &s, &c);
    cos[k] = c * mscale;
    sin[k] = s * mscale;
  }
}

template <typename T, int P, bool PAIRS>
cudaError_t launch(const void* x, void* y, const int* positions, const float* cos, const float* sin, float sign, RotaryShape s, int* err,
                   cudaStream_t st) {
  constexpr int W = PAIRS && P > 1 ? 2 * P : P;
  s.turned = s.rot / 2 / P;
  s.units = s.turned + (x == y ? 0 : (s.d - s.rot) / W);
  // a thread takes up to 4 heads; in small calls fewer, so that more of the GPU takes part
  const long long work = (long long)s.rows * s.units * s.heads;
  const int each = work >= 148ll * 2048 * 4 ? 4 : work >= 148ll * 2048 ? 2 : 1;
  s.lanes = (s.heads + each - 1) / each;
  const int per_row = s.units * s.lanes, rows_a_block = per_row < 256 ? 256 / per_row : 1;
  const long long want = ((long long)s.rows + rows_a_block - 1) / rows_a_block;
  return launch_pdl(rotary_kernel<T, P, PAIRS>, dim3((unsigned)(want < 148 * 64 ? want : 148 * 64)), dim3(256), 0, st,
                    reinterpret_cast<const T*>(x), reinterpret_cast<T*>(y), positions, cos, sin, sign, s, err);
}

template <typename T, bool PAIRS>
cudaError_t dispatch(int p, const void* x, void* y, const int* positions, const float* cos, const float* sin, float sign,
                     const RotaryShape& s, int* err, cudaStream_t st) {
  constexpr int MOST = 16 / (int)sizeof(T) / (PAIRS ? 2 : 1);
  if constexpr (MOST >= 8) if (p == 8) return launch<T, 8, PAIRS>(x, y, positions, cos, sin, sign, s, err, st);
  if constexpr (MOST >= 4) if (p == 4) return launch<T, 4, PAIRS>(x, y, positions, cos, sin, sign, s, err, st);
  if (p == 2) return launch<T, 2, PAIRS>(x, y, positions, cos, sin, sign, s, err, st);
  if (p == 1) return launch<T, 1, PAIRS>(x, y, positions, cos, sin, sign, s, err, st);
  return cudaErrorInvalidValue;
}

// Pairs a unit: the widest power of two, up to 16 bytes a piece, with which every piece and every run of the tables is aligned.
int pairs_a_unit(const void* x, const void* y, const void* cos, const void* sin, const RotaryShape& s, int elem, bool interleaved) {
  for (int p = 16 / elem / (interleaved ? 2 : 1); p > 1; p >>= 1) {
    const int w = interleaved ? 2 * p : p;
    const uint64_t sizes = (uint64_t)s.ldx | (uint64_t)s.ldy | (uint64_t)s.d | (uint64_t)s.rot;
    if ((s.rot / 2) % p == 0 && sizes % w == 0 && ((uintptr_t)x | (uintptr_t)y) % (w * elem) == 0 &&
        ((uintptr_t)cos | (uintptr_t)sin) % (p < 4 ? 4 * p : 16) == 0)
      return p;
  }
  return 1;
}

}  // namespace
}  // namespace fs

extern "C" ft_status ft_k_rotary(const void* dev_x, int64_t ldx, void* dev_y, int64_t ldy, const int32_t* dev_positions, const float* dev_cos,
                                 const float* dev_sin, int32_t n_positions, int32_t rows, int32_t n_heads, int32_t head_dim, int32_t rot,
                                 int32_t interleaved, int32_t inverse, int32_t dtype, void* stream) {
  if (!dev_x || !dev_y || !dev_cos || !dev_sin || rows <= 0 || n_heads <= 0 || head_dim <= 0 || head_dim > 16384 || n_positions <= 0) return FT_EINVAL;
  if (rot < 2 || (rot & 1) || rot > head_dim || (dtype != 0 && dtype != 1) || (interleaved & ~1) || (inverse & ~1)) return FT_EINVAL;
  const long long width = (long long)n_heads * head_dim;
  if (width > INT32_MAX / 4 || ldx < width || ldy < width || (!dev_positions && rows > n_positions)) return FT_EINVAL;
  if (rows > 1 && dev_y == dev_x && ldy != ldx) return FT_EINVAL;
  const int elem = dtype == 0 ? 2 : 4;
  if (((uintptr_t)dev_x | (uintptr_t)dev_y) % elem || ((uintptr_t)dev_cos | (uintptr_t)dev_sin | (uintptr_t)dev_positions) & 3u) return FT_EINVAL;
  int* status = fs::attention_status_word();
  if (!status) return FT_ECUDA;
  fs::RotaryShape s{};
  s.ldx = rows > 1 ? ldx : 0; s.ldy = rows > 1 ? ldy : 0;
  s.rows = rows; s.heads = n_heads; s.d = head_dim; s.rot = rot; s.n_pos = n_positions;
  const int p = fs::pairs_a_unit(dev_x, dev_y, dev_cos, dev_sin, s, elem, interleaved != 0);
  const float sign = inverse ? -1.f : 1.f;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (dtype == 0)
    e = interleaved ? fs::dispatch<fs::bf16, true>(p, dev_x, dev_y, dev_positions, dev_cos, dev_sin, sign, s, status, st)
                    : fs::dispatch<fs::bf16, false>(p, dev_x, dev_y, dev_positions, dev_cos, dev_sin, sign, s, status, st);
  else
    e = interleaved ? fs::dispatch<float, true>(p, dev_x, dev_y, dev_positions, dev_cos, dev_sin, sign, s, status, st)
                    : fs::dispatch<float, false>(p, dev_x, dev_y, dev_positions, dev_cos, dev_sin, sign, s, status, st);
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}

extern "C" ft_status ft_k_rotary_tables(float* dev_cos, float* dev_sin, const float* dev_factors, int32_t n_positions, int32_t rot, float theta,
                                        float mscale, void* stream) {
  if (!dev_cos || !dev_sin || n_positions <= 0 || rot < 2 || (rot & 1) || rot > 8192 || !(theta > 0.f) || !isfinite(theta) || !isfinite(mscale))
    return FT_EINVAL;
  if (((uintptr_t)dev_cos | (uintptr_t)dev_sin | (uintptr_t)dev_factors) & 3u) return FT_EINVAL;
  const size_t n = (size_t)n_positions * (rot / 2), bytes = n * sizeof(float);
  const uintptr_t c = (uintptr_t)dev_cos, s = (uintptr_t)dev_sin, f = (uintptr_t)dev_factors, fb = (size_t)rot / 2 * sizeof(float);
  if ((c < s + bytes && s < c + bytes) || (f && ((f < c + bytes && c < f + fb) || (f < s + bytes && s < f + fb)))) return FT_EINVAL;
  const size_t blocks = (n + 1023) / 1024;
  const cudaError_t e = fs::launch_pdl(fs::rotary_tables_kernel, dim3((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8)), dim3(256),
                                       (size_t)rot / 2 * sizeof(double), reinterpret_cast<cudaStream_t>(stream), dev_cos, dev_sin, dev_factors,
                                       n_positions, rot / 2, -2.0 / rot * log2((double)theta), mscale);
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}
