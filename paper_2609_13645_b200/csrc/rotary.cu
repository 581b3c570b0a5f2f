// Rotary positions as an operator of its own: every pair (a, b) of a head becomes (a c - b s, b c + a s) with the cosine and sine of
// its row's position and its frequency, read from fp32 tables.  Pairs are (i, i + rot / 2) or (2 i, 2 i + 1) of the first `rot`
// elements of a head; the others are passed on.  With -s it is the transpose, which is the backward pass.
//
// Bound by memory: each element is read and written once.  A thread keeps its pairs' table entries in registers and walks over
// heads of its row, two in flight, so that the tables cost one read for four heads; blocks stay, four an SM, and look at the next
// row's position early.  (Four heads in flight take 117 registers: 21.4 us for 4096 rows of 40 heads of 128 bf16 in place, of which
// two take 18.0; a block for every three rows 19.5 with two, 18.0 with four heads in flight behind the tables.)
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
  int lanes;   // threads that share the heads of a unit; units * lanes is at most 256, or lanes is 1
};

// P pairs a unit: two pieces of P elements, or one of 2 P (interleaved, P > 1); what is passed on goes in pieces of W.
template <typename T, int P, bool PAIRS>
__global__ void __launch_bounds__(256, 4)
rotary_kernel(const T* x, T* y, const int* __restrict__ positions, const float* __restrict__ cos, const float* __restrict__ sin,
              float sign, const __grid_constant__ RotaryShape s, int* err) {
  constexpr bool WHOLE = PAIRS && P > 1;
  constexpr int W = WHOLE ? 2 * P : P, U = 2, N = WHOLE ? 1 : 2;  // N: pieces a unit
  pdl_trigger();
  const int per_row = s.units * s.lanes, half = s.rot / 2;
  const int rows_a_block = per_row <= 256 ? 256 / per_row : 1;  // whole rows; a longer one is walked over
  const int mine = per_row <= 256 ? (int)threadIdx.x / per_row : 0;
  if (mine >= rows_a_block) return;
  const int lane = per_row <= 256 ? ((int)threadIdx.x - mine * per_row) / s.units : 0;
  const int u0 = (int)threadIdx.x - mine * per_row - lane * s.units;
  pdl_wait();
  const long long stride = (long long)gridDim.x * rows_a_block;
  auto position = [&](long long row) { return row >= s.rows ? 0 : positions != nullptr ? __ldg(positions + row) : (int)row; };
  int next = position((long long)blockIdx.x * rows_a_block + mine);
  for (long long row = (long long)blockIdx.x * rows_a_block + mine; row < s.rows; row += stride) {
    const int pos = next;
    next = position(row + stride);
    const T* in = x + row * s.ldx;
    T* out = y + row * s.ldy;
    for (int u = u0; u < s.units; u += 256) {
      const bool turn = u < s.turned;
      const int first = !turn ? s.rot + (u - s.turned) * W : PAIRS ? u * 2 * P : u * P, partner = PAIRS ? 1 : half;
      float c[P], n[P];
      for (int h0 = lane; h0 < s.heads; h0 += U * s.lanes) {
        // the elements are on their way before the position is looked at, on which the tables' rows hang
        Piece<T, W> v[U][N];
#pragma unroll
        for (int k = 0; k < U; ++k) {
          if (h0 + k * s.lanes >= s.heads) break;
          const T* from = in + (long long)(h0 + k * s.lanes) * s.d + first;
          v[k][0].load(from);
          if (N == 2 && turn) v[k][N - 1].load(from + partner);
        }
        if (pos < 0 || pos >= s.n_pos) {
          atomicCAS(err, (int)ERR_NONE, (int)ERR_BAD_INDEX);
          break;
        }
        if (turn && h0 == lane) {
          constexpr int F = P < 4 ? P : 4;
          const float *cr = cos + (long long)pos * half + u * P, *sr = sin + (long long)pos * half + u * P;
          Piece<float, F> a[P / F], b[P / F];
#pragma unroll
          for (int e = 0; e < P / F; ++e) {
            a[e].load(cr + e * F);
            b[e].load(sr + e * F);
          }
#pragma unroll
          for (int e = 0; e < P / F; ++e) {
            float fa[F], fb[F];
            a[e].unpack(fa);
            b[e].unpack(fb);
#pragma unroll
            for (int k = 0; k < F; ++k) { c[e * F + k] = fa[k]; n[e * F + k] = sign * fb[k]; }
          }
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
          if (h0 + k * s.lanes >= s.heads) break;
          T* to = out + (long long)(h0 + k * s.lanes) * s.d + first;
          if (!turn) {
            v[k][0].store(to);
          } else if constexpr (WHOLE) {
            float f[W], r[W];
            v[k][0].unpack(f);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              r[2 * e] = f[2 * e] * c[e] - f[2 * e + 1] * n[e];
              r[2 * e + 1] = f[2 * e + 1] * c[e] + f[2 * e] * n[e];
            }
            v[k][0].pack(r);
            v[k][0].store(to);
          } else {
            float a[P], b[P], ra[P], rb[P];
            v[k][0].unpack(a);
            v[k][N - 1].unpack(b);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              ra[e] = a[e] * c[e] - b[e] * n[e];
              rb[e] = b[e] * c[e] + a[e] * n[e];
            }
            v[k][0].pack(ra);
            v[k][N - 1].pack(rb);
            v[k][0].store(to);
            v[k][N - 1].store(to + partner);
          }
        }
      }
    }
  }
}

// Tables of position p and frequency i: angle = p theta^(-2 i / rot) / factor_i, cos and sin times mscale.  A position's step is kept as
// a 64-bit fraction of a turn, of which p times is taken modulo one turn by integer products: far positions lose no more than the step's own
// rounding to 53 bits.  The fp32 functions of pi x take the fraction's first 24 bits, and what is left, under 2^-24 of a turn, turns their
// result by its angle.  A thread keeps its frequency and walks over positions.
__global__ void __launch_bounds__(256)
rotary_tables_kernel(float* __restrict__ cos, float* __restrict__ sin, const float* __restrict__ factors, int n_pos, int half,
                     double log2_step, float mscale) {
  pdl_trigger();
  pdl_wait();
  extern __shared__ unsigned long long steps[];  // formed once a block: 64-bit floating point is what this kernel has least of
  for (int i = threadIdx.x; i < half; i += 256) {
    const double turns = exp2(i * log2_step) * 0.15915494309189533577 / (factors != nullptr ? (double)__ldg(factors + i) : 1.0);
    const double part = turns - floor(turns);
    steps[i] = part < 1.0 ? (unsigned long long)(part * 18446744073709551616.0) : 0ull;
  }
  __syncthreads();
  const int rows = half < 256 ? 256 / half : 1;  // positions a block takes at a time
  const int mine = half < 256 ? (int)threadIdx.x / half : 0;
  if (mine >= rows) return;
  for (int i = (int)threadIdx.x - mine * half; i < half; i += 256) {
    const unsigned long long step = steps[i];
    const float factor = factors != nullptr ? __ldg(factors + i) : 1.f;
    const float scale = factor == factor && factor != 0.f ? mscale : NAN;  // no angle
    const int by = (int)gridDim.x * rows;
#pragma unroll 4
    for (int p = (int)blockIdx.x * rows + mine; p < n_pos; p += by) {
      const unsigned long long turn = step * (unsigned long long)p;
      const int lead = (int)(turn >> 32) >> 8;  // 2^-24 turns, in [-1/2, 1/2) of one
      float s, c;
      sincospif((float)lead * 1.1920928955078125e-7f, &s, &c);
      const float angle = (float)(uint32_t)(turn >> 8) * 8.719671245021579e-17f;  // 2 pi / 2^56
      cos[(long long)p * half + i] = fmaf(-s, angle, c) * scale;
      sin[(long long)p * half + i] = fmaf(c, angle, s) * scale;
      if (p > n_pos - by) break;  // p + by may not fit
    }
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
  if (s.units * s.lanes > 256) s.lanes = s.units < 256 ? 256 / s.units : 1;
  const int per_row = s.units * s.lanes, rows_a_block = per_row <= 256 ? 256 / per_row : 1;
  const long long want = ((long long)s.rows + rows_a_block - 1) / rows_a_block;
  return launch_pdl(rotary_kernel<T, P, PAIRS>, dim3((unsigned)(want < 148 * 4 ? want : 148 * 4)), dim3(256), 0, st,
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

bool overlap(uintptr_t a, size_t na, uintptr_t b, size_t nb) { return a < b + nb && b < a + na; }
// Whether rows of `width` bytes at x and at y share any: with equal strides they may lie beside each other in the same rows.
bool rows_share(uintptr_t x, size_t ldx, uintptr_t y, size_t ldy, size_t rows, size_t width) {
  if (!overlap(x, (rows - 1) * ldx + width, y, (rows - 1) * ldy + width)) return false;
  if (ldx != ldy) return true;
  const size_t apart = (x < y ? y - x : x - y) % ldx;
  return apart < width || apart > ldx - width;
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
  const size_t w = (size_t)width * elem, lx = (rows > 1 ? (size_t)ldx : (size_t)width) * elem, ly = (rows > 1 ? (size_t)ldy : (size_t)width) * elem;
  const uintptr_t x = (uintptr_t)dev_x, y = (uintptr_t)dev_y;
  const size_t span = (size_t)(rows - 1) * ly + w, table = (size_t)n_positions * (rot / 2) * sizeof(float);
  if ((x != y && fs::rows_share(x, lx, y, ly, (size_t)rows, w)) || fs::overlap((uintptr_t)dev_cos, table, y, span) ||
      fs::overlap((uintptr_t)dev_sin, table, y, span) || (dev_positions && fs::overlap((uintptr_t)dev_positions, (size_t)rows * 4, y, span)))
    return FT_EINVAL;
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
  const int at_a_time = rot / 2 < 256 ? 256 / (rot / 2) : 1;
  const size_t blocks = ((size_t)n_positions + 4 * at_a_time - 1) / (4 * at_a_time);  // 4 positions a thread and more
  const cudaError_t e = fs::launch_pdl(fs::rotary_tables_kernel, dim3((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8)), dim3(256),
                                       (size_t)rot / 2 * sizeof(unsigned long long), reinterpret_cast<cudaStream_t>(stream), dev_cos, dev_sin, dev_factors,
                                       n_positions, rot / 2, -2.0 / rot * log2((double)theta), mscale);
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}
