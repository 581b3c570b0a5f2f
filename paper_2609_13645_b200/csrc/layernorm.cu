// LayerNorm, forward and backward, over rows of any width and stride.  Reductions run in a fixed order (no floating-point
// atomics), statistics and sums are fp32, each output is rounded once.
//
// A row belongs to a group of GW warps; a lane holds NCH chunks of VEC elements of it, chunk k of lane l of the group
// being elements (k GW 32 + l) VEC, so every load of a warp is one contiguous run.  The whole row stays in registers
// between the load and the store: the mean and then the centred sum of squares are taken from there (the difference of
// sum(x^2) and mean^2 would lose the variance of rows whose mean is large), and nothing is read twice.
#include "layernorm.cuh"

#include "../../include/forgestep.h"
#include "rows.cuh"

namespace fs {
namespace {

constexpr int kSms = 148;

// barrier of one group of warps (bar 0 is __syncthreads)
__device__ __forceinline__ void group_sync(int group, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
}

// ---------------------------------------------------------------- forward
// y = (x - mean) rstd gain + bias.
template <typename T, int VEC, int NCH>
__global__ void __launch_bounds__(512)
layernorm_fwd_kernel(const T* __restrict__ x, long long ldx, const T* __restrict__ gain, const T* __restrict__ bias, T* __restrict__ y,
                     long long ldy, float* __restrict__ mean, float* __restrict__ rstd, int rows, int h, int gw, float eps) {
  using V = RowVec<T, VEC>;
  pdl_trigger();
  pdl_wait();
  __shared__ float s_part[2][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / gw, gwarp = warp - group * gw, groups = (blockDim.x >> 5) / gw;
  const int first = (gwarp * 32 + lane) * VEC, stride = gw * 32 * VEC;
  const float inv_h = 1.0f / (float)h;
  // sum over the group's lanes; every thread gets the same bits.  The two sums of a row use different slots, and the
  // second barrier of a row lies between the reads of the first sum and its next overwrite.
  auto group_sum = [&](float v, int which) {
    v = warp_sum(v);
    if (gw == 1) return v;
    if (lane == 0) s_part[which][warp] = v;
    group_sync(group, gw * 32);
    float t = 0.f;
    for (int w = 0; w < gw; ++w) t += s_part[which][group * gw + w];
    return t;
  };
  for (long long row = (long long)blockIdx.x * groups + group; row < rows; row += (long long)gridDim.x * groups) {
    const T* xr = x + row * ldx;
    typename V::Raw raw[NCH];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = first + k * stride;
      raw[k] = c < h ? V::load(xr + c) : V::zero();
    }
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      float f[VEC];
      V::unpack(raw[k], f);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += f[e];
    }
    const float mu = group_sum(s, 0) * inv_h;
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      float f[VEC];
      V::unpack(raw[k], f);
      if (first + k * stride < h) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss += (f[e] - mu) * (f[e] - mu);
      }
    }
    const float rs = 1.0f / sqrtf(group_sum(ss, 1) * inv_h + eps);
    if (gwarp == 0 && lane == 0) {
      mean[row] = mu;
      rstd[row] = rs;
    }
    T* yr = y + row * ldy;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = first + k * stride;
      if (c < h) {
        float f[VEC], g[VEC], b[VEC];
        V::unpack(raw[k], f);
        V::unpack(V::load(gain + c), g);
        if (bias != nullptr) V::unpack(V::load(bias + c), b);
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = (f[e] - mu) * rs * g[e] + (bias != nullptr ? b[e] : 0.f);
        V::store(yr + c, f);
      }
    }
  }
}

template <typename T, int VEC, int EPL>
cudaError_t fwd_launch(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean, float* rstd,
                       int rows, int h, int gw, float eps, cudaStream_t st) {
  constexpr int NCH = EPL / VEC > 0 ? EPL / VEC : 1;
  const int groups = gw >= 8 ? 1 : 8 / gw;
  const long long want = (rows + groups - 1) / groups;
  const int blocks = (int)(want < kSms * 16 ? want : kSms * 16);
  return launch_pdl(layernorm_fwd_kernel<T, VEC, NCH>, dim3(blocks), dim3(groups * gw * 32), 0, st, reinterpret_cast<const T*>(x),
                    (long long)ldx, reinterpret_cast<const T*>(gain), reinterpret_cast<const T*>(bias), reinterpret_cast<T*>(y),
                    (long long)ldy, mean, rstd, rows, h, gw, eps);
}

template <typename T, int VEC>
cudaError_t fwd_width(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean, float* rstd,
                      int rows, int h, float eps, cudaStream_t st) {
  // one warp a row up to 1024 elements (2048 in bf16, whose lane then holds 64 elements in 32 registers), then a warp
  // for every 1024 elements of the row
  if (h <= 256) return fwd_launch<T, VEC, 8>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, 1, eps, st);
  if constexpr (sizeof(T) == 2 && VEC == 8)
    if (h > 1024 && h <= 2048) return fwd_launch<T, VEC, 64>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, 1, eps, st);
  return fwd_launch<T, VEC, 32>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, (h + 1023) / 1024, eps, st);
}

// ---------------------------------------------------------------- backward
// dx = rstd (g - mean_h(g) - xhat mean_h(g xhat)) + resid with g = dy gain; dgain = sum over rows of dy xhat, dbias of dy.
// A thread owns the same columns of every row it meets, so its share of dgain and dbias stays in registers for the whole
// launch; a block leaves one partial row of each, which a second kernel adds in block order.  R rows are in flight at a
// time: their two sums are reduced over the group together (one barrier for R rows).  HOLD: the rows stay in registers
// between the sums and the update; the widest rows are read a second time (from L1 or L2) instead of spilling.
constexpr int kBwdMaxBlocks = kSms * 2;

// Sums of N values over a warp, N a power of two up to 32: each step halves the values a lane still carries, so it takes
// N - 1 + log2(32 / N) shuffles instead of 5 N.  Lane l ends with the total of value index l / (32 / N).
template <int N>
__device__ __forceinline__ float warp_sum_many(float (&v)[N], int lane) {
  int half = 16;
#pragma unroll
  for (int n = N; n > 1; n >>= 1) {
    const bool up = (lane & half) != 0;
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
      const float send = up ? v[i] : v[i + n / 2];
      const float keep = up ? v[i + n / 2] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, half);
    }
    half >>= 1;
  }
  float t = v[0];
  for (; half > 0; half >>= 1) t += __shfl_xor_sync(0xffffffffu, t, half);
  return t;
}

template <typename T, int VEC, int NCH, int R, bool HOLD>
__global__ void __launch_bounds__(VEC * NCH == 8 ? 256 : 512, VEC * NCH == 8 ? 2 : 1)
layernorm_bwd_kernel(const T* __restrict__ dy, long long lddy, const T* __restrict__ x, long long ldx, const float* __restrict__ mean,
                     const float* __restrict__ rstd, const T* __restrict__ gain, const T* resid, long long ldr, T* dx, long long lddx,
                     float* __restrict__ partial, int rows, int h, int gw) {
  using V = RowVec<T, VEC>;
  pdl_trigger();
  pdl_wait();
  extern __shared__ float smem[];  // [2][warps][2 R] row sums, then (several groups) [2 h] column sums
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int group = warp / gw, gwarp = warp - group * gw, groups = warps / gw;
  const int first = (gwarp * 32 + lane) * VEC, stride = gw * 32 * VEC;
  const float inv_h = 1.0f / (float)h;
  float acc_g[NCH][VEC], acc_b[NCH][VEC];
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc_g[k][e] = acc_b[k][e] = 0.f;
  }
  int parity = 0;
  for (long long row0 = ((long long)blockIdx.x * groups + group) * R; row0 < rows; row0 += (long long)gridDim.x * groups * R) {
    typename V::Raw rdy[R][NCH], rx[R][NCH], rr[R][NCH];
    float mu[R], rs[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool live = row0 + r < rows;
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        const int c = first + k * stride;
        const bool ok = live && c < h;
        rdy[r][k] = ok ? V::load(dy + (row0 + r) * lddy + c) : V::zero();
        rx[r][k] = ok ? V::load(x + (row0 + r) * ldx + c) : V::zero();
        if (HOLD) rr[r][k] = ok && resid != nullptr ? V::load(resid + (row0 + r) * ldr + c) : V::zero();
      }
      mu[r] = live ? mean[row0 + r] : 0.f;
      rs[r] = live ? rstd[row0 + r] : 0.f;
    }
    float sums[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        const int c = first + k * stride;
        float a[VEC], b[VEC], gn[VEC];
        V::unpack(rdy[r][k], a);
        V::unpack(rx[r][k], b);
        V::unpack(c < h ? V::load(gain + c) : V::zero(), gn);  // gains stay in L1
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float xh = (b[e] - mu[r]) * rs[r], g = a[e] * gn[e];  // a = 0 outside the row
          s1 += g;
          s2 += g * xh;
          acc_g[k][e] += a[e] * xh;
          acc_b[k][e] += a[e];
        }
      }
      sums[2 * r] = s1;
      sums[2 * r + 1] = s2;
    }
    const float tot = warp_sum_many<2 * R>(sums, lane);
    float m1[R], m2[R];
    float* slot = smem + parity * warps * 2 * R;
    if ((lane & (32 / (2 * R) - 1)) == 0) slot[warp * 2 * R + lane / (32 / (2 * R))] = tot;
    if (gw == 1) __syncwarp(); else group_sync(group, gw * 32);
#pragma unroll
    for (int r = 0; r < R; ++r) m1[r] = m2[r] = 0.f;
    for (int w = 0; w < gw; ++w) {
      const float* p = slot + (group * gw + w) * 2 * R;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        m1[r] += p[2 * r];
        m2[r] += p[2 * r + 1];
      }
    }
    parity ^= 1;  // the other slot is free: everyone passed this barrier after its last reads
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row0 + r < rows) {
        const float a1 = m1[r] * inv_h, a2 = m2[r] * inv_h;
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
          const int c = first + k * stride;
          if (c < h) {
            if (HOLD) {
              forget(rdy[r][k]);
              forget(rx[r][k]);
            } else {
              rdy[r][k] = V::load(dy + (row0 + r) * lddy + c);
              rx[r][k] = V::load(x + (row0 + r) * ldx + c);
              rr[r][k] = resid != nullptr ? V::load(resid + (row0 + r) * ldr + c) : V::zero();
            }
            float a[VEC], b[VEC], q[VEC], o[VEC], gn[VEC];
            V::unpack(rdy[r][k], a);
            V::unpack(rx[r][k], b);
            V::unpack(rr[r][k], q);
            V::unpack(V::load(gain + c), gn);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const float xh = (b[e] - mu[r]) * rs[r];
              o[e] = rs[r] * (a[e] * gn[e] - a1 - xh * a2) + q[e];
            }
            V::store(dx + (row0 + r) * lddx + c, o);
          }
        }
      }
    }
  }
  // one partial row a block: its groups are added in group order
  float* out_g = partial + (long long)blockIdx.x * 2 * h;
  float* out_b = out_g + h;
  float* col = smem + 2 * warps * 2 * R;
  for (int g = 0; g < groups; ++g) {
    if (group == g) {
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int c = first + k * stride + e;
          if (c < h) {
            float tg = acc_g[k][e], tb = acc_b[k][e];
            if (g > 0) { tg += col[c]; tb += col[h + c]; }
            if (g + 1 < groups) { col[c] = tg; col[h + c] = tb; }
            else { out_g[c] = tg; out_b[c] = tb; }
          }
        }
      }
    }
    if (groups > 1) __syncthreads();
  }
}

// Column sums of the block partials in block order: 32 columns x 8 strided row groups a CTA, the groups added in order.
__global__ void __launch_bounds__(256)
layernorm_colsum_kernel(const float* __restrict__ partial, float* __restrict__ dgain, float* __restrict__ dbias, int nblk, int h) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s[8][33];
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
  const int cols = dbias != nullptr ? 2 * h : h;
  const int c = blockIdx.x * 32 + cx;
  float a = 0.f;
  if (c < cols)
    for (int b = ry; b < nblk; b += 8) a += partial[(long long)b * 2 * h + c];
  s[ry][cx] = a;
  __syncthreads();
  if (ry == 0 && c < cols) {
    float tot = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) tot += s[w][cx];
    if (c < h) dgain[c] = tot; else dbias[c - h] = tot;
  }
}

struct BwdShape {
  int epl, gw, groups, blocks;
};

// 8 columns a thread up to 2048 columns; wider rows take 16 and 32 columns a thread, so that a block never exceeds 16
// warps and a thread 128 registers.  At least 8 warps a block.  One block for every 32 / epl rows of its groups, at most two
// an SM: the scratch size follows from rows and h alone.
BwdShape bwd_shape(int rows, int h) {
  BwdShape s;
  s.epl = h <= 2048 ? 8 : h <= 8192 ? 16 : 32;
  const int r = 32 / s.epl;
  s.gw = (h + 32 * s.epl - 1) / (32 * s.epl);
  s.groups = s.gw >= 8 ? 1 : 8 / s.gw;
  const long long want = ((long long)rows + s.groups * r - 1) / (s.groups * r);
  s.blocks = (int)(want < kBwdMaxBlocks ? want : kBwdMaxBlocks);
  return s;
}

template <typename T, int VEC, int EPL, int R, bool HOLD>
cudaError_t bwd_launch(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd, const void* gain,
                       const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias, float* scratch, int rows,
                       int h, const BwdShape& s, cudaStream_t st) {
  const int warps = s.gw * s.groups;
  const size_t smem = (size_t)(2 * warps * 2 * R + (s.groups > 1 ? 2 * h : 0)) * sizeof(float);
  cudaError_t e = launch_pdl(layernorm_bwd_kernel<T, VEC, EPL / VEC, R, HOLD>, dim3(s.blocks), dim3(warps * 32), smem, st,
                             reinterpret_cast<const T*>(dy), (long long)lddy, reinterpret_cast<const T*>(x), (long long)ldx, mean, rstd,
                             reinterpret_cast<const T*>(gain), reinterpret_cast<const T*>(resid), (long long)ldr,
                             reinterpret_cast<T*>(dx), (long long)lddx, scratch, rows, h, s.gw);
  if (e != cudaSuccess) return e;
  const int cols = dbias != nullptr ? 2 * h : h;
  return launch_pdl(layernorm_colsum_kernel, dim3((cols + 31) / 32), dim3(256), 0, st, scratch, dgain, dbias, s.blocks, h);
}

template <typename T, int VEC>
cudaError_t bwd_width(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd, const void* gain,
                      const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias, float* scratch, int rows,
                      int h, cudaStream_t st) {
  const BwdShape s = bwd_shape(rows, h);
  // rows in flight at 8 columns a thread, by the registers a row takes (a packed 16-byte chunk: 4, single elements: 8)
  constexpr int R8 = sizeof(T) == 2 && VEC >= 4 ? 4 : 2;
#define LN_BWD_W(EPL, R, HOLD) bwd_launch<T, VEC, EPL, R, HOLD>(dy, lddy, x, ldx, mean, rstd, gain, resid, ldr, dx, lddx, dgain, dbias, scratch, rows, h, s, st)
  return s.epl == 8 ? LN_BWD_W(8, R8, true) : s.epl == 16 ? LN_BWD_W(16, R8 / 2, true) : LN_BWD_W(32, 1, false);
#undef LN_BWD_W
}

}  // namespace

cudaError_t layernorm_fwd(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean,
                          float* rstd, int rows, int h, float eps, int dtype, cudaStream_t st) {
  const int elem = dtype == 0 ? 2 : 4;
  const uintptr_t ptrs = (uintptr_t)x | (uintptr_t)gain | (uintptr_t)bias | (uintptr_t)y;
  const int v = row_vec((uint64_t)h | (uint64_t)ldx | (uint64_t)ldy, ptrs, elem);
  if (dtype == 0) {
    if (v == 8) return fwd_width<bf16, 8>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st);
    if (v == 4) return fwd_width<bf16, 4>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st);
    if (v == 2) return fwd_width<bf16, 2>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st);
    return fwd_width<bf16, 1>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st);
  }
  if (v == 4) return fwd_width<float, 4>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st);
  if (v == 2) return fwd_width<float, 2>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st);
  return fwd_width<float, 1>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st);
}

size_t layernorm_scratch_bytes(int rows, int h) {
  if (rows <= 0 || h <= 0 || h > kLayerNormMaxWidth) return 0;
  return (size_t)bwd_shape(rows, h).blocks * 2 * (size_t)h * sizeof(float);
}

cudaError_t layernorm_bwd(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd,
                          const void* gain, const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias,
                          float* scratch, int rows, int h, int dtype, cudaStream_t st) {
  const int elem = dtype == 0 ? 2 : 4;
  const uintptr_t ptrs = (uintptr_t)dy | (uintptr_t)x | (uintptr_t)gain | (uintptr_t)resid | (uintptr_t)dx;
  const int v = row_vec((uint64_t)h | (uint64_t)lddy | (uint64_t)ldx | (resid ? (uint64_t)ldr : 0) | (uint64_t)lddx, ptrs, elem);
#define LN_BWD(T, V) bwd_width<T, V>(dy, lddy, x, ldx, mean, rstd, gain, resid, ldr, dx, lddx, dgain, dbias, scratch, rows, h, st)
  if (dtype == 0) return v == 8 ? LN_BWD(bf16, 8) : v == 4 ? LN_BWD(bf16, 4) : v == 2 ? LN_BWD(bf16, 2) : LN_BWD(bf16, 1);
  return v == 4 ? LN_BWD(float, 4) : v == 2 ? LN_BWD(float, 2) : LN_BWD(float, 1);
#undef LN_BWD
}

}  // namespace fs

// =============================================================================== entry points
namespace {
bool rows_ok(int32_t rows, int32_t h, int32_t dtype) {
  return rows > 0 && h > 0 && h <= fs::kLayerNormMaxWidth && (dtype == 0 || dtype == 1);
}
bool elem_aligned(const void* p, int32_t dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == 0 ? 1u : 3u)) == 0; }
}  // namespace

extern "C" ft_status ft_k_layernorm_fwd(const void* dev_x, int64_t ldx, const void* dev_gain, const void* dev_bias, void* dev_y,
                                        int64_t ldy, float* dev_mean, float* dev_rstd, int32_t rows, int32_t h, float eps,
                                        int32_t dtype, void* stream) {
  if (!dev_x || !dev_gain || !dev_y || !dev_mean || !dev_rstd || !rows_ok(rows, h, dtype)) return FT_EINVAL;
  if (ldx < h || ldy < h || !(eps >= 0.f)) return FT_EINVAL;
  if (!elem_aligned(dev_x, dtype) || !elem_aligned(dev_gain, dtype) || !elem_aligned(dev_bias, dtype) || !elem_aligned(dev_y, dtype))
    return FT_EINVAL;
  cudaError_t e = fs::layernorm_fwd(dev_x, ldx, dev_gain, dev_bias, dev_y, ldy, dev_mean, dev_rstd, rows, h, eps, dtype,
                                    reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}

extern "C" size_t ft_k_layernorm_scratch_bytes(int32_t rows, int32_t h) { return fs::layernorm_scratch_bytes(rows, h); }

extern "C" ft_status ft_k_layernorm_bwd(const void* dev_dy, int64_t lddy, const void* dev_x, int64_t ldx, const float* dev_mean,
                                        const float* dev_rstd, const void* dev_gain, const void* dev_resid, int64_t ldr,
                                        void* dev_dx, int64_t lddx, float* dev_dgain, float* dev_dbias, void* dev_scratch,
                                        uint64_t scratch_bytes, int32_t rows, int32_t h, int32_t dtype, void* stream) {
  if (!dev_dy || !dev_x || !dev_mean || !dev_rstd || !dev_gain || !dev_dx || !dev_dgain || !dev_scratch || !rows_ok(rows, h, dtype))
    return FT_EINVAL;
  if (lddy < h || ldx < h || lddx < h || (dev_resid && ldr < h)) return FT_EINVAL;
  if (!elem_aligned(dev_dy, dtype) || !elem_aligned(dev_x, dtype) || !elem_aligned(dev_gain, dtype) ||
      !elem_aligned(dev_resid, dtype) || !elem_aligned(dev_dx, dtype) || (reinterpret_cast<uintptr_t>(dev_scratch) & 15u) != 0)
    return FT_EINVAL;
  if (scratch_bytes < fs::layernorm_scratch_bytes(rows, h)) return FT_ENOMEM;
  cudaError_t e = fs::layernorm_bwd(dev_dy, lddy, dev_x, ldx, dev_mean, dev_rstd, dev_gain, dev_resid, ldr, dev_dx, lddx, dev_dgain,
                                    dev_dbias, reinterpret_cast<float*>(dev_scratch), rows, h, dtype,
                                    reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}
