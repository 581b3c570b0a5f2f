// LayerNorm, forward and backward, over rows of any width and stride.  Reductions run in a fixed order (no floating-point
// atomics), statistics and sums are fp32, each output is rounded once.
//
// A row belongs to a group of warps; a thread holds EPL elements of it as chunks of VEC, chunk k of thread l of the group
// being elements (k threads + l) VEC, so every load of a warp is one contiguous run.  A thread thus owns the same columns of
// every row it meets: gains and biases stay in registers (read again for every row they would double the L1 traffic), and
// so do its shares of the gain and bias gradients.
//
// Rows come through a ring of NS slots in shared memory, filled by asynchronous copies that each thread issues for its own
// elements NS - 1 rows ahead: the loads of a row do not wait for the reductions of the one before, and cost no registers.
// NS = 0, for rows that are only 2-byte aligned, reads global memory directly.
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

// The elements of one thread in a ring of NS rows of NT tensors (NS = 0: no ring).
template <typename T, int VEC, int NCH, int NT, int NS>
struct RowRing {
  using V = RowVec<T, VEC>;
  typedef typename V::Raw Raw;
  static constexpr int SLOT = (int)sizeof(Raw), PAIRS = NCH * VEC / 2;
  uint32_t base;  // this thread's first slot
  int threads;
  static constexpr size_t bytes(int threads) { return (size_t)(NS * NT * NCH * SLOT) * threads; }
  __device__ __forceinline__ RowRing(const void* smem, int threads) : base(smem_u32(smem) + threadIdx.x * SLOT), threads(threads) {}
  __device__ __forceinline__ uint32_t slot(int stage, int t, int k) const { return base + (uint32_t)(((stage * NT + t) * NCH + k) * threads * SLOT); }
  __device__ __forceinline__ void fetch(int stage, int t, const T* row, bool live, int first, int stride, int h) const {
    if constexpr (NS > 0) {
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        const int c = first + k * stride;
        const bool ok = live && c < h;
        async_copy<SLOT>(slot(stage, t, k), ok ? row + c : row, ok);
      }
    }
  }
  // this thread's elements of tensor t of the row in `stage` (row: where it lies in global memory, read when there is no
  // ring); 0 outside the row
  __device__ __forceinline__ void get(int stage, int t, const T* row, int first, int stride, int h, float2 (&v)[PAIRS]) const {
    float f[NCH * VEC];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      Raw r;
      if constexpr (NS > 0) {
        const uint32_t at = slot(stage, t, k);
        uint32_t* w = reinterpret_cast<uint32_t*>(&r);
        if constexpr (SLOT == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
        else if constexpr (SLOT == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
        else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
      } else {
        const int c = first + k * stride;
        r = c < h ? V::load(row + c) : V::zero();
      }
      float u[VEC];
      V::unpack(r, u);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[k * VEC + e] = u[e];
    }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) v[i] = make_float2(f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ static void put(T* row, int first, int stride, int h, const float2 (&v)[PAIRS]) {
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = first + k * stride;
      if (c < h) {
        float u[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] = (k * VEC + e) & 1 ? v[(k * VEC + e) / 2].y : v[(k * VEC + e) / 2].x;
        V::store(row + c, u);
      }
    }
  }
};

// A row vector (gain, bias) in registers: as fp32 pairs where a thread has few columns of it, packed as it came otherwise.
template <typename T, int VEC, int NCH>
struct RowConst {
  using V = RowVec<T, VEC>;
  static constexpr int PAIRS = NCH * VEC / 2;
  static constexpr bool WIDE = PAIRS > 8;
  float2 v[WIDE ? 1 : PAIRS];
  const T* p;
  __device__ __forceinline__ void init(const T* ptr, int first, int stride, int h) {
    p = ptr;
    if constexpr (!WIDE) fill(first, stride, h, v);
  }
  __device__ __forceinline__ void fill(int first, int stride, int h, float2 (&o)[PAIRS]) const {
    float f[NCH * VEC];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = first + k * stride;
      float u[VEC];
      V::unpack(p != nullptr && c < h ? V::load(p + c) : V::zero(), u);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[k * VEC + e] = u[e];
    }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) o[i] = make_float2(f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ void get(int first, int stride, int h, float2 (&o)[PAIRS]) const {
    if constexpr (WIDE) {
      fill(first, stride, h, o);  // stays in L1
    } else {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) o[i] = v[i];
    }
  }
};

// ---------------------------------------------------------------- forward
// y = (x - mean) rstd gain + bias.  The row stays in registers: first the mean, then the centred sum of squares (the
// difference of sum(x^2) / h and mean^2 would lose the variance of rows whose mean is large).
template <typename T, int VEC, int NCH, int NS, int MAXT>
__global__ void __launch_bounds__(MAXT)
layernorm_fwd_kernel(const T* x, long long ldx, const T* __restrict__ gain, const T* __restrict__ bias, T* y, long long ldy,
                     float* __restrict__ mean, float* __restrict__ rstd, int rows, int h, int gw, float eps) {
  using Ring = RowRing<T, VEC, NCH, 1, NS>;
  constexpr int PAIRS = Ring::PAIRS;
  pdl_trigger();
  pdl_wait();
  extern __shared__ __align__(16) uint8_t ring_mem[];
  __shared__ float s_part[2][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / gw, gwarp = warp - group * gw, groups = (blockDim.x >> 5) / gw;
  const int first = (gwarp * 32 + lane) * VEC, stride = gw * 32 * VEC;
  const float inv_h = 1.0f / (float)h;
  const Ring ring(ring_mem, blockDim.x);
  // sum over the group; every thread gets the same bits.  The two sums of a row use different slots: each slot's readers
  // have passed the other's barrier before it is written again.
  auto group_sum = [&](float2 p, int which) {
    const float v = warp_sum(p.x + p.y);
    if (gw == 1) return v;
    if (lane == 0) s_part[which][warp] = v;
    group_sync(group, gw * 32);
    float t = s_part[which][group * gw];
    for (int w = 1; w < gw; ++w) t += s_part[which][group * gw + w];
    return t;
  };
  const long long step = (long long)gridDim.x * groups;
  long long row = (long long)blockIdx.x * groups + group, ahead = row;
#pragma unroll
  for (int s = 0; s < NS - 1; ++s, ahead += step) {
    ring.fetch(s, 0, x + (ahead < rows ? ahead : 0) * ldx, ahead < rows, first, stride, h);
    async_commit();
  }
  RowConst<T, VEC, NCH> cg, cb;
  cg.init(gain, first, stride, h);
  cb.init(bias, first, stride, h);
  int stage = 0;
  for (; row < rows; row += step, ahead += step) {
    if constexpr (NS > 0) {
      ring.fetch(stage == 0 ? NS - 1 : stage - 1, 0, x + (ahead < rows ? ahead : 0) * ldx, ahead < rows, first, stride, h);
      async_commit();
      async_wait<NS - 1>();
    }
    float2 v[PAIRS], s = both(0.f), ss = both(0.f);
    ring.get(stage, 0, x + row * ldx, first, stride, h, v);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) s = add2(s, v[i]);
    const float mu = group_sum(s, 0) * inv_h;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      float2 m = both(-mu);  // columns outside the row stay 0
      if (first + (2 * i / VEC) * stride >= h) m.x = 0.f;
      if (first + ((2 * i + 1) / VEC) * stride >= h) m.y = 0.f;
      v[i] = add2(v[i], m);
      ss = fma2(v[i], v[i], ss);
    }
    const float rs = 1.0f / sqrtf(group_sum(ss, 1) * inv_h + eps);
    if (gwarp == 0 && lane == 0) {
      mean[row] = mu;
      rstd[row] = rs;
    }
    float2 g[PAIRS], b[PAIRS];
    cg.get(first, stride, h, g);
    cb.get(first, stride, h, b);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) v[i] = fma2(mul2(v[i], both(rs)), g[i], b[i]);
    Ring::put(y + row * ldy, first, stride, h, v);
    if (NS > 0 && ++stage == NS) stage = 0;
  }
}

// ---------------------------------------------------------------- backward
// dx = rstd (g - mean_h(g) - xhat mean_h(g xhat)) + resid with g = dy gain; dgain = sum over rows of dy xhat, dbias of dy.
// g and xhat stay in registers between the two sums of a row and its update.  A block leaves one partial row of dgain and
// dbias, which a second kernel adds in block order.
template <typename T, int VEC, int NCH, int NS, int MAXT>
__global__ void __launch_bounds__(MAXT, 1)
layernorm_bwd_kernel(const T* dy, long long lddy, const T* x, long long ldx, const float* __restrict__ mean,
                     const float* __restrict__ rstd, const T* __restrict__ gain, const T* resid, long long ldr, T* dx, long long lddx,
                     float* __restrict__ partial, int rows, int h, int gw) {
  using Ring = RowRing<T, VEC, NCH, 3, NS>;
  constexpr int PAIRS = Ring::PAIRS;
  pdl_trigger();
  pdl_wait();
  // the ring; after the last row the groups of a block add their column sums in its place
  extern __shared__ __align__(16) uint8_t ring_mem[];
  __shared__ float s_part[2][16][2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / gw, gwarp = warp - group * gw, groups = (blockDim.x >> 5) / gw;
  const int first = (gwarp * 32 + lane) * VEC, stride = gw * 32 * VEC;
  const float inv_h = 1.0f / (float)h;
  const Ring ring(ring_mem, blockDim.x);
  const long long step = (long long)gridDim.x * groups;
  long long row = (long long)blockIdx.x * groups + group, ahead = row;
  auto fetch = [&](int stage) {
    const bool live = ahead < rows;
    const long long r = live ? ahead : 0;
    ring.fetch(stage, 0, dy + r * lddy, live, first, stride, h);
    ring.fetch(stage, 1, x + r * ldx, live, first, stride, h);
    if (resid != nullptr) ring.fetch(stage, 2, resid + r * ldr, live, first, stride, h);
    ahead += step;
    async_commit();
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) fetch(s);
  float mu_next = row < rows ? mean[row] : 0.f, rs_next = row < rows ? rstd[row] : 0.f;
  RowConst<T, VEC, NCH> cg;
  cg.init(gain, first, stride, h);
  float2 acc_g[PAIRS], acc_b[PAIRS];
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) acc_g[i] = acc_b[i] = both(0.f);
  int parity = 0, stage = 0;
  for (; row < rows; row += step) {
    const float mu = mu_next, rs = rs_next;
    if constexpr (NS > 0) fetch(stage == 0 ? NS - 1 : stage - 1);
    if (row + step < rows) {
      mu_next = mean[row + step];
      rs_next = rstd[row + step];
    }
    if constexpr (NS > 0) async_wait<NS - 1>();
    float2 a[PAIRS], xh[PAIRS], g[PAIRS], p1 = both(0.f), p2 = both(0.f);
    ring.get(stage, 0, dy + row * lddy, first, stride, h, a);
    ring.get(stage, 1, x + row * ldx, first, stride, h, xh);
    cg.get(first, stride, h, g);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      xh[i] = mul2(add2(xh[i], both(-mu)), both(rs));  // outside the row a = 0 and what xh holds does not matter
      acc_g[i] = fma2(a[i], xh[i], acc_g[i]);
      acc_b[i] = add2(a[i], acc_b[i]);
      a[i] = mul2(a[i], g[i]);
      p1 = add2(p1, a[i]);
      p2 = fma2(a[i], xh[i], p2);
    }
    float s1 = p1.x + p1.y, s2 = p2.x + p2.y;
    {  // both sums in 6 shuffles: the half warps keep one each after the first
      const bool up = (lane & 16) != 0;
      float v = (up ? s2 : s1) + __shfl_xor_sync(0xffffffffu, up ? s1 : s2, 16);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if ((lane & 15) == 0) s_part[parity][warp][lane >> 4] = v;
    }
    if (gw == 1) __syncwarp(); else group_sync(group, gw * 32);
    s1 = s_part[parity][group * gw][0];
    s2 = s_part[parity][group * gw][1];
    for (int w = 1; w < gw; ++w) {
      s1 += s_part[parity][group * gw + w][0];
      s2 += s_part[parity][group * gw + w][1];
    }
    parity ^= 1;  // the other slot is free: everyone passed this barrier after its last reads
    const float2 c1 = both(-rs * (s1 * inv_h)), c2 = both(-rs * (s2 * inv_h));
    if (resid != nullptr) {
      float2 q[PAIRS];
      ring.get(stage, 2, resid + row * ldr, first, stride, h, q);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) a[i] = add2(fma2(a[i], both(rs), fma2(xh[i], c2, c1)), q[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) a[i] = fma2(a[i], both(rs), fma2(xh[i], c2, c1));
    }
    Ring::put(dx + row * lddx, first, stride, h, a);
    if (NS > 0 && ++stage == NS) stage = 0;
  }
  // One partial row a block.  Its groups leave their sums side by side in shared memory and all threads add them, in group
  // order.
  float* out = partial + (long long)blockIdx.x * 2 * h;
  float* col = reinterpret_cast<float*>(ring_mem);
  if (groups > 1) {
    if constexpr (NS > 0) async_wait<0>();
    __syncthreads();
  }
  float* mine = groups > 1 ? col + (long long)group * 2 * h : out;
#pragma unroll
  for (int i = 0; i < PAIRS * 2; ++i) {
    const int c = first + (i / VEC) * stride + i % VEC;
    if (c < h) {
      mine[c] = i & 1 ? acc_g[i / 2].y : acc_g[i / 2].x;
      mine[h + c] = i & 1 ? acc_b[i / 2].y : acc_b[i / 2].x;
    }
  }
  if (groups > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * h; c += blockDim.x) {
      float t = col[c];
      for (int g = 1; g < groups; ++g) t += col[(long long)g * 2 * h + c];
      out[c] = t;
    }
  }
}

// Column sums of the block partials in a fixed order: a CTA takes 32 columns, 32 strided subsets of the blocks run side by
// side (each thread reads 4 columns at a time where they are aligned) and are then added in subset order.
template <int VEC>
__global__ void __launch_bounds__(32 * 32 / VEC)
layernorm_colsum_kernel(const float* __restrict__ partial, float* __restrict__ dgain, float* __restrict__ dbias, int nblk, int h) {
  using V = RowVec<float, VEC>;
  pdl_trigger();
  pdl_wait();
  __shared__ float s[32][33];
  constexpr int TX = 32 / VEC;
  const int cx = threadIdx.x % TX, ry = threadIdx.x / TX;
  const int cols = dbias != nullptr ? 2 * h : h;
  const int c = blockIdx.x * 32 + cx * VEC;
  float a[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = 0.f;
  if (c < cols) {
#pragma unroll 4
    for (int b = ry; b < nblk; b += 32) {
      float f[VEC];
      V::unpack(V::load(partial + (long long)b * 2 * h + c), f);
#pragma unroll
      for (int e = 0; e < VEC; ++e) a[e] += f[e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[ry][cx * VEC + e] = a[e];
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const int col = blockIdx.x * 32 + threadIdx.x;
  if (col >= cols) return;
  float tot = 0.f;
#pragma unroll
  for (int w = 0; w < 32; ++w) tot += s[w][threadIdx.x];
  if (col < h) dgain[col] = tot; else dbias[col - h] = tot;
}

int blocks_for(int rows, int groups, int most) {
  const long long want = ((long long)rows + groups - 1) / groups;
  return (int)(want < most ? want : most);
}

// Elements a thread holds of a row.  16 up to 8192 columns and 32 beyond, so that a group never exceeds 16 warps; 8 where a
// warp covers the row with them, and for rows whose accesses are narrower than 16 bytes (every one of them is an
// instruction: fewer a thread, more threads; 4099 x 771 fp32 backward 17.7 us with 8, 28.7 with 16).
int elements_per_thread(int h, bool narrow) { return h <= 256 || (narrow && h <= 4096) ? 8 : h <= 8192 ? 16 : 32; }

template <typename T, int VEC, int EPL, int NS, int MAXT>
cudaError_t fwd_launch(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean, float* rstd,
                       int rows, int h, float eps, cudaStream_t st) {
  using Ring = RowRing<T, VEC, EPL / VEC, 1, NS>;
  auto kern = layernorm_fwd_kernel<T, VEC, EPL / VEC, NS, MAXT>;
  const int gw = (h + 32 * EPL - 1) / (32 * EPL);
  int groups = MAXT / 32 / gw;
  if (rows <= kSms * groups) groups = 1;  // few rows: spread them over the SMs
  const int threads = groups * gw * 32;
  static unsigned long long smem_set = 0;
  cudaError_t e = ensure_dynamic_smem(kern, (int)Ring::bytes(MAXT), smem_set);
  if (e != cudaSuccess) return e;
  // 768 threads an SM (8192 x 2048 bf16: 3 blocks of 256 15.9 us, 1 of 512 20.2, 4 of 256 18.9; as many as fit 17.0)
  return launch_pdl(kern, dim3(blocks_for(rows, groups, kSms * (MAXT == 256 ? 3 : 1))), dim3(threads), Ring::bytes(threads), st,
                    reinterpret_cast<const T*>(x), (long long)ldx, reinterpret_cast<const T*>(gain), reinterpret_cast<const T*>(bias),
                    reinterpret_cast<T*>(y), (long long)ldy, mean, rstd, rows, h, gw, eps);
}

template <typename T, int VEC>
cudaError_t fwd_width(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean, float* rstd,
                      int rows, int h, float eps, cudaStream_t st) {
  constexpr int NS = VEC * sizeof(T) >= 4 ? 3 : 0;
  const int epl = elements_per_thread(h, VEC * sizeof(T) < 16);
#define LN_FWD_W(EPL, MAXT) fwd_launch<T, VEC, EPL, NS, MAXT>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st)
  const bool small = h <= 256 * epl;  // a row fits a block of 256 threads
  if (epl == 8) return small ? LN_FWD_W(8, 256) : LN_FWD_W(8, 512);
  if (epl == 16) return small ? LN_FWD_W(16, 256) : LN_FWD_W(16, 512);
  return LN_FWD_W(32, 512);
#undef LN_FWD_W
}

template <typename T, int VEC, int EPL, int NS>
cudaError_t bwd_launch(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd, const void* gain,
                       const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias, float* scratch, int rows,
                       int h, cudaStream_t st) {
  using Ring = RowRing<T, VEC, EPL / VEC, 3, NS>;
  auto kern = layernorm_bwd_kernel<T, VEC, EPL / VEC, NS, 512>;
  const int gw = (h + 32 * EPL - 1) / (32 * EPL), groups = 16 / gw, threads = groups * gw * 32;
  const int blocks = blocks_for(rows, groups, kSms);
  const size_t col = groups > 1 ? (size_t)groups * 2 * h * sizeof(float) : 0;  // at most 2 * 512 * EPL floats
  constexpr size_t most = Ring::bytes(512) > 4096 * EPL ? Ring::bytes(512) : 4096 * EPL;
  static unsigned long long smem_set = 0;
  cudaError_t e = ensure_dynamic_smem(kern, (int)most, smem_set);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kern, dim3(blocks), dim3(threads), Ring::bytes(threads) > col ? Ring::bytes(threads) : col, st,
                 reinterpret_cast<const T*>(dy), (long long)lddy, reinterpret_cast<const T*>(x), (long long)ldx, mean, rstd,
                 reinterpret_cast<const T*>(gain), reinterpret_cast<const T*>(resid), (long long)ldr, reinterpret_cast<T*>(dx),
                 (long long)lddx, scratch, rows, h, gw);
  if (e != cudaSuccess) return e;
  const int cols = dbias != nullptr ? 2 * h : h;
  if (h % 4 == 0) return launch_pdl(layernorm_colsum_kernel<4>, dim3((cols + 31) / 32), dim3(256), 0, st, scratch, dgain, dbias, blocks, h);
  return launch_pdl(layernorm_colsum_kernel<1>, dim3((cols + 31) / 32), dim3(1024), 0, st, scratch, dgain, dbias, blocks, h);
}

template <typename T, int VEC>
cudaError_t bwd_width(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd, const void* gain,
                      const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias, float* scratch, int rows,
                      int h, cudaStream_t st) {
  // two rows in the ring: one under way hides the memory (a third changes nothing); none where 512 threads' slots would
  // not fit an SM's shared memory (fp32 rows of more than 8192 columns) or the accesses are too narrow to be copied
  constexpr bool RING = VEC * sizeof(T) >= 4;
#define LN_BWD_W(EPL, NS) bwd_launch<T, VEC, EPL, RING ? NS : 0>(dy, lddy, x, ldx, mean, rstd, gain, resid, ldr, dx, lddx, dgain, dbias, scratch, rows, h, st)
  const int epl = elements_per_thread(h, VEC * sizeof(T) < 16);
  return epl == 8 ? LN_BWD_W(8, 2) : epl == 16 ? LN_BWD_W(16, 2) : LN_BWD_W(32, (sizeof(T) == 2 ? 2 : 0));
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
  return (size_t)(rows < kSms ? rows : kSms) * 2 * (size_t)h * sizeof(float);  // one partial row of both gradients a block
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
