// LayerNorm, forward and backward, over rows of any width and stride.  Reductions run in a fixed order (no floating-point
// atomics), statistics and sums are fp32, each output is rounded once.
//
// A row belongs to a group of warps; a thread holds EPL elements of it as chunks of VEC, chunk k of thread l of the group
// being elements (k threads + l) VEC, so every load of a warp is one contiguous run.  A thread thus owns the same columns of
// every row it meets: gains and biases stay in registers (read again for every row they would double the L1 traffic), and
// so do its shares of the gain and bias gradients.
//
// Rows come through a ring of NS slots in shared memory, filled by asynchronous copies that each thread issues NS - 1 rows
// ahead: the loads of a row do not wait for the reductions of the one before, and cost no registers.
#include "layernorm.cuh"

#include "../../include/forgestep.h"
#include "rows.cuh"

namespace fs {
namespace {

constexpr int kSms = 148;

// barrier of a group of `warps` warps (bar 0 is __syncthreads; a block has at most 8 groups of more than one warp)
__device__ __forceinline__ void group_sync(int group, int warps) {
  if (warps == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(warps * 32) : "memory");
}

// The elements of one thread in a ring of NS rows of NT tensors (NS = 0: no ring).  A thread copies its own chunks and needs
// no barrier.
template <typename T, int VEC, int EPL, int NT, int NS>
struct RowRing {
  static constexpr bool kShared = false;  // slots between the threads of a group
  static constexpr int NCH = EPL / VEC, PAIRS = EPL / 2;
  using V = RowVec<T, VEC>;
  typedef typename V::Raw Raw;
  static constexpr int SLOT = (int)sizeof(Raw);
  uint32_t base;  // this thread's first slot
  int threads, first, stride, h;
  static constexpr size_t bytes(int threads) { return (size_t)(NS * NT * NCH * SLOT) * threads; }
  // l: this thread's number among the gthreads of its group
  __device__ __forceinline__ RowRing(const void* smem, int gthreads, int l, int h, const T*)
      : base(smem_u32(smem) + threadIdx.x * SLOT), threads(blockDim.x), first(l * VEC), stride(gthreads * VEC), h(h) {}
  __device__ __forceinline__ uint32_t slot(int stage, int t, int k) const { return base + (uint32_t)(((stage * NT + t) * NCH + k) * threads * SLOT); }
  // column of this thread's element i, and whether the row has it
  __device__ __forceinline__ int column(int i) const { return first + i / VEC * stride + i % VEC; }
  __device__ __forceinline__ bool inside(int i) const { return first + i / VEC * stride < h; }
  __device__ __forceinline__ void fetch(int stage, int t, const T* row, bool live, bool) const {
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
  __device__ __forceinline__ void get(int stage, int t, const T* row, float2 (&v)[PAIRS]) const {
    float f[EPL];
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
  // the same of a vector that every row uses (null: 0)
  __device__ __forceinline__ void constant(const T* p, float2 (&v)[PAIRS]) const {
    float f[EPL];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = first + k * stride;
      float u[VEC];
      V::unpack(p != nullptr && c < h ? V::load(p + c) : V::zero(), u);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[k * VEC + e] = u[e];
    }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) v[i] = make_float2(f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ void put(T* row, const float2 (&v)[PAIRS]) const {
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

// The same for bf16 rows that start at any element.  Chunks of 8 are cut at the 16-byte boundaries of the OUTPUT rows (the
// first and the last of a row are partial), so that all others are stored whole; a group takes only rows that start equally far
// behind a boundary, which keeps its threads' columns.  The ring holds the aligned pieces of the input rows, and a thread
// puts a chunk together from its own piece and its neighbour's: the group passes a barrier between the pieces' arrival and
// get, and another one before the slot is filled again.
template <int EPL, int NT, int NS>
struct EdgeRing {
  static constexpr bool kShared = true;
  static constexpr int VEC = 8, NCH = EPL / VEC, PAIRS = EPL / 2;
  uint32_t base;  // this thread's first slot
  int threads, first, stride, h;
  bool last;      // thread of its group
  static constexpr size_t bytes(int threads) { return (size_t)(NS * NT * NCH * 16) * threads; }
  // out: an output row of the group
  __device__ __forceinline__ EdgeRing(const void* smem, int gthreads, int l, int h, const bf16* out)
      : base(smem_u32(smem) + threadIdx.x * 16), threads(blockDim.x), first(l * VEC - behind_boundary(out)), stride(gthreads * VEC), h(h),
        last(l == gthreads - 1) {}
  __device__ __forceinline__ uint32_t slot(int stage, int t, int k) const { return base + (uint32_t)(((stage * NT + t) * NCH + k) * threads * 16); }
  __device__ __forceinline__ int column(int i) const { return first + i / VEC * stride + i % VEC; }
  __device__ __forceinline__ bool inside(int i) const { return (unsigned)column(i) < (unsigned)h; }
  __device__ __forceinline__ bool partial(int k) const { return first + k * stride < 0 || first + k * stride + VEC > h; }
  // inner: the 15 bytes on either side of the row are inside the tensor too
  __device__ __forceinline__ void fetch(int stage, int t, const bf16* row, bool live, bool inner) const {
    const int d = behind_boundary(row + first);  // the same in all threads and chunks
    const bf16* at = row + first - d;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      // a piece that holds nothing of the row is left out
      if (!live || (unsigned)(first - d + VEC - 1 + k * stride) >= (unsigned)(h + VEC - 1)) continue;
      if (inner) {
        async_copy<16>(slot(stage, t, k), at + k * stride, true);
      } else {
#pragma unroll 1
        for (int e = 0; e < VEC; ++e) {
          const bf16* p = at + k * stride + e;
          if (p >= row && p < row + h)
            asm volatile("st.shared.b16 [%0], %1;" ::"r"(slot(stage, t, k) + e * 2), "h"(*reinterpret_cast<const unsigned short*>(p)) : "memory");
        }
      }
    }
  }
  static __device__ __forceinline__ uint4 load(uint32_t at) {
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at) : "memory");
    return r;
  }
  __device__ __forceinline__ void spread(int k, const uint4& r, float2 (&v)[PAIRS]) const {
    float u[VEC];
    unpack_piece(r, u);
    if (partial(k)) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (!inside(k * VEC + e)) u[e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) v[k * VEC / 2 + i] = make_float2(u[2 * i], u[2 * i + 1]);
  }
  __device__ __forceinline__ void get(int stage, int t, const bf16* row, float2 (&v)[PAIRS]) const {
    const int d = behind_boundary(row + first);
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      uint4 r = load(slot(stage, t, k));
      if (d != 0) {  // behind the group's last piece lies nothing of the row
        const uint32_t next = !last ? slot(stage, t, k) + 16 : slot(stage, t, k + 1 < NCH ? k + 1 : k) - (uint32_t)(stride / VEC - 1) * 16;
        r = realign(r, load(next), d, 2);
      }
      spread(k, r, v);
    }
  }
  __device__ __forceinline__ void constant(const bf16* p, float2 (&v)[PAIRS]) const {
#pragma unroll
    for (int i = 0; i < PAIRS; ++i)
      v[i] = make_float2(p != nullptr && inside(2 * i) ? to_float(p[column(2 * i)]) : 0.f,
                         p != nullptr && inside(2 * i + 1) ? to_float(p[column(2 * i + 1)]) : 0.f);
  }
  __device__ __forceinline__ void put(bf16* row, const float2 (&v)[PAIRS]) const {
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      bf16* out = row + first + k * stride;
      if (!partial(k)) {
        const float2* p = v + k * VEC / 2;
        *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(p[0].x, p[0].y), pack_bf16(p[1].x, p[1].y), pack_bf16(p[2].x, p[2].y), pack_bf16(p[3].x, p[3].y));
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (inside(k * VEC + e)) store_one(out + e, e & 1 ? v[(k * VEC + e) / 2].y : v[(k * VEC + e) / 2].x);
      }
    }
  }
};

// VEC = 0: EdgeRing.
template <typename T, int VEC, int EPL, int NT, int NS>
struct RingOf {
  typedef RowRing<T, VEC, EPL, NT, NS> type;
};
template <int EPL, int NT, int NS>
struct RingOf<bf16, 0, EPL, NT, NS> {
  typedef EdgeRing<EPL, NT, NS> type;
};

// A row vector (gain, bias) in registers, where a thread has few columns of it; read again for every row otherwise.
template <typename Ring, typename T>
struct RowConst {
  static constexpr int PAIRS = Ring::PAIRS;
  static constexpr bool WIDE = PAIRS > 8;
  float2 v[WIDE ? 1 : PAIRS];
  const T* p;
  __device__ __forceinline__ void init(const T* ptr, const Ring& ring) {
    p = ptr;
    if constexpr (!WIDE) ring.constant(p, v);
  }
  __device__ __forceinline__ void get(const Ring& ring, float2 (&o)[PAIRS]) const {
    if constexpr (WIDE) {
      ring.constant(p, o);  // stays in L1
    } else {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) o[i] = v[i];
    }
  }
};

// The 15 bytes on either side of this row are inside the tensor too: it has rows of 16 bytes before and behind.
__device__ __forceinline__ bool inner_row(long long row, int rows, int h) { return row > 0 && row + 1 < rows && h >= 8; }

// ---------------------------------------------------------------- forward
// y = (x - mean) rstd gain + bias.  The row stays in registers: first the mean, then the centred sum of squares (the
// difference of sum(x^2) / h and mean^2 would lose the variance of rows whose mean is large).  Bound by memory: 8192 x 2048
// bf16 11.4 us (5.9 TB/s), fp32 21.3 (6.3 TB/s); 8192 x 2047 bf16 30 us, by instructions.
template <typename T, int VEC, int EPL, int NS, int MAXT, int GW>
__global__ void __launch_bounds__(VEC == 0 && EPL <= 16 ? 1024 : MAXT == 256 ? 768 : MAXT)  // of all blocks of an SM (fwd_launch)
layernorm_fwd_kernel(const T* x, long long ldx, const T* __restrict__ gain, const T* __restrict__ bias, T* y, long long ldy,
                     float* __restrict__ mean, float* __restrict__ rstd, int rows, int h, int any_gw, float eps) {
  const int gw = GW > 0 ? GW : any_gw;  // warps of a group
  using Ring = typename RingOf<T, VEC, EPL, 1, NS>::type;
  constexpr int PAIRS = Ring::PAIRS;
  pdl_trigger();
  pdl_wait();
  extern __shared__ __align__(16) uint8_t ring_mem[];
  __shared__ float s_part[2][MAXT / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / gw, gwarp = warp - group * gw, groups = (blockDim.x >> 5) / gw;
  const float inv_h = 1.0f / (float)h;
  const long long step = (long long)gridDim.x * groups;
  long long row = (long long)blockIdx.x * groups + group, ahead = row;
  const Ring ring(ring_mem, gw * 32, gwarp * 32 + lane, h, y + row * ldy);
  const T* x_ahead = x + ahead * ldx;
  auto fetch = [&](int stage) {
    const bool live = ahead < rows;
    ring.fetch(stage, 0, live ? x_ahead : x, live, inner_row(ahead, rows, h));
    ahead += step;
    x_ahead += step * ldx;
    async_commit();
  };
  // sum over the group; every thread gets the same bits.  The two sums of a row use different slots: each slot's readers
  // have passed the other's barrier before it is written again.
  auto group_sum = [&](float2 p, int which) {
    const float v = warp_sum(p.x + p.y);
    if (gw == 1) return v;
    if (lane == 0) s_part[which][warp] = v;
    group_sync(group, gw);
    float t = s_part[which][group * gw];
#pragma unroll
    for (int w = 1; w < (GW > 0 ? GW : gw); ++w) t += s_part[which][group * gw + w];
    return t;
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) fetch(s);
  RowConst<Ring, T> cg, cb;
  cg.init(gain, ring);
  cb.init(bias, ring);
  int stage = 0;
  for (; row < rows; row += step) {
    fetch(stage == 0 ? NS - 1 : stage - 1);
    async_wait<NS - 1>();
    if (Ring::kShared) group_sync(group, gw);
    float2 v[PAIRS], s = both(0.f), ss = both(0.f);
    ring.get(stage, 0, x + row * ldx, v);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) s = add2(s, v[i]);
    const float mu = group_sum(s, 0) * inv_h;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      float2 m = both(-mu);  // columns outside the row stay 0
      if (!ring.inside(2 * i)) m.x = 0.f;
      if (!ring.inside(2 * i + 1)) m.y = 0.f;
      v[i] = add2(v[i], m);
      ss = fma2(v[i], v[i], ss);
    }
    const float rs = rsqrtf(group_sum(ss, 1) * inv_h + eps);  // within 2 units of the last place
    if (gwarp == 0 && lane == 0) {
      mean[row] = mu;
      rstd[row] = rs;
    }
    float2 g[PAIRS], b[PAIRS];
    cg.get(ring, g);
    cb.get(ring, b);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) v[i] = fma2(mul2(v[i], both(rs)), g[i], b[i]);
    ring.put(y + row * ldy, v);
    if (++stage == NS) stage = 0;
  }
}

// ---------------------------------------------------------------- backward
// dx = rstd (g - mean_h(g) - xhat mean_h(g xhat)) + resid with g = dy gain; dgain = sum over rows of dy xhat, dbias of dy.
// g and xhat stay in registers between the two sums of a row and its update.  A block leaves one partial row of dgain and
// dbias, which a second kernel adds in block order; small calls are one cluster of blocks (dgain given), which add them through
// distributed shared memory.  Bound by memory beside 7 us of start, drain and column sums: 8192 x
// 2048 bf16 with resid 27.8 us for 134 MB; 8192 x 2047 bf16 58 us with resid, 47 without, by instructions.
template <typename T, int VEC, int EPL, int NS, int MAXT, int GW>
__global__ void __launch_bounds__(MAXT, 1)
layernorm_bwd_kernel(const T* dy, long long lddy, const T* x, long long ldx, const float* __restrict__ mean,
                     const float* __restrict__ rstd, const T* __restrict__ gain, const T* resid, long long ldr, T* dx, long long lddx,
                     float* __restrict__ partial, float* __restrict__ dgain, float* __restrict__ dbias, int rows, int h, int hp, int any_gw) {
  const int gw = GW > 0 ? GW : any_gw;  // warps of a group
  using Ring = typename RingOf<T, VEC, EPL, 3, NS>::type;
  constexpr int PAIRS = Ring::PAIRS;
  pdl_trigger();
  pdl_wait();
  // the ring; after the last row the groups of a block add their column sums in its place
  extern __shared__ __align__(16) uint8_t ring_mem[];
  __shared__ float s_part[2][MAXT / 32][2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / gw, gwarp = warp - group * gw, groups = (blockDim.x >> 5) / gw;
  const float inv_h = 1.0f / (float)h;
  const long long step = (long long)gridDim.x * groups;
  long long row = (long long)blockIdx.x * groups + group, ahead = row;
  const Ring ring(ring_mem, gw * 32, gwarp * 32 + lane, h, dx + row * lddx);
  // Rows found by advancing pointers for words of 4 bytes (20000 x 771 fp32: 45.3 us against 47.6), by multiplication elsewhere
  // (20000 x 771 bf16: 35.4 against 41.4, whose registers the pointers would need)
  constexpr bool STEP = VEC * sizeof(T) == 4;
  const T *dy_ahead = dy + ahead * lddy, *x_ahead = x + ahead * ldx, *r_ahead = resid != nullptr ? resid + ahead * ldr : nullptr;
  auto fetch = [&](int stage) {
    const bool live = ahead < rows;
    const bool inner = inner_row(ahead, rows, h);
    const long long r = live ? ahead : 0;
    ring.fetch(stage, 0, STEP ? (live ? dy_ahead : dy) : dy + r * lddy, live, inner);
    ring.fetch(stage, 1, STEP ? (live ? x_ahead : x) : x + r * ldx, live, inner);
    if (resid != nullptr) ring.fetch(stage, 2, STEP ? (live ? r_ahead : resid) : resid + r * ldr, live, inner);
    ahead += step;
    if (STEP) {
      dy_ahead += step * lddy;
      x_ahead += step * ldx;
      r_ahead += step * ldr;
    }
    async_commit();
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) fetch(s);
  float mu_next = row < rows ? mean[row] : 0.f, rs_next = row < rows ? rstd[row] : 0.f;
  RowConst<Ring, T> cg;
  cg.init(gain, ring);
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
    if constexpr (NS > 0) {
      async_wait<NS - 1>();
      if (Ring::kShared) group_sync(group, gw);
    }
    float2 a[PAIRS], xh[PAIRS], g[PAIRS], q[PAIRS], p1 = both(0.f), p2 = both(0.f);
    ring.get(stage, 0, dy + row * lddy, a);
    ring.get(stage, 1, x + row * ldx, xh);
    // shared slots are read ahead of the barrier below, after which they may be filled again
    if (Ring::kShared && resid != nullptr) ring.get(stage, 2, resid + row * ldr, q);
    cg.get(ring, g);
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
    group_sync(group, gw);
    s1 = s_part[parity][group * gw][0];
    s2 = s_part[parity][group * gw][1];
#pragma unroll
    for (int w = 1; w < (GW > 0 ? GW : gw); ++w) {
      s1 += s_part[parity][group * gw + w][0];
      s2 += s_part[parity][group * gw + w][1];
    }
    parity ^= 1;  // the other slot is free: everyone passed this barrier after its last reads
    const float2 c1 = both(-rs * (s1 * inv_h)), c2 = both(-rs * (s2 * inv_h));
    if (resid != nullptr) {
      if (!Ring::kShared) ring.get(stage, 2, resid + row * ldr, q);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) a[i] = add2(fma2(a[i], both(rs), fma2(xh[i], c2, c1)), q[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) a[i] = fma2(a[i], both(rs), fma2(xh[i], c2, c1));
    }
    ring.put(dx + row * lddx, a);
    if (NS > 0 && ++stage == NS) stage = 0;
  }
  // One partial row a block.  Its groups leave their sums side by side in shared memory and all threads add them, in group
  // order.
  float* out = partial + (long long)blockIdx.x * 2 * hp;
  float* col = reinterpret_cast<float*>(ring_mem);
  const bool one_cluster = dgain != nullptr;
  if (groups > 1 || one_cluster) {
    if constexpr (NS > 0) async_wait<0>();
    __syncthreads();
    if (one_cluster) out = col;
  }
  float* mine = groups > 1 ? col + (long long)group * 2 * hp : out;
#pragma unroll
  for (int i = 0; i < PAIRS * 2; ++i) {
    if (ring.inside(i)) {
      mine[ring.column(i)] = i & 1 ? acc_g[i / 2].y : acc_g[i / 2].x;
      mine[hp + ring.column(i)] = i & 1 ? acc_b[i / 2].y : acc_b[i / 2].x;
    }
  }
  if (groups > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * hp; c += blockDim.x) {  // (what lies between h and hp is never read)
      float t = col[c];
      for (int g = 1; g < groups; ++g) t += col[(long long)g * 2 * hp + c];
      out[c] = t;
    }
  }
  if (one_cluster) {
    cluster_sync_all();
    for (int c = (int)(blockIdx.x * blockDim.x + threadIdx.x); c < 2 * hp; c += (int)(gridDim.x * blockDim.x)) {
      const int rest = c - hp;
      if ((rest < 0 && c >= h) || rest >= h || (rest >= 0 && dbias == nullptr)) continue;
      float v[8], t = 0.f;
#pragma unroll
      for (unsigned r = 0; r < 8; ++r) {
        uint32_t at;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(col + c)), "r"(r < gridDim.x ? r : 0u));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r]) : "r"(at) : "memory");
      }
#pragma unroll
      for (unsigned r = 0; r < 8; ++r)
        if (r < gridDim.x) t += v[r];
      if (rest < 0) dgain[c] = t; else dbias[rest] = t;
    }
    cluster_sync_all();  // nobody leaves while its sums are read
  }
}

// Column sums of the block partials (rows of hp columns each of dgain and dbias, hp: h rounded up to 4) in a fixed order: a CTA
// takes 32 columns, 32 strided subsets of the blocks run side by side and are then added in subset order.  Bound by latency:
// single columns and 1024 threads (8192 x 2048: 28.4 us with the kernel in front) do better than 16-byte loads by 256 (29.3).
__global__ void __launch_bounds__(1024)
layernorm_colsum_kernel(const float* __restrict__ partial, float* __restrict__ dgain, float* __restrict__ dbias, int nblk, int h, int hp) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s[32][33];
  const int cx = threadIdx.x % 32, ry = threadIdx.x / 32;
  const int cols = dbias != nullptr ? 2 * hp : hp;
  const int c = blockIdx.x * 32 + cx;
  float a = 0.f;
  if (c < cols) {
    float v[(kSms + 31) / 32];  // all in flight at once
#pragma unroll
    for (int k = 0; k < (kSms + 31) / 32; ++k) {
      const int b = ry + 32 * k;
      v[k] = b < nblk ? partial[(long long)b * 2 * hp + c] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < (kSms + 31) / 32; ++k) a += v[k];
  }
  s[ry][cx] = a;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const int col = blockIdx.x * 32 + threadIdx.x, rest = col - hp;
  if (col >= cols || (col >= h && rest < 0) || rest >= h) return;
  float tot = 0.f;
#pragma unroll
  for (int w = 0; w < 32; ++w) tot += s[w][threadIdx.x];
  if (col < h) dgain[col] = tot; else dbias[rest] = tot;
}

int blocks_for(int rows, int groups, int most) {
  const long long want = ((long long)rows + groups - 1) / groups;
  return (int)(want < most ? want : most);
}

// Blocks of a launch whose groups take every (blocks * groups)-th row, so that these start equally far behind a boundary.
int blocks_of_period(int blocks, int groups, int rows, int64_t ld) {
  int period = 1;
  while (ld * period % 8 != 0) period *= 2;
  while ((long long)blocks * groups < rows && blocks * groups % period != 0) --blocks;
  return blocks;
}

// Columns that a group has chunks for; EdgeRing: the partial chunk's in front and one chunk's behind the row too.
int cover_of(int h, int vec) { return vec == 0 ? h + 15 : h; }

// Elements a thread holds of a row.  16 up to 8192 columns and 32 beyond, so that a group never exceeds 16 warps (17 of
// EdgeRing); 8 where a warp covers the row with them, and for words of 4 bytes (every one of them is an instruction: fewer a thread,
// more threads; 20000 x 771 fp32 29 us forward and 48 backward with 8, 34 and 53 with 16; 8-byte chunks, 8192 x 2044 bf16:
// 18 and 27 with 8, 13 and 23 with 16).
int elements_per_thread(int cover, bool narrow) { return cover <= 256 || (narrow && cover <= 4096) ? 8 : cover <= 8192 ? 16 : 32; }

// Warps of a group, if the kernel is compiled for that number (0: any).  The sums over a group are then straight code, and the
// kernel's integer work shrinks: in a graph, 8192 x 2048 bf16 10.8 us forward (13.8 with any number) and 21.5 backward (22.7),
// 2048 x 8192 bf16 14.8 (22.6) and 34.3 (35.5), 20000 x 771 fp32 29.5 (42) and 47.5 (56.5), 8192 x 2047 bf16 backward 46 (51).
// (backward without resid).  Not where it was slower: EdgeRing forward (8192 x 2047: 34.7 against 30.8) and 16 warps of fp32
// backward (2048 x 8192: 46.9 against 40.5).  The numbers compiled in are those of the widths timed: powers of two and odd
// neighbours.  Widths between take the kernel for any number and pay for it: bf16 rows of 5, 10 and 12 warps, 8192 x 2560 24 us forward
// and 31 backward, 8192 x 5120 67 and 68, 8192 x 6144 70 and 75.  Whether they gain as much was not tried.
template <typename T, int VEC, int EPL, bool FWD>
constexpr int fixed_warps(int gw) {
  if (VEC == 0 && EPL == 16 && !FWD) return gw <= 5 ? gw : 0;
  if (VEC * sizeof(T) >= 8 && EPL == 16) return gw <= 4 || gw == 8 || (gw == 16 && (FWD || sizeof(T) == 2)) ? gw : 0;
  if (VEC * sizeof(T) == 4 && EPL == 8) return gw == 2 || gw == 4 || gw == 8 ? gw : 0;
  return 0;
}

// kern becomes the instantiation for gw warps, where there is one and a block of MAXT threads can hold them.
#define LN_PICK(KERNEL, FWD, N) \
  if constexpr (fixed_warps<T, VEC, EPL, FWD>(N) == N && N * 32 <= MAXT) { if (gw == N) kern = KERNEL<T, VEC, EPL, NS, MAXT, N>; }
#define LN_PICK_ALL(K, F) \
  LN_PICK(K, F, 1) LN_PICK(K, F, 2) LN_PICK(K, F, 3) LN_PICK(K, F, 4) LN_PICK(K, F, 5) LN_PICK(K, F, 8) LN_PICK(K, F, 16)

template <typename T, int VEC, int EPL, int MAXT>
cudaError_t fwd_launch(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean, float* rstd,
                       int rows, int h, float eps, cudaStream_t st) {
  constexpr int NS = 3;
  using Ring = typename RingOf<T, VEC, EPL, 1, NS>::type;
  const int gw = (cover_of(h, VEC) + 32 * EPL - 1) / (32 * EPL), fixed = fixed_warps<T, VEC, EPL, true>(gw);
  auto kern = layernorm_fwd_kernel<T, VEC, EPL, NS, MAXT, 0>;
  LN_PICK_ALL(layernorm_fwd_kernel, true)
  int groups = MAXT / 32 / gw;
  if (rows <= kSms * groups) groups = 1;  // few rows: spread them over the SMs
  const int threads = groups * gw * 32;
  static unsigned long long smem_set[17] = {};  // by kernel
  cudaError_t e = ensure_dynamic_smem(kern, (int)Ring::bytes(MAXT), smem_set[fixed]);
  if (e != cudaSuccess) return e;
  // 768 threads an SM (8192 x 2048 bf16: 3 blocks of 256 15.9 us, 1 of 512 20.2, 4 of 256 18.9; as many as fit 17.0).  EdgeRing,
  // which computes more for its bytes: 1024 (8192 x 2047: 30 us, 40 with 480)
  int blocks = blocks_for(rows, groups, kSms * (VEC == 0 && EPL <= 16 ? 1024 / MAXT : MAXT == 256 ? 3 : 1));
  if (VEC == 0) blocks = blocks_of_period(blocks, groups, rows, ldy);
  return launch_pdl(kern, dim3(blocks), dim3(threads), Ring::bytes(threads), st, reinterpret_cast<const T*>(x), (long long)ldx,
                    reinterpret_cast<const T*>(gain), reinterpret_cast<const T*>(bias), reinterpret_cast<T*>(y), (long long)ldy, mean,
                    rstd, rows, h, gw, eps);
}

template <typename T, int VEC>
cudaError_t fwd_width(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean, float* rstd,
                      int rows, int h, float eps, cudaStream_t st) {
  const int cover = cover_of(h, VEC), epl = elements_per_thread(cover, VEC * sizeof(T) == 4);
#define LN_FWD_W(EPL, MAXT) fwd_launch<T, VEC, EPL, MAXT>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st)
  const bool small = cover <= 256 * epl;  // a row fits a block of 256 threads
  if (epl == 8) return small ? LN_FWD_W(8, 256) : LN_FWD_W(8, 512);
  if (epl == 16) return small ? LN_FWD_W(16, (VEC == 0 ? 512 : 256)) : LN_FWD_W(16, 512);
  return LN_FWD_W(32, (VEC == 0 ? 544 : 512));
#undef LN_FWD_W
}

// Rows that each group of 8 blocks may take for the backward pass to be ONE launch of a cluster of them.  Up to one it is quicker
// on the GPU too (8 x 8192 bf16: 7.7 us in a graph against 14.2, 64 x 1024 6.7 and 6.9), at two the launch that a call saves
// still outweighs it (64 x 2048: 9.6 us a call against 12.1, in a graph 8.5 against 7.4); EdgeRing's rows take longer (48 x 2047 at two
// 13.9 against 12.1).
constexpr int one_cluster_rows(int vec) { return vec == 0 ? 1 : 2; }

template <typename T, int VEC, int EPL, int NS, int MAXT>
cudaError_t bwd_launch(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd, const void* gain,
                       const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias, float* scratch, int rows,
                       int h, cudaStream_t st) {
  using Ring = typename RingOf<T, VEC, EPL, 3, NS>::type;
  const int gw = (cover_of(h, VEC) + 32 * EPL - 1) / (32 * EPL), groups = MAXT / 32 / gw, threads = groups * gw * 32;
  const int fixed = fixed_warps<T, VEC, EPL, false>(gw);
  auto kern = layernorm_bwd_kernel<T, VEC, EPL, NS, MAXT, 0>;
  LN_PICK_ALL(layernorm_bwd_kernel, false)
  const int hp = (h + 3) / 4 * 4;
  const size_t col = (size_t)groups * 2 * hp * sizeof(float);  // at most 2 * MAXT * EPL floats
  constexpr size_t most = Ring::bytes(MAXT) > 8 * MAXT * EPL ? Ring::bytes(MAXT) : 8 * MAXT * EPL;
  static unsigned long long smem_set[17] = {};  // by kernel
  cudaError_t e = ensure_dynamic_smem(kern, (int)most, smem_set[fixed]);
  if (e != cudaSuccess) return e;
  const T *dyp = reinterpret_cast<const T*>(dy), *xp = reinterpret_cast<const T*>(x), *gp = reinterpret_cast<const T*>(gain), *rp = reinterpret_cast<const T*>(resid);
  T* dxp = reinterpret_cast<T*>(dx);
  float* none = nullptr;
  if (rows <= one_cluster_rows(VEC) * 8 * groups) {
    int blocks = 1;
    while (blocks < 8 && blocks * groups < rows) blocks *= 2;  // (8 blocks fit any period of rows)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = Ring::bytes(threads) > col ? Ring::bytes(threads) : col;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = g_pdl ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, dyp, (long long)lddy, xp, (long long)ldx, mean, rstd, gp, rp, (long long)ldr, dxp, (long long)lddx,
                              none, dgain, dbias, rows, h, hp, gw);
  }
  int blocks = blocks_for(rows, groups, kSms);
  if (VEC == 0) blocks = blocks_of_period(blocks, groups, rows, lddx);
  const size_t shared = groups > 1 && col > Ring::bytes(threads) ? col : Ring::bytes(threads);
  e = launch_pdl(kern, dim3(blocks), dim3(threads), shared, st, dyp, (long long)lddy, xp, (long long)ldx, mean, rstd, gp, rp, (long long)ldr,
                 dxp, (long long)lddx, scratch, none, none, rows, h, hp, gw);
  if (e != cudaSuccess) return e;
  const int cols = dbias != nullptr ? 2 * hp : hp;
  return launch_pdl(layernorm_colsum_kernel, dim3((cols + 31) / 32), dim3(1024), 0, st, scratch, dgain, dbias, blocks, h, hp);
}

template <typename T, int VEC>
cudaError_t bwd_width(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd, const void* gain,
                      const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias, float* scratch, int rows,
                      int h, cudaStream_t st) {
  // two rows in the ring: one under way hides the memory (a third changes nothing); none where 512 threads' slots would
  // not fit an SM's shared memory (fp32 rows of more than 8192 columns)
#define LN_BWD_W(EPL, NS, MAXT) bwd_launch<T, VEC, EPL, NS, MAXT>(dy, lddy, x, ldx, mean, rstd, gain, resid, ldr, dx, lddx, dgain, dbias, scratch, rows, h, st)
  const int epl = elements_per_thread(cover_of(h, VEC), VEC * sizeof(T) == 4);
  return epl == 8 ? LN_BWD_W(8, 2, 512) : epl == 16 ? LN_BWD_W(16, 2, 512) : LN_BWD_W(32, (sizeof(T) == 2 ? 2 : 0), (VEC == 0 ? 544 : 512));
#undef LN_BWD_W
}

}  // namespace

cudaError_t layernorm_fwd(const void* x, int64_t ldx, const void* gain, const void* bias, void* y, int64_t ldy, float* mean,
                          float* rstd, int rows, int h, float eps, int dtype, cudaStream_t st) {
  const uintptr_t ptrs = (uintptr_t)x | (uintptr_t)gain | (uintptr_t)bias | (uintptr_t)y;
  const int v = row_vec((uint64_t)h | (uint64_t)ldx | (uint64_t)ldy, ptrs, dtype == 0 ? 2 : 4);
#define LN_FWD(T, V) fwd_width<T, V>(x, ldx, gain, bias, y, ldy, mean, rstd, rows, h, eps, st)
  if (dtype == 0) return v == 8 ? LN_FWD(bf16, 8) : v == 4 ? LN_FWD(bf16, 4) : v == 2 ? LN_FWD(bf16, 2) : LN_FWD(bf16, 0);
  return v == 4 ? LN_FWD(float, 4) : v == 2 ? LN_FWD(float, 2) : LN_FWD(float, 1);
#undef LN_FWD
}

size_t layernorm_scratch_bytes(int rows, int h) {
  if (rows <= 0 || h <= 0 || h > kLayerNormMaxWidth) return 0;
  return (size_t)(rows < kSms ? rows : kSms) * 2 * (size_t)((h + 3) / 4 * 4) * sizeof(float);  // one partial row of both gradients a block
}

cudaError_t layernorm_bwd(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd,
                          const void* gain, const void* resid, int64_t ldr, void* dx, int64_t lddx, float* dgain, float* dbias,
                          float* scratch, int rows, int h, int dtype, cudaStream_t st) {
  const uintptr_t ptrs = (uintptr_t)dy | (uintptr_t)x | (uintptr_t)gain | (uintptr_t)resid | (uintptr_t)dx;
  const int v = row_vec((uint64_t)h | (uint64_t)lddy | (uint64_t)ldx | (resid ? (uint64_t)ldr : 0) | (uint64_t)lddx, ptrs, dtype == 0 ? 2 : 4);
#define LN_BWD(T, V) bwd_width<T, V>(dy, lddy, x, ldx, mean, rstd, gain, resid, ldr, dx, lddx, dgain, dbias, scratch, rows, h, st)
  if (dtype == 0) return v == 8 ? LN_BWD(bf16, 8) : v == 4 ? LN_BWD(bf16, 4) : v == 2 ? LN_BWD(bf16, 2) : LN_BWD(bf16, 0);
  return v == 4 ? LN_BWD(float, 4) : v == 2 ? LN_BWD(float, 2) : LN_BWD(float, 1);
#undef LN_BWD
}

}  // namespace fs

// =============================================================================== entry points
namespace {
bool rows_ok(int32_t rows, int32_t h, int32_t dtype) {
  return rows > 0 && h > 0 && h <= fs::kLayerNormMaxWidth && (dtype == 0 || dtype == 1);
}
// the same rows, or rows that start elsewhere: an output over an input has to lie as it does
bool same_rows(const void* out, int64_t ldo, const void* in, int64_t ldi, int32_t rows) { return out != in || ldo == ldi || rows == 1; }
bool elem_aligned(const void* p, int32_t dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == 0 ? 1u : 3u)) == 0; }
bool f32_aligned(const float* p) { return elem_aligned(p, 1); }
}  // namespace

extern "C" ft_status ft_k_layernorm_fwd(const void* dev_x, int64_t ldx, const void* dev_gain, const void* dev_bias, void* dev_y,
                                        int64_t ldy, float* dev_mean, float* dev_rstd, int32_t rows, int32_t h, float eps,
                                        int32_t dtype, void* stream) {
  if (!dev_x || !dev_gain || !dev_y || !dev_mean || !dev_rstd || !rows_ok(rows, h, dtype)) return FT_EINVAL;
  if (ldx < h || ldy < h || !(eps >= 0.f) || !same_rows(dev_y, ldy, dev_x, ldx, rows)) return FT_EINVAL;
  if (!elem_aligned(dev_x, dtype) || !elem_aligned(dev_gain, dtype) || !elem_aligned(dev_bias, dtype) || !elem_aligned(dev_y, dtype) ||
      !f32_aligned(dev_mean) || !f32_aligned(dev_rstd))
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
  if (!same_rows(dev_dx, lddx, dev_dy, lddy, rows) || !same_rows(dev_dx, lddx, dev_x, ldx, rows) || !same_rows(dev_dx, lddx, dev_resid, ldr, rows))
    return FT_EINVAL;
  if (!elem_aligned(dev_dy, dtype) || !elem_aligned(dev_x, dtype) || !elem_aligned(dev_gain, dtype) ||
      !elem_aligned(dev_resid, dtype) || !elem_aligned(dev_dx, dtype) || !f32_aligned(dev_mean) || !f32_aligned(dev_rstd) ||
      !f32_aligned(dev_dgain) || !f32_aligned(dev_dbias) || (reinterpret_cast<uintptr_t>(dev_scratch) & 15u) != 0)
    return FT_EINVAL;
  if (scratch_bytes < fs::layernorm_scratch_bytes(rows, h)) return FT_ENOMEM;
  cudaError_t e = fs::layernorm_bwd(dev_dy, lddy, dev_x, ldx, dev_mean, dev_rstd, dev_gain, dev_resid, ldr, dev_dx, lddx, dev_dgain,
                                    dev_dbias, reinterpret_cast<float*>(dev_scratch), rows, h, dtype,
                                    reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}
