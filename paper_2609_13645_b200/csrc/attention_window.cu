// Causal attention over a sliding window with sink keys, forward and backward, on the 5th-generation tensor cores.
//
// Query i sees key j iff j <= i and (i - j < window or j < sinks).  The kernels have the structure of the causal ones (one
// CTA per tile of 128 rows, 64-row blocks of the other side streamed through a TMA ring, scores in TMEM, the softmax row
// reference an integer power of two so that the order of the blocks does not show in the result), with three differences:
//
//   * Which blocks are streamed is a list of two runs: the blocks that hold sink keys, then the blocks of the window.  Work
//     and traffic are linear in the sequence; only blocks on the edge of a run test single elements.
//   * A row can meet a block of which it sees nothing (the oldest block of its tile's window): its running maximum may
//     still be -inf then, and the reference, the rescaling factor and the exponentials are guarded for it.
//   * A block of sink keys is seen by every later query, so its gradient is a sum over the whole sequence while every other
//     key block's is one over window + 128 queries.  The streamed list of a key block is therefore cut into parts of about
//     equal length that run as CTAs of their own and leave fp32 partial sums; a small kernel adds them in part order (no
//     atomics: results are bit-identical from run to run).  Key blocks are also cut when a batch has fewer of them than
//     the GPU has SMs (few kv heads, short sequences).
#include "attention_window.cuh"

#include <limits.h>
#include <math.h>

#include "../../include/forgestep.h"
#include "attention.cuh"
#include "attention_tile.cuh"
#include "tmap.cuh"

namespace fs {
namespace {

constexpr int kSms = 148;

// The 64-key blocks that the 128 queries from q0 see: [0, n_sink) and then [first, first + count - n_sink).
struct KeyRuns {
  int n_sink, first, count;
  __device__ __forceinline__ KeyRuns(int q0, int S, int window, int sinks) {
    const int end = (min(S, q0 + 128) + 63) >> 6;
    first = max(0, q0 - window + 1) >> 6;
    n_sink = min((min(sinks, S) + 63) >> 6, first);
    count = n_sink + end - first;
  }
  __device__ __forceinline__ int block(int j) const { return j < n_sink ? j : first + j - n_sink; }
};

// ============================================================================ forward
enum { B_QFULL = 0, B_KFULL = 1, B_KEMPTY = 4, B_VFULL = 7, B_VEMPTY = 9, B_SFULL = 11, B_PFULL = 13, B_ODONE = 15,
       B_OFINAL = 16, B_COUNT = 17 };
constexpr int FWD_THREADS = 224;  // Q + K producer, MMA issuer, 4 softmax warps, V producer

template <int D>
struct FwdCfg {
  static constexpr int BQ = 128, BK = 64, KC = D / 64;
  static constexpr int NK = 3, NV = 2;
  static constexpr int Q_BYTES = BQ * D * 2;
  static constexpr int KV_BYTES = BK * D * 2;
  static constexpr int OFF_K = Q_BYTES;
  static constexpr int OFF_V = OFF_K + NK * KV_BYTES;
  static constexpr int OFF_BAR = OFF_V + NV * KV_BYTES;
  static constexpr int SMEM_BYTES = OFF_BAR + 160;
  static constexpr int TMEM_COLS = 256;  // S0 [0,64) S1 [64,128) (bf16 P over the first 32 columns of each), O from 128
  static constexpr int O_COL = 128;
};

template <int D>
__global__ void __launch_bounds__(FWD_THREADS, 2)
attn_window_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmKV, bf16* __restrict__ o,
                       float* __restrict__ lse, int S, int n_heads, int n_kv, int n_batch, int n_qblocks, int window, int sinks,
                       float scale_log2, int* err) {
  using C = FwdCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + B_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((sbase & 1023u) != 0u) {  // the swizzled tiles need a 1024-byte aligned base
    if (threadIdx.x == 0) atomicExch(err, (int)ERR_BAD_ALIGNMENT);
    return;
  }
  // last query blocks first: the tiles at the start of the sequence, the only ones with fewer blocks, end the launch
  const int groups = n_heads * n_batch;
  const int qb = n_qblocks - 1 - (int)blockIdx.x / groups;
  const int grp = (int)blockIdx.x % groups;
  const int n = grp % n_heads, b = grp / n_heads;
  const int kvh = n / (n_heads / n_kv);
  const int hq = n_heads * D, hkv = n_kv * D;
  const int q0 = qb * C::BQ;
  const KeyRuns runs(q0, S, window, sinks);
  const int nb = runs.count;

  if (threadIdx.x == 0) {
    mbar_init(bar(B_QFULL), 1);
    for (int i = 0; i < C::NK; ++i) {
      mbar_init(bar(B_KFULL + i), 1);
      mbar_init(bar(B_KEMPTY + i), 1);
    }
    for (int i = 0; i < C::NV; ++i) {
      mbar_init(bar(B_VFULL + i), 1);
      mbar_init(bar(B_VEMPTY + i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_PFULL + i), 4);  // two: a warp that need not rescale O may run a block ahead of a slower one
    }
    mbar_init(bar(B_ODONE), 1);
    mbar_init(bar(B_OFINAL), 1);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmKV);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_trigger();
  pdl_wait();  // set-up done; from here on the kernel touches what its predecessor wrote

  if (warp == 0) {
    if (lane == 0) {
      mbar_expect_tx(bar(B_QFULL), C::Q_BYTES);
#pragma unroll
      for (int kc = 0; kc < C::KC; ++kc)
        tma_load_3d(sbase + kc * (C::BQ * 128), &tmQ, bar(B_QFULL), n * D + kc * 64, q0, b);
      for (int j = 0; j < nb; ++j) {
        const int st = j % C::NK;
        if (!mbar_wait(bar(B_KEMPTY + st), ((uint32_t)(j / C::NK) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x61)) break;
        mbar_expect_tx(bar(B_KFULL + st), C::KV_BYTES);
#pragma unroll
        for (int kc = 0; kc < C::KC; ++kc)
          tma_load_3d(sbase + C::OFF_K + st * C::KV_BYTES + kc * (C::BK * 128), &tmKV, bar(B_KFULL + st),
                      hq + kvh * D + kc * 64, runs.block(j) * C::BK, b);
      }
    }
  } else if (warp == 6) {
    if (lane == 0) {
      for (int j = 0; j < nb; ++j) {
        const int st = j % C::NV;
        if (!mbar_wait(bar(B_VEMPTY + st), ((uint32_t)(j / C::NV) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x62)) break;
        mbar_expect_tx(bar(B_VFULL + st), C::KV_BYTES);
#pragma unroll
        for (int kc = 0; kc < C::KC; ++kc)
          tma_load_3d(sbase + C::OFF_V + st * C::KV_BYTES + kc * (C::BK * 128), &tmKV, bar(B_VFULL + st),
                      hq + hkv + kvh * D + kc * 64, runs.block(j) * C::BK, b);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc_base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(C::BQ >> 4) << 24);
      const uint32_t idesc_s = idesc_base | ((uint32_t)(C::BK >> 3) << 17);            // N = 64 keys, both K-major
      const uint32_t idesc_pv = idesc_base | (1u << 16) | ((uint32_t)(D >> 3) << 17);  // N = D, B (V) mn-major
      const uint64_t dq = umma_desc_sw128(sbase, 0, 1024);
      auto issue_s = [&](int j) -> bool {
        const int st = j % C::NK;
        if (!mbar_wait(bar(B_KFULL + st), (uint32_t)(j / C::NK) & 1u, abort_flag, err, kWaitLimitCycles, 0x63)) return false;
        tc_fence_after();
        const uint64_t dk = umma_desc_sw128(sbase + C::OFF_K + st * C::KV_BYTES, 0, 1024);
        const uint32_t d_tmem = tmem_base + (uint32_t)((j & 1) * C::BK);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t qo = (uint64_t)(((k >> 2) * (C::BQ * 128) + (k & 3) * 32) >> 4);
          const uint64_t ko = (uint64_t)(((k >> 2) * (C::BK * 128) + (k & 3) * 32) >> 4);
          umma_bf16(d_tmem, dq + qo, dk + ko, idesc_s, k > 0 ? 1u : 0u);
        }
        umma_commit(bar(B_SFULL + (j & 1)));
        umma_commit(bar(B_KEMPTY + st));
        return true;
      };
      bool ok = mbar_wait(bar(B_QFULL), 0, abort_flag, err, kWaitLimitCycles, 0x64);
      if (ok) ok = issue_s(0);
      for (int j = 0; j < nb && ok; ++j) {
        if (j + 1 < nb && !issue_s(j + 1)) { ok = false; break; }
        const int st = j % C::NV;
        if (!mbar_wait(bar(B_VFULL + st), (uint32_t)(j / C::NV) & 1u, abort_flag, err, kWaitLimitCycles, 0x65)) { ok = false; break; }
        if (!mbar_wait(bar(B_PFULL + (j & 1)), ((uint32_t)j >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x66)) { ok = false; break; }
        tc_fence_after();
        const uint64_t dv = umma_desc_sw128(sbase + C::OFF_V + st * C::KV_BYTES, C::BK * 128, 1024);
        const uint32_t tp = tmem_base + (uint32_t)((j & 1) * C::BK);  // bf16 P: 16 keys = 8 columns per K step
#pragma unroll
        for (int k = 0; k < C::BK / 16; ++k)
          umma_bf16_ts(tmem_base + C::O_COL, tp + (uint32_t)(k * 8), dv + (uint64_t)((k * 2048) >> 4), idesc_pv,
                       (j > 0 || k > 0) ? 1u : 0u);
        umma_commit(bar(B_VEMPTY + st));
        umma_commit(bar(B_ODONE));
      }
      if (ok) umma_commit(bar(B_OFINAL));
    }
  } else {
    // softmax warps (2..5): one query row per thread = TMEM lane
    const int q = warp & 3;
    const int row = q0 + q * 32 + lane;
    const uint32_t tlane = tmem_base + ((uint32_t)(q * 32) << 16);
    const int wmin = q0 + q * 32, wmax = wmin + 31;  // rows of this warp
    float mref = -INFINITY, lsum = 0.f;
    bool ok = true;
    for (int j = 0; j < nb; ++j) {
      ok = mbar_wait(bar(B_SFULL + (j & 1)), ((uint32_t)j >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x67);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      uint32_t r0[32], r1[32];
      tmem_ld32(tlane + (uint32_t)((j & 1) * C::BK), r0);
      tmem_ld32(tlane + (uint32_t)((j & 1) * C::BK + 32), r1);
      tmem_ld_wait();

      const int k0 = runs.block(j) * C::BK;
      // every row of the warp sees every key of the block: nothing to test (warp-uniform)
      const bool full = k0 + C::BK - 1 <= wmin && (wmax - k0 < window || k0 + C::BK <= sinks);
      if (!full) {
        const int hi = row - k0, lo = row - window + 1 - k0, sk = sinks - k0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          if (i > hi || (i < lo && i >= sk)) r0[i] = 0xff800000u;  // -inf
          if (i + 32 > hi || (i + 32 < lo && i + 32 >= sk)) r1[i] = 0xff800000u;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 32; ++i) mx = fmaxf(mx, fmaxf(__uint_as_float(r0[i]), __uint_as_float(r1[i])));
      // the reference is an integer that moves once the maximum has passed it by more than 2^kRefSlack; it stays -inf
      // (and 0 stands in for it below: the exponentials of -inf are 0) until the row has seen its first key
      const float mcand = ceilf(mx * scale_log2);
      const float mnew = mcand > mref + kRefSlack ? mcand : mref;
      const float alpha = mnew == mref ? 1.0f : fast_exp2(mref - mnew);
      const float ref = mnew == -INFINITY ? 0.f : mnew;
      float psum = 0.f;
      uint32_t pw[32];  // bf16 pairs: keys 2c, 2c+1 in word c
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const float a0 = fast_exp2(fmaf(__uint_as_float(r0[i]), scale_log2, -ref));
        const float a1 = fast_exp2(fmaf(__uint_as_float(r0[i + 1]), scale_log2, -ref));
        const float c0 = fast_exp2(fmaf(__uint_as_float(r1[i]), scale_log2, -ref));
        const float c1 = fast_exp2(fmaf(__uint_as_float(r1[i + 1]), scale_log2, -ref));
        psum += (a0 + a1) + (c0 + c1);
        pw[i >> 1] = pack_bf16(a0, a1);
        pw[16 + (i >> 1)] = pack_bf16(c0, c1);
      }
      lsum = lsum * alpha + psum;
      mref = mnew;

      if (j > 0 && __any_sync(0xffffffffu, alpha != 1.0f)) {
        ok = mbar_wait(bar(B_ODONE), (uint32_t)(j - 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x68);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t t[32];
          tmem_ld32(tlane + (uint32_t)(C::O_COL + c), t);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) t[i] = __float_as_uint(__uint_as_float(t[i]) * alpha);
          tmem_st32(tlane + (uint32_t)(C::O_COL + c), t);
        }
      }
      tmem_st32(tlane + (uint32_t)((j & 1) * C::BK), pw);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_PFULL + (j & 1)));
    }
    if (ok) {  // a barrier of its own: the parity of B_ODONE cannot tell the last product from the one two before
      ok = mbar_wait(bar(B_OFINAL), 0, abort_flag, err, kWaitLimitCycles, 0x69);
      ok = __all_sync(0xffffffffu, ok);
    }
    if (ok) {
      tc_fence_after();
      const float inv = 1.0f / lsum;
      bf16* orow = o + ((long long)b * S + row) * hq + n * D;
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        float t[32];
        tmem_load_cols<32>(tlane + (uint32_t)(C::O_COL + c), t);
        if (row < S) {
#pragma unroll
          for (int i = 0; i < 32; ++i) t[i] *= inv;
          store_bf16_row<32>(orow + c, t);
        }
      }
      if (row < S) lse[((long long)b * n_heads + n) * S + row] = (mref + log2f(lsum)) * kLn2;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag != 0) {
    // give copies and MMAs still in flight time to land before shared memory and TMEM are released
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, C::TMEM_COLS);
  }
}

template <int D>
cudaError_t fwd_t(const bf16* qkv, bf16* o, float* lse, int B, int S, int nh, int nkv, int window, int sinks, int* err,
                  cudaStream_t st) {
  using C = FwdCfg<D>;
  static unsigned long long smem_set = 0;
  cudaError_t e = ensure_dynamic_smem(attn_window_fwd_kernel<D>, C::SMEM_BYTES, smem_set);
  if (e != cudaSuccess) return e;
  const int nqkv = (nh + 2 * nkv) * D;
  CUtensorMap tmQ, tmKV;
  if (!make_tmap_3d(&tmQ, qkv, nqkv, S, B, nqkv, C::BQ) || !make_tmap_3d(&tmKV, qkv, nqkv, S, B, nqkv, C::BK))
    return cudaErrorInvalidValue;
  const float scale_log2 = (float)((1.0 / sqrt((double)D)) * 1.4426950408889634);
  const int nqb = (S + C::BQ - 1) / C::BQ;
  return launch_pdl(attn_window_fwd_kernel<D>, dim3((unsigned)(nqb * nh * B)), dim3(FWD_THREADS), C::SMEM_BYTES, st, tmQ, tmKV, o, lse,
                    S, nh, nkv, B, nqb, window, sinks, scale_log2, err);
}

// ============================================================================ backward
// MODE_DQ : resident X = (Q, dO) of 128 queries, streamed Y = (K, V) blocks of 64 keys  -> dQ  = dS K
// MODE_DKV: resident X = (K, V) of 128 keys, streamed Y = (Q, dO) blocks of 64 queries of every query head of the group
//                                                                                       -> dV = P^T dO, dK = dS^T Q
// Per streamed block S = X1 Y1^T and dP = X2 Y2^T go to one of two TMEM buffers; the compute warps (one X row per thread)
// turn them into P = exp2(S c - LSE) and dS = P (dP - delta), packed to bf16 over the columns they came from, and the
// accumulating products read those as their A operand and the streamed tiles again as mn-major B operands.  warp 0 = TMA
// producer, warps 1 and 10 = MMA issuers (one thread cannot issue products this small fast enough), warps 2..9 compute.
enum { MODE_DQ = 0, MODE_DKV = 1 };
enum { BB_XFULL = 0, BB_YFULL = 1, BB_YEMPTY = 5, BB_SDPFULL = 9, BB_TFULL = 11, BB_ACCDONE = 13, BB_COUNT = 14 };
constexpr int BWD_THREADS = 352;

template <int D>
struct BwdCfg {
  static constexpr int KC = D / 64;
  static constexpr int X_BYTES = 128 * D * 2;
  static constexpr int Y_BYTES = 64 * D * 2;
  static constexpr int NST = 4;
  static constexpr int OFF_X1 = 0, OFF_X2 = X_BYTES, OFF_Y = 2 * X_BYTES;
  static constexpr int OFF_STAT = OFF_Y + NST * 2 * Y_BYTES;
  static constexpr int OFF_BAR = OFF_STAT + 2048;
  static constexpr int SMEM_BYTES = OFF_BAR + 256;
  static constexpr int TMEM_COLS = 512;  // buffer b: S at b*128, dP at b*128+64; accumulators from column 256
  static constexpr int ACC0 = 256, ACC1 = 256 + D;
};

// How the key blocks' streamed lists are cut (host and device agree on it through this).
struct Split {
  int chunk;              // streamed blocks a part has, at most
  int n_sink;             // 128-key blocks that hold sink keys
  int parts_sink, parts;  // parts of a sink block and of any other, at most
  // queries [x0, end) see a key of block x; streamed 64-query blocks, over all query heads of the group
  static __host__ __device__ int queries_end(int x, int S, int window, int sinks) {
    const int x0 = x * 128;
    return x0 < sinks || S - x0 < 127 + window ? S : x0 + 127 + window;
  }
  static __host__ __device__ int per_head(int x, int S, int window, int sinks) {
    return (queries_end(x, S, window, sinks) + 63) / 64 - x * 2;
  }
  __host__ __device__ int parts_of(int x, int S, int window, int sinks, int n_rep) const {
    return (int)(((long long)per_head(x, S, window, sinks) * n_rep + chunk - 1) / chunk);
  }
};

template <int D, int MODE>
__global__ void __launch_bounds__(BWD_THREADS, 1)
attn_window_bwd_kernel(const __grid_constant__ CUtensorMap tm_qkv128, const __grid_constant__ CUtensorMap tm_qkv64,
                       const __grid_constant__ CUtensorMap tm_do128, const __grid_constant__ CUtensorMap tm_do64,
                       const float* __restrict__ lse, const float* __restrict__ delta, bf16* __restrict__ dqkv,
                       float* __restrict__ partial, const float* __restrict__ rope_cos, const float* __restrict__ rope_sin, int S,
                       int n_heads, int n_kv, int n_batch, int n_xblocks, int window, int sinks, const Split split, float scale,
                       float scale_log2, int* err) {
  using C = BwdCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + BB_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* s_stat = reinterpret_cast<float*>(smem + C::OFF_STAT);  // [stage][0: lse*log2e, 1: delta][64]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((sbase & 1023u) != 0u) {
    if (threadIdx.x == 0) atomicExch(err, (int)ERR_BAD_ALIGNMENT);
    return;
  }
  const int n_rep = n_heads / n_kv;
  const int hq = n_heads * D, hkv = n_kv * D;
  const long long ld = hq + 2 * hkv;
  const int heads_here = MODE == MODE_DQ ? n_heads : n_kv;
  const int groups = heads_here * n_batch;
  const int rank = (int)blockIdx.x / groups, grp = (int)blockIdx.x % groups;
  const int b = grp / heads_here;
  int x0, kvh, n_q = 0, qb0 = 0, per_head = 1, first_it = 0, iters;
  bool direct = true;  // this CTA holds the whole sum of its rows
  KeyRuns runs(0, 1, 1, 0);
  if constexpr (MODE == MODE_DQ) {
    x0 = (n_xblocks - 1 - rank) * 128;  // the first query blocks, with fewer keys, end the launch
    n_q = grp % heads_here;
    kvh = n_q / n_rep;
    runs = KeyRuns(x0, S, window, sinks);
    iters = runs.count;
  } else {
    const int n_sink_ctas = split.n_sink * split.parts_sink;
    const int x = rank < n_sink_ctas ? rank / split.parts_sink : split.n_sink + (rank - n_sink_ctas) / split.parts;
    const int part = rank < n_sink_ctas ? rank % split.parts_sink : (rank - n_sink_ctas) % split.parts;
    x0 = x * 128;
    kvh = grp % heads_here;
    qb0 = x * 2;
    per_head = Split::per_head(x, S, window, sinks);
    const int total = per_head * n_rep, np = split.parts_of(x, S, window, sinks, n_rep);
    if (part >= np) return;
    first_it = (int)((long long)total * part / np);
    iters = (int)((long long)total * (part + 1) / np) - first_it;
    direct = np == 1;
  }

  if (threadIdx.x == 0) {
    mbar_init(bar(BB_XFULL), 1);
    for (int i = 0; i < C::NST; ++i) {
      mbar_init(bar(BB_YFULL + i), MODE == MODE_DKV ? 2 : 1);
      mbar_init(bar(BB_YEMPTY + i), 2);   // one commit from each MMA-issuing warp
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(BB_SDPFULL + i), 2);
      mbar_init(bar(BB_TFULL + i), 8);
    }
    mbar_init(bar(BB_ACCDONE), 2);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_qkv128);
    tma_prefetch_desc(&tm_qkv64);
    tma_prefetch_desc(&tm_do128);
    tma_prefetch_desc(&tm_do64);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_trigger();
  pdl_wait();  // set-up done; from here on the kernel touches what its predecessor wrote

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      mbar_expect_tx(bar(BB_XFULL), 2 * C::X_BYTES);
#pragma unroll
      for (int kc = 0; kc < C::KC; ++kc) {
        if constexpr (MODE == MODE_DQ) {
          tma_load_3d(sbase + C::OFF_X1 + kc * 16384, &tm_qkv128, bar(BB_XFULL), n_q * D + kc * 64, x0, b);
          tma_load_3d(sbase + C::OFF_X2 + kc * 16384, &tm_do128, bar(BB_XFULL), n_q * D + kc * 64, x0, b);
        } else {
          tma_load_3d(sbase + C::OFF_X1 + kc * 16384, &tm_qkv128, bar(BB_XFULL), hq + kvh * D + kc * 64, x0, b);
          tma_load_3d(sbase + C::OFF_X2 + kc * 16384, &tm_qkv128, bar(BB_XFULL), hq + hkv + kvh * D + kc * 64, x0, b);
        }
      }
    }
    for (int it = 0; it < iters; ++it) {
      const int st = it % C::NST;
      bool ok = mbar_wait(bar(BB_YEMPTY + st), (((uint32_t)(it / C::NST)) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x71);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const uint32_t ydst = sbase + C::OFF_Y + st * 2 * C::Y_BYTES;
      if constexpr (MODE == MODE_DQ) {
        if (lane == 0) {
          const int y0 = runs.block(it) * 64;
          mbar_expect_tx(bar(BB_YFULL + st), 2 * C::Y_BYTES);
#pragma unroll
          for (int kc = 0; kc < C::KC; ++kc) {
            tma_load_3d(ydst + kc * 8192, &tm_qkv64, bar(BB_YFULL + st), hq + kvh * D + kc * 64, y0, b);
            tma_load_3d(ydst + C::Y_BYTES + kc * 8192, &tm_qkv64, bar(BB_YFULL + st), hq + hkv + kvh * D + kc * 64, y0, b);
          }
        }
      } else {
        const int rep = (first_it + it) / per_head, qb = qb0 + (first_it + it) % per_head;
        const int n = kvh * n_rep + rep;
        if (lane == 0) {
          mbar_expect_tx(bar(BB_YFULL + st), 2 * C::Y_BYTES);
#pragma unroll
          for (int kc = 0; kc < C::KC; ++kc) {
            tma_load_3d(ydst + kc * 8192, &tm_qkv64, bar(BB_YFULL + st), n * D + kc * 64, qb * 64, b);
            tma_load_3d(ydst + C::Y_BYTES + kc * 8192, &tm_do64, bar(BB_YFULL + st), n * D + kc * 64, qb * 64, b);
          }
        }
        const long long stat = ((long long)b * n_heads + n) * S;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int qq = qb * 64 + lane * 2 + e;
          s_stat[st * 128 + lane * 2 + e] = qq < S ? lse[stat + qq] * kLog2e : 0.f;
          s_stat[st * 128 + 64 + lane * 2 + e] = qq < S ? delta[stat + qq] : 0.f;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(BB_YFULL + st));
      }
    }
  } else if (warp == 1 || warp == 10) {
    // ------------------------------------------------------------------ MMA issuers
    // side 0 owns S (and dV, which reads P^T from the S columns), side 1 owns dP (and dK / dQ, which read dS from the dP
    // columns): each chain stays in issue order
    if (lane == 0) {
      const int side = warp == 1 ? 0 : 1;
      const uint32_t idesc_base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);
      const uint32_t idesc_sdp = idesc_base | ((uint32_t)(64 >> 3) << 17);            // N = 64, both K-major
      const uint32_t idesc_acc = idesc_base | (1u << 16) | ((uint32_t)(D >> 3) << 17);  // N = D, B mn-major
      const uint64_t dx = umma_desc_sw128(sbase + (side == 0 ? C::OFF_X1 : C::OFF_X2), 0, 1024);
      auto issue_sdp = [&](int it) {
        const int st = it % C::NST;
        const uint32_t y = sbase + C::OFF_Y + st * 2 * C::Y_BYTES + side * C::Y_BYTES;
        const uint64_t dy = umma_desc_sw128(y, 0, 1024);
        const uint32_t d_t = tmem_base + (uint32_t)((it & 1) * 128 + side * 64);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t xo = (uint64_t)(((k >> 2) * 16384 + (k & 3) * 32) >> 4);
          const uint64_t yo = (uint64_t)(((k >> 2) * 8192 + (k & 3) * 32) >> 4);
          umma_bf16(d_t, dx + xo, dy + yo, idesc_sdp, k > 0 ? 1u : 0u);
        }
        umma_commit(bar(BB_SDPFULL + (it & 1)));
      };
      bool ok = mbar_wait(bar(BB_XFULL), 0, abort_flag, err, kWaitLimitCycles, 0x72) &&
                mbar_wait(bar(BB_YFULL), 0, abort_flag, err, kWaitLimitCycles, 0x73);
      if (ok) {
        tc_fence_after();
        issue_sdp(0);
      }
      for (int it = 0; it < iters && ok; ++it) {
        if (it + 1 < iters) {
          const int y1s = (it + 1) % C::NST;
          if (!mbar_wait(bar(BB_YFULL + y1s), ((uint32_t)((it + 1) / C::NST)) & 1u, abort_flag, err, kWaitLimitCycles, 0x74)) { ok = false; break; }
          // the TMEM columns this writes were last read by this same thread's accumulating MMAs of block it-1: in order
          tc_fence_after();
          issue_sdp(it + 1);
        }
        const int bf = it & 1;
        if (!mbar_wait(bar(BB_TFULL + bf), ((uint32_t)it >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x75)) { ok = false; break; }
        tc_fence_after();
        const int yst = it % C::NST;
        const uint32_t y1 = sbase + C::OFF_Y + yst * 2 * C::Y_BYTES, y2 = y1 + C::Y_BYTES;
        // A operands (bf16) sit in TMEM where S / dP were: 16 streamed rows (K = 16) = 8 columns; the two compute warps of
        // a lane quarter each wrote their 32 at the start of their own 32 fp32 columns
        const uint32_t ta = tmem_base + (uint32_t)(bf * 128 + side * 64);
        const uint32_t first = it > 0 ? 1u : 0u;
        if (MODE == MODE_DKV || side == 1) {
          const uint64_t by = umma_desc_sw128((MODE == MODE_DKV && side == 0) ? y2 : y1, 8192, 1024);
          const uint32_t dacc = tmem_base + (uint32_t)((MODE == MODE_DKV && side == 1) ? C::ACC1 : C::ACC0);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t acol = (uint32_t)((k >> 1) * 32 + (k & 1) * 8);
            umma_bf16_ts(dacc, ta + acol, by + (uint64_t)((k * 2048) >> 4), idesc_acc, k > 0 ? 1u : first);
          }
        }
        umma_commit(bar(BB_YEMPTY + yst));
      }
      if (ok) umma_commit(bar(BB_ACCDONE));
    }
  } else {
    // ------------------------------------------------------------------ compute warps
    const int q = warp & 3, ch = (warp - 2) >> 2;
    const int rloc = q * 32 + lane;
    const int row = x0 + rloc;  // query (MODE_DQ) or key (MODE_DKV) position
    const uint32_t tlane = tmem_base + ((uint32_t)(q * 32) << 16);
    const int rmin = x0 + q * 32, rmax = rmin + 31;
    float lse2_row = 0.f, delta_row = 0.f;
    if constexpr (MODE == MODE_DQ) {
      if (row < S) {
        const long long stat = ((long long)b * n_heads + n_q) * S;
        lse2_row = lse[stat + row] * kLog2e;
        delta_row = delta[stat + row];
      }
    }
    // MODE_DKV: the queries that see key `row` are [row, row_end)
    const int row_end = row < sinks || S - row < window ? S : row + window;
    bool ok = true;
    for (int it = 0; it < iters; ++it) {
      const int bf = it & 1;
      ok = mbar_wait(bar(BB_SDPFULL + bf), ((uint32_t)it >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x76);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      uint32_t rs[32], rp[32];
      tmem_ld32(tlane + (uint32_t)(bf * 128 + ch * 32), rs);
      tmem_ld32(tlane + (uint32_t)(bf * 128 + 64 + ch * 32), rp);
      tmem_ld_wait();

      // single elements are only tested where the warp's tile touches an edge of the mask (warp-uniform)
      if constexpr (MODE == MODE_DQ) {
        const int cmin = runs.block(it) * 64 + ch * 32;
        const bool full = cmin + 31 <= rmin && (rmax - cmin < window || cmin + 32 <= sinks);
        const float nl = -lse2_row;
        const int hi = row - cmin, lo = row - window + 1 - cmin, sk = sinks - cmin;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float p = fast_exp2(fmaf(__uint_as_float(rs[i]), scale_log2, nl));
          if (!full && (i > hi || (i < lo && i >= sk))) p = 0.f;
          rs[i] = __float_as_uint(p);
          rp[i] = __float_as_uint(p * (__uint_as_float(rp[i]) - delta_row));
        }
      } else {
        const int yst = it % C::NST;
        const float* st_lse = s_stat + yst * 128 + ch * 32;
        const float* st_dl = st_lse + 64;
        const int cmin = (qb0 + (first_it + it) % per_head) * 64 + ch * 32;
        ok = mbar_wait(bar(BB_YFULL + yst), ((uint32_t)(it / C::NST)) & 1u, abort_flag, err, kWaitLimitCycles, 0x77);  // acquire the staged statistics
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const bool full = cmin >= rmax && cmin + 32 <= S && (rmax < sinks || cmin + 31 - rmin < window);
        if (full) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 l4 = *reinterpret_cast<const float4*>(st_lse + i);
            const float4 d4 = *reinterpret_cast<const float4*>(st_dl + i);
            const float ll[4] = {l4.x, l4.y, l4.z, l4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const float p = fast_exp2(fmaf(__uint_as_float(rs[i + u]), scale_log2, -ll[u]));
              rs[i + u] = __float_as_uint(p);
              rp[i + u] = __float_as_uint(p * (__uint_as_float(rp[i + u]) - dd[u]));
            }
          }
        } else {
          const int lo = row - cmin, hi = row_end - cmin;
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 l4 = *reinterpret_cast<const float4*>(st_lse + i);
            const float4 d4 = *reinterpret_cast<const float4*>(st_dl + i);
            const float ll[4] = {l4.x, l4.y, l4.z, l4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              float p = fast_exp2(fmaf(__uint_as_float(rs[i + u]), scale_log2, -ll[u]));
              if (i + u < lo || i + u >= hi) p = 0.f;
              rs[i + u] = __float_as_uint(p);
              rp[i + u] = __float_as_uint(p * (__uint_as_float(rp[i + u]) - dd[u]));
            }
          }
        }
      }
      // bf16 pairs back into TMEM, over this warp's own (already loaded) fp32 columns
      uint32_t wp[16], wd[16];
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        wp[c] = pack_bf16(__uint_as_float(rs[2 * c]), __uint_as_float(rs[2 * c + 1]));
        wd[c] = pack_bf16(__uint_as_float(rp[2 * c]), __uint_as_float(rp[2 * c + 1]));
      }
      if constexpr (MODE == MODE_DKV) tmem_st16(tlane + (uint32_t)(bf * 128 + ch * 32), wp);
      tmem_st16(tlane + (uint32_t)(bf * 128 + 64 + ch * 32), wd);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BB_TFULL + bf));
    }
    if (ok) {
      ok = mbar_wait(bar(BB_ACCDONE), 0, abort_flag, err, kWaitLimitCycles, 0x78);
      ok = __all_sync(0xffffffffu, ok);
    }
    if (ok) {
      tc_fence_after();
      constexpr int W = D / 4, H = D / 2;
      const int i0 = ch * W;
      const uint32_t racc = tlane + (uint32_t)(MODE == MODE_DQ ? C::ACC0 : C::ACC1);
      if (direct) {
        // rotated output (dQ or dK): this warp owns columns [i0, i0+W) and their partners D/2 further
        float lo[W], hi[W];
        tmem_load_cols<W>(racc + (uint32_t)i0, lo);
        tmem_load_cols<W>(racc + (uint32_t)(H + i0), hi);
#pragma unroll
        for (int i = 0; i < W; ++i) { lo[i] *= scale; hi[i] *= scale; }
        if (rope_cos != nullptr) {
          const int pos = min(row, S - 1);
          const float* cs = rope_cos + (long long)pos * H + i0;
          const float* sn = rope_sin + (long long)pos * H + i0;
#pragma unroll
          for (int i = 0; i < W; i += 4) {
            const float4 c4 = *reinterpret_cast<const float4*>(cs + i);
            const float4 s4 = *reinterpret_cast<const float4*>(sn + i);
            const float cc[4] = {c4.x, c4.y, c4.z, c4.w}, ss[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const float y1 = lo[i + u], y2 = hi[i + u];
              lo[i + u] = y1 * cc[u] + y2 * ss[u];
              hi[i + u] = y2 * cc[u] - y1 * ss[u];
            }
          }
        }
        const int colbase = MODE == MODE_DQ ? n_q * D : hq + kvh * D;
        if (row < S) {
          bf16* dst = dqkv + ((long long)b * S + row) * ld + colbase;
          store_bf16_row<W>(dst + i0, lo);
          store_bf16_row<W>(dst + H + i0, hi);
        }
        if constexpr (MODE == MODE_DKV) {
          bf16* dstv = dqkv + ((long long)b * S + row) * ld + hq + hkv + kvh * D;
#pragma unroll 1
          for (int c = ch * H; c < (ch + 1) * H; c += 32) {
            float v[32];
            tmem_load_cols<32>(tlane + (uint32_t)(C::ACC0 + c), v);
            if (row < S) store_bf16_row<32>(dstv + c, v);
          }
        }
      } else if constexpr (MODE == MODE_DKV) {
        // partial sums [part][dK columns, dV columns][128 keys]: a warp writes 32 consecutive keys of a column
        float* dst = partial + (long long)blockIdx.x * (2 * D * 128) + rloc;
#pragma unroll 1
        for (int c = ch * H; c < (ch + 1) * H; c += 32) {
          float v[32];
          tmem_load_cols<32>(racc + (uint32_t)c, v);
#pragma unroll
          for (int i = 0; i < 32; ++i) dst[(c + i) * 128] = v[i];
          tmem_load_cols<32>(tlane + (uint32_t)(C::ACC0 + c), v);
#pragma unroll
          for (int i = 0; i < 32; ++i) dst[(D + c + i) * 128] = v[i];
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag != 0) {
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, C::TMEM_COLS);
  }
}

// Adds the partial sums of a key block's parts in part order, scales and rotates dK, rounds once.  One thread per key; block
// (cut key block, 8 columns of dK with their partners D / 2 further, or 8 of dV).
template <int D>
__global__ void __launch_bounds__(128)
attn_window_join_kernel(const float* __restrict__ partial, bf16* __restrict__ dqkv, const float* __restrict__ rope_cos,
                        const float* __restrict__ rope_sin, int S, int n_heads, int n_kv, int groups, int window, int sinks,
                        const Split split, float scale) {
  pdl_trigger();
  pdl_wait();
  const int x = (int)blockIdx.x / groups, grp = (int)blockIdx.x % groups;
  const int np = split.parts_of(x, S, window, sinks, n_heads / n_kv);
  if (np == 1) return;
  const int rank0 = x < split.n_sink ? x * split.parts_sink : split.n_sink * split.parts_sink + (x - split.n_sink) * split.parts;
  const int row = x * 128 + threadIdx.x;
  const int kvh = grp % n_kv, b = grp / n_kv;
  const long long part_stride = (long long)groups * (2 * D * 128);
  const float* src = partial + ((long long)rank0 * groups + grp) * (2 * D * 128) + threadIdx.x;
  constexpr int H = D / 2;
  const bool is_k = (int)blockIdx.y < H / 8;
  const int c0 = is_k ? (int)blockIdx.y * 8 : ((int)blockIdx.y - H / 8) * 8;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) lo[i] = hi[i] = 0.f;
  for (int p = 0; p < np; ++p) {
    const float* s = src + p * part_stride;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] += s[(is_k ? c0 + i : D + c0 + i) * 128];
      if (is_k) hi[i] += s[(H + c0 + i) * 128];
    }
  }
  if (row >= S) return;
  bf16* dst = dqkv + ((long long)b * S + row) * (long long)((n_heads + 2 * n_kv) * D) + (n_heads + (is_k ? 0 : n_kv) + kvh) * D + c0;
  if (is_k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y1 = lo[i] * scale, y2 = hi[i] * scale;
      const float cc = rope_cos != nullptr ? rope_cos[(long long)row * H + c0 + i] : 1.f;
      const float ss = rope_cos != nullptr ? rope_sin[(long long)row * H + c0 + i] : 0.f;
      lo[i] = y1 * cc + y2 * ss;
      hi[i] = y2 * cc - y1 * ss;
    }
    store_bf16_row<8>(dst + H, hi);
  }
  store_bf16_row<8>(dst, lo);
}

// Parts of a key block's list.  Where the launch has several times more streamed blocks than SMs, a part is as long as a
// window block's whole list (or an eighth of an SM's share, if that is longer), so that only sink blocks are cut.  Smaller
// launches are cut into one part per SM, of at least 8 blocks: the set-up and the partial sums of a part cost about as
// much as 4.
Split make_split(int B, int S, int nh, int nkv, int window, int sinks) {
  const long long n_rep = nh / nkv, groups = (long long)nkv * B;
  const int nxb = (S + 127) / 128;
  Split s;
  s.n_sink = (int)(((long long)sinks + 127) / 128);
  const long long sink_len = s.n_sink > 0 ? n_rep * Split::per_head(0, S, window, sinks) : 0;
  const long long window_len = s.n_sink < nxb ? n_rep * Split::per_head(s.n_sink, S, window, 0) : 0;
  long long total = window_len * (nxb - s.n_sink) * groups;
  for (int x = 0; x < s.n_sink; ++x) total += n_rep * Split::per_head(x, S, window, sinks) * groups;
  const long long per_sm = (total + kSms - 1) / kSms;
  const long long longest = window_len > 0 ? window_len : sink_len;
  long long chunk = per_sm < longest ? per_sm : longest;
  if (chunk < 8) chunk = 8;
  if (per_sm >= longest && chunk < (per_sm + 7) / 8) chunk = (per_sm + 7) / 8;
  if (chunk > INT_MAX) chunk = INT_MAX;
  s.chunk = (int)chunk;
  s.parts = window_len > chunk ? (int)((window_len + chunk - 1) / chunk) : 1;
  s.parts_sink = sink_len > chunk ? (int)((sink_len + chunk - 1) / chunk) : 1;
  return s;
}

struct Scratch {
  size_t delta, partial, total;  // byte offsets and size
};

Scratch scratch_layout(int B, int S, int nh, int nkv, int d, const Split& s) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  const int nxb = (S + 127) / 128;
  size_t slots = 0;
  if (s.parts > 1) slots = (size_t)s.n_sink * s.parts_sink + (size_t)(nxb - s.n_sink) * s.parts;
  else if (s.parts_sink > 1) slots = (size_t)s.n_sink * s.parts_sink;
  Scratch l;
  l.delta = 0;
  l.partial = up((size_t)B * nh * S * sizeof(float));
  l.total = l.partial + slots * B * nkv * (2 * d * 128) * sizeof(float);
  return l;
}

template <int D>
cudaError_t bwd_t(const bf16* qkv, const bf16* o, const bf16* d_o, const float* lse, bf16* dqkv, const float* cs, const float* sn,
                  uint8_t* scratch, int B, int S, int nh, int nkv, int window, int sinks, int* err, cudaStream_t st) {
  using C = BwdCfg<D>;
  static unsigned long long smem_set_q = 0, smem_set_k = 0;
  cudaError_t e = ensure_dynamic_smem(attn_window_bwd_kernel<D, MODE_DQ>, C::SMEM_BYTES, smem_set_q);
  if (e != cudaSuccess) return e;
  e = ensure_dynamic_smem(attn_window_bwd_kernel<D, MODE_DKV>, C::SMEM_BYTES, smem_set_k);
  if (e != cudaSuccess) return e;
  const Split split = make_split(B, S, nh, nkv, window, sinks);
  const Scratch l = scratch_layout(B, S, nh, nkv, D, split);
  float* delta = reinterpret_cast<float*>(scratch + l.delta);
  float* partial = reinterpret_cast<float*>(scratch + l.partial);
  const int hq = nh * D, nqkv = (nh + 2 * nkv) * D;
  CUtensorMap tq128, tq64, td128, td64;
  if (!make_tmap_3d(&tq128, qkv, nqkv, S, B, nqkv, 128) || !make_tmap_3d(&tq64, qkv, nqkv, S, B, nqkv, 64) ||
      !make_tmap_3d(&td128, d_o, hq, S, B, hq, 128) || !make_tmap_3d(&td64, d_o, hq, S, B, hq, 64))
    return cudaErrorInvalidValue;
  const float scale = (float)(1.0 / sqrt((double)D));
  const float scale_log2 = (float)((1.0 / sqrt((double)D)) * 1.4426950408889634);
  e = attention_delta(o, d_o, delta, B, S, nh, D, st);
  if (e != cudaSuccess) return e;
  const int nxb = (S + 127) / 128;
  const unsigned ranks = (unsigned)(split.n_sink * split.parts_sink + (nxb - split.n_sink) * split.parts);
  e = launch_pdl(attn_window_bwd_kernel<D, MODE_DKV>, dim3(ranks * nkv * B), dim3(BWD_THREADS), C::SMEM_BYTES, st, tq128, tq64, td128,
                 td64, lse, delta, dqkv, partial, cs, sn, S, nh, nkv, B, nxb, window, sinks, split, scale, scale_log2, err);
  if (e != cudaSuccess) return e;
  e = launch_pdl(attn_window_bwd_kernel<D, MODE_DQ>, dim3((unsigned)(nxb * nh * B)), dim3(BWD_THREADS), C::SMEM_BYTES, st, tq128, tq64,
                 td128, td64, lse, delta, dqkv, partial, cs, sn, S, nh, nkv, B, nxb, window, sinks, split, scale, scale_log2, err);
  if (e != cudaSuccess) return e;
  const int cut = split.parts > 1 ? nxb : split.parts_sink > 1 ? split.n_sink : 0;
  if (cut == 0) return cudaSuccess;
  return launch_pdl(attn_window_join_kernel<D>, dim3((unsigned)(cut * nkv * B), 3 * D / 16), dim3(128), 0, st, partial, dqkv, cs, sn, S,
                    nh, nkv, nkv * B, window, sinks, split, scale);
}

// Shapes the kernels take: 32-bit grids and tensor-map extents, element counts of one row within 31 bits.
bool shape_ok(int B, int S, int nh, int nkv, int d, int window, int sinks) {
  if (B <= 0 || S <= 0 || nh <= 0 || nkv <= 0 || nh % nkv != 0 || (d != 64 && d != 128) || window < 1 || sinks < 0) return false;
  if (S > (1 << 28) || nh > (1 << 20)) return false;
  const long long tiles = ((long long)S + 127) / 128;
  return (double)tiles * nh * B < (double)INT_MAX / 64 && (long long)(nh + 2 * nkv) * d <= INT_MAX / 4;
}

// A window or a sink count beyond the sequence is one that covers it.
void clamp_mask(int S, int& window, int& sinks) {
  if (window > S) window = S;
  if (sinks > S) sinks = S;
  if (window == S) sinks = 0;  // plain causal attention
}

}  // namespace

cudaError_t attention_window_fwd(const bf16* qkv, bf16* o, float* lse, int B, int S, int nh, int nkv, int d, int window, int sinks,
                                 int* err, cudaStream_t st) {
  if (!shape_ok(B, S, nh, nkv, d, window, sinks) || !err) return cudaErrorInvalidValue;
  clamp_mask(S, window, sinks);
  if (d == 64) return fwd_t<64>(qkv, o, lse, B, S, nh, nkv, window, sinks, err, st);
  return fwd_t<128>(qkv, o, lse, B, S, nh, nkv, window, sinks, err, st);
}

size_t attention_window_scratch_bytes(int B, int S, int nh, int nkv, int d, int window, int sinks) {
  if (!shape_ok(B, S, nh, nkv, d, window, sinks)) return 0;
  clamp_mask(S, window, sinks);
  return scratch_layout(B, S, nh, nkv, d, make_split(B, S, nh, nkv, window, sinks)).total;
}

cudaError_t attention_window_bwd(const bf16* qkv, const bf16* o, const bf16* d_o, const float* lse, bf16* dqkv, const float* cs,
                                 const float* sn, void* scratch, int B, int S, int nh, int nkv, int d, int window, int sinks, int* err,
                                 cudaStream_t st) {
  if (!shape_ok(B, S, nh, nkv, d, window, sinks) || !err || (cs == nullptr) != (sn == nullptr)) return cudaErrorInvalidValue;
  clamp_mask(S, window, sinks);
  uint8_t* s = reinterpret_cast<uint8_t*>(scratch);
  if (d == 64) return bwd_t<64>(qkv, o, d_o, lse, dqkv, cs, sn, s, B, S, nh, nkv, window, sinks, err, st);
  return bwd_t<128>(qkv, o, d_o, lse, dqkv, cs, sn, s, B, S, nh, nkv, window, sinks, err, st);
}

}  // namespace fs

// =============================================================================== entry points
namespace {
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
ft_status status_of(cudaError_t e) { return e == cudaSuccess ? FT_OK : e == cudaErrorInvalidValue ? FT_EINVAL : FT_ECUDA; }
}  // namespace

extern "C" ft_status ft_k_attention_window_fwd(const void* dev_qkv, void* dev_o, float* dev_lse, int32_t B, int32_t S, int32_t n_heads,
                                               int32_t n_kv_heads, int32_t head_dim, int32_t window, int32_t n_sinks, void* stream) {
  if (!dev_qkv || !dev_o || !dev_lse || !aligned16(dev_qkv) || !aligned16(dev_o)) return FT_EINVAL;
  int* status = fs::attention_status_word();
  if (!status) return FT_ECUDA;
  return status_of(fs::attention_window_fwd(reinterpret_cast<const fs::bf16*>(dev_qkv), reinterpret_cast<fs::bf16*>(dev_o), dev_lse, B,
                                            S, n_heads, n_kv_heads, head_dim, window, n_sinks, status,
                                            reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" size_t ft_k_attention_window_scratch_bytes(int32_t B, int32_t S, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                                      int32_t window, int32_t n_sinks) {
  return fs::attention_window_scratch_bytes(B, S, n_heads, n_kv_heads, head_dim, window, n_sinks);
}

extern "C" ft_status ft_k_attention_window_bwd(const void* dev_qkv, const void* dev_o, const void* dev_do, const float* dev_lse,
                                               void* dev_dqkv, const float* dev_cos, const float* dev_sin, void* dev_scratch,
                                               uint64_t scratch_bytes, int32_t B, int32_t S, int32_t n_heads, int32_t n_kv_heads,
                                               int32_t head_dim, int32_t window, int32_t n_sinks, void* stream) {
  if (!dev_qkv || !dev_o || !dev_do || !dev_lse || !dev_dqkv || !dev_scratch) return FT_EINVAL;
  if (!aligned16(dev_qkv) || !aligned16(dev_o) || !aligned16(dev_do) || !aligned16(dev_dqkv) || !aligned16(dev_cos) ||
      !aligned16(dev_sin) || (reinterpret_cast<uintptr_t>(dev_scratch) & 255u) != 0)
    return FT_EINVAL;
  const size_t need = fs::attention_window_scratch_bytes(B, S, n_heads, n_kv_heads, head_dim, window, n_sinks);
  if (need == 0) return FT_EINVAL;
  if (scratch_bytes < need) return FT_ENOMEM;
  int* status = fs::attention_status_word();
  if (!status) return FT_ECUDA;
  return status_of(fs::attention_window_bwd(
      reinterpret_cast<const fs::bf16*>(dev_qkv), reinterpret_cast<const fs::bf16*>(dev_o), reinterpret_cast<const fs::bf16*>(dev_do),
      dev_lse, reinterpret_cast<fs::bf16*>(dev_dqkv), dev_cos, dev_sin, dev_scratch, B, S, n_heads, n_kv_heads, head_dim, window,
      n_sinks, status, reinterpret_cast<cudaStream_t>(stream)));
}
