// Causal attention over a sliding window with sink keys, forward and backward, on the 5th-generation tensor cores.
//
// Query i sees key j iff j <= i and (i - j < window or j < sinks).  The kernels have the structure of the causal ones (one
// CTA per tile of 128 rows, 64-row blocks of the other side streamed through a TMA ring, scores in TMEM, the softmax row
// reference an integer power of two so that the order of the blocks does not show in the result), with three differences:
//
//   * Which blocks are streamed is a list of two runs: the blocks that hold sink keys, then the blocks of the window.  Work
//     and traffic are linear in the sequence; only blocks on the edge of a run test single elements.
//   * A row can meet a block of which it sees nothing (the oldest block of its tile's window) before any other: maxima of
//     -inf and empty sums are part of the softmax loop.
//   * A block of sink keys is seen by every later query, so its gradient is a sum over the whole sequence while every other
//     key block's is one over window + 128 queries.  The streamed list of a key block is therefore cut into parts of about
//     equal length that run as CTAs of their own and leave fp32 partial sums, which are added in part order (no atomics:
//     results are bit-identical from run to run).  Key blocks are also cut when a batch has fewer of them than
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
// One CTA per (128 queries, head, batch row), two an SM; K and V blocks of 64 keys are streamed, S_{j+1} = Q K_{j+1}^T is
// issued ahead of O += P_j V_j, four softmax warps hold a query row a thread.  Bound by that chain and by power: the tensor
// pipe is 46 % busy, the exponential unit 45, instruction issue 45.  S 16384, 16 / 8 heads of 128, window 1024, 4 sinks: 158 us
// (845 TFLOP/s of visible pairs), 185 sustained, where the clock drops by a sixth; B 4, S 2048, window 512: 58; B 8, S 1024, 12
// heads of 64, window 256: 24.  128-key blocks, two query tiles a CTA, 8 or 16 softmax warps and persistent CTAs were all
// slower (188 to 220 us).
// P is rounded to bf16 on its way to the tensor cores, which multiply it with the bf16 V; sums, references and the log-sum-exp are
// fp32.  Against fp32 weights this takes the error of o from 1.6e-3 (its own rounding) to 2.2e-3 in the 2-norm, as in the
// dense kernel; wider operands would halve the product's rate and double P's share of TMEM.
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

// Bit e: key e of 32 is seen, given that keys e <= hi are causal, e >= lo in the window and e < sk sinks.
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t visible(int hi, int lo, int sk) { return below(hi + 1) & (~below(lo) | below(sk)); }

// The exponentials of 32 scores against the row's reference: their bf16 pairs, their sum and the scores' maximum.
__device__ __forceinline__ void softmax_chunk(const uint32_t (&r)[32], float scale_log2, float mref, uint32_t* pw, float2& psum, float& mx) {
#pragma unroll
  for (int e = 0; e < 32; e += 2) {
    const float s0 = __uint_as_float(r[e]), s1 = __uint_as_float(r[e + 1]);
    mx = fmaxf(mx, fmaxf(s0, s1));
    const float2 x = fma2(make_float2(s0, s1), both(scale_log2), both(-mref));
    const float2 a = make_float2(fast_exp2(x.x), fast_exp2(x.y));
    psum = add2(psum, a);
    pw[e >> 1] = pack_bf16(a.x, a.y);
  }
}

template <int D>
__global__ void __launch_bounds__(FWD_THREADS, 2)
attn_window_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmKV,
                       const __grid_constant__ CUtensorMap tmO, float* __restrict__ lse, int S, int n_heads, int n_kv, int n_batch, int n_qblocks, int window, int sinks,
                       float scale_log2, int* err) {
  using C = FwdCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + B_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
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

  auto load_k = [&](int j) {
    const int st = j % C::NK;
    mbar_expect_tx(bar(B_KFULL + st), C::KV_BYTES);
#pragma unroll
    for (int kc = 0; kc < C::KC; ++kc)
      tma_load_3d(sbase + C::OFF_K + st * C::KV_BYTES + kc * (C::BK * 128), &tmKV, bar(B_KFULL + st), hq + kvh * D + kc * 64,
                  runs.block(j) * C::BK, b);
  };
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
    // the first loads do not wait for the rest of the set-up
    pdl_wait();
    mbar_expect_tx(bar(B_QFULL), C::Q_BYTES);
#pragma unroll
    for (int kc = 0; kc < C::KC; ++kc)
      tma_load_3d(sbase + kc * (C::BQ * 128), &tmQ, bar(B_QFULL), n * D + kc * 64, q0, b);
    for (int j = 0; j < nb && j < C::NK; ++j) load_k(j);
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
      for (int j = C::NK; j < nb; ++j) {
        if (!mbar_wait(bar(B_KEMPTY + j % C::NK), ((uint32_t)(j / C::NK) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x61)) break;
        load_k(j);
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
    {
      const uint32_t elected = elect_one();
      const uint32_t idesc_base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(C::BQ >> 4) << 24);
      const uint32_t idesc_s = idesc_base | ((uint32_t)(C::BK >> 3) << 17);            // N = 64 keys, both K-major
      const uint32_t idesc_pv = idesc_base | (1u << 16) | ((uint32_t)(D >> 3) << 17);  // N = D, B (V) mn-major
      const uint64_t dq = umma_desc_sw128(sbase, 0, 1024);
      auto wait_all = [&](int i, uint32_t parity, int site) {
        const bool ok = mbar_wait(bar(i), parity, abort_flag, err, kWaitLimitCycles, site);
        return __all_sync(0xffffffffu, ok) != 0;
      };
      auto issue_s = [&](int j) -> bool {
        const int st = j % C::NK;
        if (!wait_all(B_KFULL + st, (uint32_t)(j / C::NK) & 1u, 0x63)) return false;
        tc_fence_after();
        const uint64_t dk = umma_desc_sw128(sbase + C::OFF_K + st * C::KV_BYTES, 0, 1024);
        const uint32_t d_tmem = tmem_base + (uint32_t)((j & 1) * C::BK);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t qo = (uint64_t)(((k >> 2) * (C::BQ * 128) + (k & 3) * 32) >> 4);
          const uint64_t ko = (uint64_t)(((k >> 2) * (C::BK * 128) + (k & 3) * 32) >> 4);
          umma_bf16_if(elected, d_tmem, dq + qo, dk + ko, idesc_s, k > 0 ? 1u : 0u);
        }
        umma_commit_if(elected, bar(B_SFULL + (j & 1)));
        umma_commit_if(elected, bar(B_KEMPTY + st));
        return true;
      };
      bool ok = wait_all(B_QFULL, 0, 0x64) && issue_s(0);
      for (int j = 0; j < nb && ok; ++j) {
        if (j + 1 < nb && !issue_s(j + 1)) { ok = false; break; }
        const int st = j % C::NV;
        ok = wait_all(B_VFULL + st, (uint32_t)(j / C::NV) & 1u, 0x65) && wait_all(B_PFULL + (j & 1), ((uint32_t)j >> 1) & 1u, 0x66);
        if (!ok) break;
        tc_fence_after();
        const uint64_t dv = umma_desc_sw128(sbase + C::OFF_V + st * C::KV_BYTES, C::BK * 128, 1024);
        const uint32_t tp = tmem_base + (uint32_t)((j & 1) * C::BK);  // bf16 P: 16 keys = 8 columns per K step
#pragma unroll
        for (int k = 0; k < C::BK / 16; ++k)
          umma_bf16_ts_if(elected, tmem_base + C::O_COL, tp + (uint32_t)(k * 8), dv + (uint64_t)((k * 2048) >> 4), idesc_pv,
                       (j > 0 || k > 0) ? 1u : 0u);
        umma_commit_if(elected, bar(B_VEMPTY + st));
        umma_commit_if(elected, bar(B_ODONE));
      }
      if (ok) umma_commit_if(elected, bar(B_OFINAL));
    }
  } else {
    // softmax warps (2..5): one query row per thread = TMEM lane
    const int q = warp & 3;
    const int row = q0 + q * 32 + lane;
    const uint32_t tlane = tmem_base + ((uint32_t)(q * 32) << 16);
    const int wmin = q0 + q * 32, wmax = wmin + 31;  // rows of this warp
    // The row reference is an integer in the log2 domain: any such reference gives the same softmax, and bf16 rounding commutes
    // with powers of two.  So it need not be the maximum, only near it: the exponentials of a block are taken against the
    // reference that the blocks before left, in one pass, and taken again against a new one only if their maximum turns out
    // more than 2^kRefSlack above it (or, for a row that has seen nothing, far below it).
    // lsum is the sum of the exponentials; o is divided by nsum, in which blocks on an edge of the mask count with their
    // rounded P: the weights of a row that sees few keys then add up to 1, and a row that sees one key returns its value.
    // (Over many keys the roundings average out, and the unrounded sum serves.)
    float mref = 0.f, lsum = 0.f, nsum = 0.f;
    bool ok = true;
    for (int j = 0; j < nb && ok; ++j) {
      ok = mbar_wait(bar(B_SFULL + (j & 1)), ((uint32_t)j >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x67);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t t_s = tlane + (uint32_t)((j & 1) * C::BK);
      const int first = runs.block(j) * C::BK, last = first + C::BK - 1;
      // 64 keys of which no row of the warp sees any are not read, and only those on an edge of the mask are tested one by one
      // (both warp-uniform)
      const bool none = first > wmax || (last < wmin - window + 1 && first >= sinks);
      const bool all = last <= wmin && (first > wmax - window || last < sinks);
      uint32_t pw[32];  // bf16 pairs: keys 2c, 2c+1 in word c
      float2 psum = both(0.f);
      if (none) {
#pragma unroll
        for (int e = 0; e < 32; ++e) pw[e] = 0u;
      } else {
        for (;;) {
          uint32_t r0[32], r1[32];
          tmem_ld32(t_s, r0);
          tmem_ld32(t_s + 32, r1);
          tmem_ld_wait();
          if (!all) {
            const int hi = row - first;
            const uint32_t seen0 = visible(hi, hi - window + 1, sinks - first);
            const uint32_t seen1 = visible(hi - 32, hi - 32 - window + 1, sinks - first - 32);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              r0[e] = seen0 & (1u << e) ? r0[e] : 0xff800000u;  // -inf
              r1[e] = seen1 & (1u << e) ? r1[e] : 0xff800000u;
            }
          }
          float mx = -INFINITY;
          psum = both(0.f);
          softmax_chunk(r0, scale_log2, mref, pw, psum, mx);
          softmax_chunk(r1, scale_log2, mref, pw + 16, psum, mx);
          const float mcand = ceilf(mx * scale_log2);  // scale_log2 > 0: the maximum commutes with it
          const bool move = mcand > mref + kRefSlack || (lsum == 0.f && mx > -INFINITY && mcand < mref - 2.f * kRefSlack);
          if (!__any_sync(0xffffffffu, move)) break;
          const float alpha = move && lsum > 0.f ? fast_exp2(mref - mcand) : 1.0f;  // an exact power of two
          if (move) mref = mcand;
          lsum *= alpha;
          nsum *= alpha;
          if (j > 0 && __any_sync(0xffffffffu, alpha != 1.0f)) {  // rescale O, behind the previous P V product
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
        }
        if (!ok) break;
        lsum += psum.x + psum.y;
        if (!all) {
          psum = both(0.f);
#pragma unroll
          for (int e = 0; e < 32; ++e) psum = add2(psum, make_float2(bf16_lo(pw[e]), bf16_hi(pw[e])));
        }
        nsum += psum.x + psum.y;
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
      const uint32_t out = sbase + (uint32_t)(q * 32 * D * 2);  // Q has been read
      stage_rows<D>(out, lane, tlane + (uint32_t)C::O_COL, 1.0f / nsum);
      send_rows<D>(&tmO, out, lane, n * D, q0 + q * 32, b, S);
      if (row < S) lse[((long long)b * n_heads + n) * S + row] = (mref + log2f(lsum)) * kLn2;
      if (lane == 0) bulk_wait_group0();
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
  CUtensorMap tmQ, tmKV, tmO;
  if (!make_tmap_3d(&tmQ, qkv, nqkv, S, B, nqkv, C::BQ) || !make_tmap_3d(&tmKV, qkv, nqkv, S, B, nqkv, C::BK) ||
      !make_tmap_3d(&tmO, o, nh * D, S, B, nh * D, 32))
    return cudaErrorInvalidValue;
  const float scale_log2 = (float)((1.0 / sqrt((double)D)) * 1.4426950408889634);
  const int nqb = (S + C::BQ - 1) / C::BQ;
  return launch_pdl(attn_window_fwd_kernel<D>, dim3((unsigned)(nqb * nh * B)), dim3(FWD_THREADS), C::SMEM_BYTES, st, tmQ, tmKV, tmO, lse,
                    S, nh, nkv, B, nqb, window, sinks, scale_log2, err);
}

// ============================================================================ backward
// dK, dV: one CTA per (128 keys, kv head, batch row) or part of its queries; K and V stay in shared memory, 128-query blocks
// of Q and dO of every query head of the group are streamed.  Per block (D = 128; all products 128 x 128 x D on the tensor cores)
//   S^T = K Q^T, dP^T = V dO^T        accumulators in TMEM
//   P^T = exp2(S^T c - LSE), dS^T = P^T (dP^T - delta)    compute warps, bf16 back over the columns they came from
//   dV += P^T dO, dK += dS^T Q        A operand from TMEM, the streamed tiles again as mn-major B operands
// TMEM is full (four 128-column accumulators at D = 128), so S and dP have one buffer each; what keeps the tensor pipe busy is
// that two chains alternate: dV_j and S_{j+1} run while the compute warps turn dP_j into dS_j, dK_j and dP_{j+1} while they
// turn S_{j+1} into P_{j+1}.  Blocks of 128 queries and not 64: an MMA of N = 64 takes as long as one
// of N = 128, because it is bound by the reads of its operands from shared memory.  (D = 64: blocks of 64 queries, half of
// everything, and two CTAs an SM: there the products are small against what a CTA's start and end cost, and the other CTA
// fills both.)
// dS^T also goes to a scratch array, from which dQ = dS K is one banded contraction (below): five products per pair of
// blocks in all instead of the seven of a backward pass that computes S and dP twice.
// P and dS enter their products, and the scratch, rounded to bf16 (the other operand's type): 2.4e-3 of a gradient's 2-norm where
// the gradient's own rounding takes 1.7e-3.
// A block of 128 queries takes 3150 cycles at D = 128, of which 2500 are the 320 KB that its products, loads and stores move
// through shared memory; a CTA's start takes 6000 and its end 5000.  S 16384, 16 / 8 heads, window 1024: 335 us.  B 8, S 1024, 12
// heads of 64, window 256: 48 us.
enum { K_XFULL = 0, K_QFULL = 1, K_QEMPTY = 4, K_OFULL = 7, K_OEMPTY = 10, K_STFULL = 13, K_STEMPTY = 15, K_SFULL = 17, K_DPFULL = 18,
       K_PFULL = 19, K_DSFULL = 20, K_ACCDONE = 21, K_COUNT = 22 };
constexpr int DKV_THREADS = 320;  // producer, MMA issuer, 8 compute warps

template <int D, int BLOCK>
struct DkvCfg {
  static constexpr int KC = D / 64;
  static constexpr int BQ = BLOCK, SUB = 128 / BQ, W = BQ / 2;  // queries a block; blocks in 128 queries; queries a thread
  static constexpr int TILE = 128 * D * 2, Y_TILE = BQ * D * 2;  // bytes of a resident, of a streamed tile
  static constexpr int NQ = D == 64 ? 3 : 2, NO = BQ == 128 && D == 64 ? 3 : 2;
  static constexpr int OFF_K = 0, OFF_V = TILE, OFF_Q = 2 * TILE, OFF_O = OFF_Q + NQ * Y_TILE;
  static constexpr int OFF_DS = OFF_O + NO * Y_TILE;  // 4 KB a compute warp: its share of dS^T on the way to memory
  static constexpr int OFF_STAT = OFF_DS + 8 * 4096;  // [2][lse * log2e, delta][BQ]
  static constexpr int OFF_BAR = OFF_STAT + 16 * BQ;
  static constexpr int SMEM_BYTES = OFF_BAR + 256;
  static constexpr int CTAS = BQ == 64 ? 2 : 1;  // an SM
  static constexpr int TMEM_COLS = BQ == 64 ? 256 : 512;
  static constexpr int COL_S = 0, COL_DP = BQ, COL_DV = 2 * BQ, COL_DK = 2 * BQ + D;
};
static_assert(DkvCfg<128, 128>::SMEM_BYTES <= 232448 && DkvCfg<64, 64>::SMEM_BYTES <= 115712, "shared memory of one SM, of half of one");

// The backward pass as the host plans it and the kernels read it.  A key block's streamed list (128-query blocks of every
// query head of the group) is cut into parts; dS^T is kept for a number of (batch row, kv head) groups at a time.
struct Plan {
  int S, n_heads, n_kv, window, sinks;
  int nxb;                // 128-row blocks of the sequence
  int nb;                 // query blocks a key block meets through the window
  int n_sink;             // key blocks that hold sink keys
  int chunk;              // streamed blocks a part has, at most
  int parts_sink, parts;  // parts of a sink block and of any other, at most
  int group0, groups;     // groups of this launch: [group0, group0 + groups)
  int all_groups;
  // blocks [x, queries_end(x)) of the queries see a key of block x
  __host__ __device__ int blocks_seen(int x) const {
    if (x < n_sink) return nxb - x;
    return nxb - x < nb ? nxb - x : nb;
  }
  __host__ __device__ int parts_of(int x) const {
    return (int)(((long long)blocks_seen(x) * (n_heads / n_kv) + chunk - 1) / chunk);
  }
  // first slot of a key block's partial sums
  __host__ __device__ int rank_of(int x) const {
    return x < n_sink ? x * parts_sink : n_sink * parts_sink + (x - n_sink) * parts;
  }
  __host__ __device__ int ranks() const { return n_sink * parts_sink + (nxb - n_sink) * parts; }
};

// A thread's row of 32 or 64 scores out of TMEM, and their bf16 pairs back into it.
template <int W>
__device__ __forceinline__ void load_scores(uint32_t t, float (&v)[W]) {
  uint32_t r[W / 32][32];
#pragma unroll
  for (int c = 0; c < W / 32; ++c) tmem_ld32(t + 32 * c, r[c]);
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = __uint_as_float(r[i / 32][i % 32]);
}
__device__ __forceinline__ void store_pairs(uint32_t t, const uint32_t (&w)[32]) { tmem_st32(t, w); }
__device__ __forceinline__ void store_pairs(uint32_t t, const uint32_t (&w)[16]) { tmem_st16(t, w); }

template <int D, int BLOCK>
__global__ void __launch_bounds__(DKV_THREADS, DkvCfg<D, BLOCK>::CTAS)
attn_window_dkv_kernel(const __grid_constant__ CUtensorMap tm_qkv, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do,
                       const __grid_constant__ CUtensorMap tm_out, const float* __restrict__ lse, const float* __restrict__ delta,
                       float* __restrict__ partial, bf16* __restrict__ ds_band, bf16* __restrict__ ds_sink,
                       const float* __restrict__ rope_cos, const float* __restrict__ rope_sin, const __grid_constant__ Plan pl,
                       float scale, float scale_log2, int* err) {
  using C = DkvCfg<D, BLOCK>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + K_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* s_stat = reinterpret_cast<float*>(smem + C::OFF_STAT);

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if ((sbase & 1023u) != 0u) {
    if (threadIdx.x == 0) atomicExch(err, (int)ERR_BAD_ALIGNMENT);
    return;
  }
  const int S = pl.S, n_heads = pl.n_heads, n_kv = pl.n_kv, n_rep = n_heads / n_kv;
  const int hq = n_heads * D, hkv = n_kv * D;
  // sink blocks, with the longest lists, first
  const int rank = (int)blockIdx.x / pl.groups, local = (int)blockIdx.x % pl.groups, grp = pl.group0 + local;
  const int kvh = grp % n_kv, b = grp / n_kv;
  const int n_sink_ranks = pl.n_sink * pl.parts_sink;
  const int x = rank < n_sink_ranks ? rank / pl.parts_sink : pl.n_sink + (rank - n_sink_ranks) / pl.parts;
  const int part = rank < n_sink_ranks ? rank % pl.parts_sink : (rank - n_sink_ranks) % pl.parts;
  const int x0 = x * 128;
  const int per_head = pl.blocks_seen(x), total = per_head * n_rep, np = pl.parts_of(x);
  if (part >= np) return;
  const int first128 = (int)((long long)total * part / np);
  const int iters = ((int)((long long)total * (part + 1) / np) - first128) * C::SUB;

  // block `it` of this CTA: query head of the group, 128-query block counted from x, first query
  auto rep_of = [&](int it) { return (first128 + it / C::SUB) / per_head; };
  auto rel_of = [&](int it) { return (first128 + it / C::SUB) % per_head; };
  auto head_of = [&](int it) { return kvh * n_rep + rep_of(it); };
  auto query_of = [&](int it) { return (x + rel_of(it)) * 128 + it % C::SUB * C::BQ; };
  auto load_q = [&](int it) {
    const int st = it % C::NQ;
    mbar_expect_tx(bar(K_QFULL + st), C::Y_TILE);
#pragma unroll
    for (int kc = 0; kc < C::KC; ++kc)
      tma_load_3d(sbase + C::OFF_Q + st * C::Y_TILE + kc * (C::BQ * 128), &tm_q, bar(K_QFULL + st), head_of(it) * D + kc * 64, query_of(it), b);
  };
  auto load_do = [&](int it) {
    const int st = it % C::NO;
    mbar_expect_tx(bar(K_OFULL + st), C::Y_TILE);
#pragma unroll
    for (int kc = 0; kc < C::KC; ++kc)
      tma_load_3d(sbase + C::OFF_O + st * C::Y_TILE + kc * (C::BQ * 128), &tm_do, bar(K_OFULL + st), head_of(it) * D + kc * 64, query_of(it), b);
  };
  if (threadIdx.x == 0) {
    mbar_init(bar(K_XFULL), 1);
    for (int i = 0; i < C::NQ; ++i) {
      mbar_init(bar(K_QFULL + i), 1);
      mbar_init(bar(K_QEMPTY + i), 1);
    }
    for (int i = 0; i < C::NO; ++i) {
      mbar_init(bar(K_OFULL + i), 1);
      mbar_init(bar(K_OEMPTY + i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(K_STFULL + i), 1);
      mbar_init(bar(K_STEMPTY + i), 8);
    }
    mbar_init(bar(K_SFULL), 1);
    mbar_init(bar(K_DPFULL), 1);
    mbar_init(bar(K_PFULL), 8);
    mbar_init(bar(K_DSFULL), 8);
    mbar_init(bar(K_ACCDONE), 1);
    *abort_flag = 0;
    mbar_fence_init();
    // the first loads do not wait for the rest of the set-up
    pdl_wait();
    mbar_expect_tx(bar(K_XFULL), 2 * C::TILE);
#pragma unroll
    for (int kc = 0; kc < C::KC; ++kc)
      tma_load_3d(sbase + C::OFF_K + kc * 16384, &tm_qkv, bar(K_XFULL), hq + kvh * D + kc * 64, x0, b);
    load_q(0);
#pragma unroll
    for (int kc = 0; kc < C::KC; ++kc)
      tma_load_3d(sbase + C::OFF_V + kc * 16384, &tm_qkv, bar(K_XFULL), hq + hkv + kvh * D + kc * 64, x0, b);
    load_do(0);
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
    for (int it = 0; it < iters; ++it) {
      const int n = head_of(it), q0 = query_of(it), ss = it & 1;
      bool ok = true;
      if (it > 0) {  // block 0 is on its way
        ok = mbar_wait(bar(K_QEMPTY + it % C::NQ), ((uint32_t)(it / C::NQ) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x71);
        if (!__all_sync(0xffffffffu, ok)) break;
        if (lane == 0) load_q(it);
        ok = mbar_wait(bar(K_OEMPTY + it % C::NO), ((uint32_t)(it / C::NO) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x72);
        if (!__all_sync(0xffffffffu, ok)) break;
        if (lane == 0) load_do(it);
      }
      ok = mbar_wait(bar(K_STEMPTY + ss), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x73);
      if (!__all_sync(0xffffffffu, ok)) break;
      const long long stat = ((long long)b * n_heads + n) * S;
#pragma unroll
      for (int e = 0; e < C::BQ / 32; ++e) {
        const int qq = q0 + lane + 32 * e;
        s_stat[ss * 2 * C::BQ + lane + 32 * e] = qq < S ? lse[stat + qq] * kLog2e : 0.f;
        s_stat[ss * 2 * C::BQ + C::BQ + lane + 32 * e] = qq < S ? delta[stat + qq] : 0.f;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(K_STFULL + ss));
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    // One queue in the order dV_j, S_{j+1}, dK_j, dP_{j+1}.  A score buffer is overwritten by the product issued behind its
    // last reader.  (Two issuers, one a chain, let the four products of a block run interleaved: S_{j+1} then ends with
    // the last of them and the compute warps wait for all four; 3800 cycles a block.)
    const uint32_t elected = elect_one();
    const uint32_t idesc_base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);
    const uint32_t idesc_s = idesc_base | ((uint32_t)(C::BQ >> 3) << 17);             // N = BQ, both K-major
    const uint32_t idesc_acc = idesc_base | (1u << 16) | ((uint32_t)(D >> 3) << 17);  // N = D, B mn-major
    auto wait_all = [&](int i, uint32_t parity, int site) {
      const bool ok = mbar_wait(bar(i), parity, abort_flag, err, kWaitLimitCycles, site);
      return __all_sync(0xffffffffu, ok) != 0;
    };
    // K or V (resident, at x_off) times the streamed tile y
    auto scores = [&](uint32_t x_off, uint32_t y_off, uint32_t col) {
      const uint64_t dx = umma_desc_sw128(sbase + x_off, 0, 1024), dy = umma_desc_sw128(sbase + y_off, 0, 1024);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint64_t ox = (uint64_t)(((k >> 2) * 16384 + (k & 3) * 32) >> 4);
        const uint64_t oy = (uint64_t)(((k >> 2) * (C::BQ * 128) + (k & 3) * 32) >> 4);
        umma_bf16_if(elected, tmem_base + col, dx + ox, dy + oy, idesc_s, k > 0 ? 1u : 0u);
      }
    };
    // the bf16 tile at score column `col` (TMEM) times the streamed tile y; each half of the queries sits at the start of its
    // fp32 columns, 16 queries = 8 columns
    auto accumulate = [&](uint32_t col, uint32_t y_off, uint32_t acc_col, bool first) {
      const uint64_t by = umma_desc_sw128(sbase + y_off, C::BQ * 128, 1024);
      constexpr int HALF = C::W / 16;  // steps of 16 queries in a half
#pragma unroll
      for (int k = 0; k < 2 * HALF; ++k)
        umma_bf16_ts_if(elected, tmem_base + acc_col, tmem_base + col + (uint32_t)(k / HALF * C::W + k % HALF * 8),
                        by + (uint64_t)((k * 2048) >> 4), idesc_acc, (first && k == 0) ? 0u : 1u);
    };
    bool ok = wait_all(K_XFULL, 0, 0x74) && wait_all(K_QFULL, 0, 0x75) && wait_all(K_OFULL, 0, 0x76);
    if (ok) {
      tc_fence_after();
      scores(C::OFF_K, C::OFF_Q, C::COL_S);
      umma_commit_if(elected, bar(K_SFULL));
      scores(C::OFF_V, C::OFF_O, C::COL_DP);
      umma_commit_if(elected, bar(K_DPFULL));
    }
    for (int it = 0; it < iters && ok; ++it) {
      const int sq = it % C::NQ, so = it % C::NO, nq = (it + 1) % C::NQ, no = (it + 1) % C::NO;
      const bool more = it + 1 < iters;
      if (!(ok = wait_all(K_PFULL, (uint32_t)it & 1u, 0x77))) break;
      tc_fence_after();
      accumulate(C::COL_S, C::OFF_O + so * C::Y_TILE, C::COL_DV, it == 0);
      umma_commit_if(elected, bar(K_OEMPTY + so));  // dP_j and dV_j have read dO_j
      if (more) {
        if (!(ok = wait_all(K_QFULL + nq, (uint32_t)((it + 1) / C::NQ) & 1u, 0x78))) break;
        tc_fence_after();
        scores(C::OFF_K, C::OFF_Q + nq * C::Y_TILE, C::COL_S);
        umma_commit_if(elected, bar(K_SFULL));
      }
      if (!(ok = wait_all(K_DSFULL, (uint32_t)it & 1u, 0x79))) break;
      tc_fence_after();
      accumulate(C::COL_DP, C::OFF_Q + sq * C::Y_TILE, C::COL_DK, it == 0);
      umma_commit_if(elected, bar(K_QEMPTY + sq));  // S_j and dK_j have read Q_j
      if (more) {
        if (!(ok = wait_all(K_OFULL + no, (uint32_t)((it + 1) / C::NO) & 1u, 0x7a))) break;
        tc_fence_after();
        scores(C::OFF_V, C::OFF_O + no * C::Y_TILE, C::COL_DP);
        umma_commit_if(elected, bar(K_DPFULL));
      }
    }
    if (ok) umma_commit_if(elected, bar(K_ACCDONE));
  } else {
    // ------------------------------------------------------------------ compute warps: one key a thread, half of the queries each
    const int q = warp & 3, ch = (warp - 2) >> 2;
    const int rloc = q * 32 + lane, row = x0 + rloc;
    const int rmin = x0 + q * 32, rmax = rmin + 31;
    const uint32_t tlane = tmem_base + ((uint32_t)(q * 32) << 16);
    const uint32_t t_s = tlane + (uint32_t)(C::COL_S + ch * C::W), t_dp = tlane + (uint32_t)(C::COL_DP + ch * C::W);
    const uint32_t stage = sbase + (uint32_t)(C::OFF_DS + (warp - 2) * 4096);
    // the queries that see key `row` are [row, row_end)
    const int row_end = row < pl.sinks || S - row < pl.window ? S : row + pl.window;
    bool ok = true;
    for (int it = 0; it < iters; ++it) {
      const int ss = it & 1;
      const int rel = rel_of(it);
      const int cmin = query_of(it) + ch * C::W;
      const float* st_lse = s_stat + ss * 2 * C::BQ + ch * C::W;
      const float* st_dl = st_lse + C::BQ;
      ok = mbar_wait(bar(K_STFULL + ss), (uint32_t)(it >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x7b) &&
           mbar_wait(bar(K_SFULL), (uint32_t)it & 1u, abort_flag, err, kWaitLimitCycles, 0x7c);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      float p[C::W];
      load_scores(t_s, p);
#pragma unroll
      for (int i = 0; i < C::W; i += 4) {
        const float4 l4 = *reinterpret_cast<const float4*>(st_lse + i);
        p[i] = fast_exp2(fmaf(p[i], scale_log2, -l4.x));
        p[i + 1] = fast_exp2(fmaf(p[i + 1], scale_log2, -l4.y));
        p[i + 2] = fast_exp2(fmaf(p[i + 2], scale_log2, -l4.z));
        p[i + 3] = fast_exp2(fmaf(p[i + 3], scale_log2, -l4.w));
      }
      // single elements are only tested where the warp's tile touches an edge of the mask (warp-uniform)
      const bool full = cmin >= rmax && cmin + C::W <= S && (rmax < pl.sinks || cmin + C::W - 1 - rmin < pl.window);
      if (!full) {
        const int lo = row - cmin, hi = row_end - cmin;
#pragma unroll
        for (int i = 0; i < C::W; ++i)
          if (i < lo || i >= hi) p[i] = 0.f;
      }
      uint32_t w[C::W / 2];
#pragma unroll
      for (int c = 0; c < C::W / 2; ++c) w[c] = pack_bf16(p[2 * c], p[2 * c + 1]);
      store_pairs(t_s, w);  // over this warp's own (already loaded) columns
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(K_PFULL));

      ok = mbar_wait(bar(K_DPFULL), (uint32_t)it & 1u, abort_flag, err, kWaitLimitCycles, 0x7d);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      {
        float d[C::W];
        load_scores(t_dp, d);
#pragma unroll
        for (int i = 0; i < C::W; i += 4) {
          const float4 e4 = *reinterpret_cast<const float4*>(st_dl + i);
          p[i] *= d[i] - e4.x;
          p[i + 1] *= d[i + 1] - e4.y;
          p[i + 2] *= d[i + 2] - e4.z;
          p[i + 3] *= d[i + 3] - e4.w;
        }
      }
#pragma unroll
      for (int c = 0; c < C::W / 2; ++c) w[c] = pack_bf16(p[2 * c], p[2 * c + 1]);
      store_pairs(t_dp, w);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(K_DSFULL));
        mbar_arrive(bar(K_STEMPTY + ss));
      }
      // Off the chain's critical path: the same rounded dS^T to the scratch of the dQ contraction, whose operand tiles of
      // 64 keys x 128 queries lie there as the very bytes its shared memory will hold: [key half][32-query chunk][64 keys]
      // rows of 64 bytes under the 64-byte swizzle.  A warp's 32 keys of a chunk are 2 KB in one piece and leave as a bulk
      // copy.  (Stored by the threads themselves they held up the next block by 1900 cycles.)
      if (ds_band != nullptr) {
        const long long z = (long long)local * n_rep + rep_of(it);
        const int chunk = (cmin & 127) >> 5;  // of the 128 queries' four
        if (rel < pl.nb) {
          if (lane == 0) bulk_wait_group_read0();
          __syncwarp();
#pragma unroll
          for (int c = 0; c < C::W / 8; ++c) {  // 16-byte piece c & 3 of chunk c >> 2
            const uint32_t at = stage + (uint32_t)((c >> 2) * 2048 + lane * 64 + (((c & 3) ^ ((lane >> 1) & 3)) * 16));
            st_shared_v4(at, make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]));
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            uint8_t* dst = reinterpret_cast<uint8_t*>(ds_band) +
                           (((z * pl.nxb + x) * pl.nb + rel) * 8 + (q >> 1) * 4 + chunk) * 4096 + (q & 1) * 2048;
#pragma unroll
            for (int c = 0; c < C::W / 32; ++c) bulk_store(dst + c * 4096, stage + c * 2048, 2048);
            bulk_commit_group();
          }
        } else if (row < pl.sinks) {  // beyond the window only sink keys are seen: rows of [chunk][sink key][32 queries]
          bf16* dst = ds_sink + ((((z * pl.nxb + x + rel) * 4 + chunk) * pl.sinks + row) * 32);
#pragma unroll
          for (int c = 0; c < C::W / 32; ++c, dst += (long long)pl.sinks * 32) {
            store8_b32(dst, w + 16 * c);
            store8_b32(dst + 16, w + 16 * c + 8);
          }
        }
      }
    }
    if (lane == 0) bulk_wait_group0();
    __syncwarp();
    if (ok) {
      ok = mbar_wait(bar(K_ACCDONE), 0, abort_flag, err, kWaitLimitCycles, 0x7e);
      ok = __all_sync(0xffffffffu, ok);
    }
    if (ok) {
      tc_fence_after();
      constexpr int H = D / 2;
      const uint32_t t_dk = tlane + (uint32_t)C::COL_DK, t_dv = tlane + (uint32_t)C::COL_DV;
      if (np == 1) {
        // this CTA holds the whole sum: one warp of a lane quarter takes dK (scaled, rotated back), the other dV
        const uint32_t out = sbase + (uint32_t)((warp - 2) * 32 * D * 2);  // K and V have been read
        if (ch == 0) {
          if (rope_cos != nullptr) stage_rows_unrotated<D>(out, stage, lane, t_dk, scale, rope_cos, rope_sin, rmin, S);
          else stage_rows<D>(out, lane, t_dk, scale);
        } else {
          stage_rows<D>(out, lane, t_dv, 1.0f);
        }
        send_rows<D>(&tm_out, out, lane, hq + ch * hkv + kvh * D, rmin, b, S);
        if (lane == 0) bulk_wait_group0();
      } else {
        // partial sums [part][dK columns, dV columns][128 keys]: a warp writes 32 consecutive keys of a column
        float* dst = partial + ((long long)rank * pl.all_groups + grp) * (2 * D * 128) + rloc;
#pragma unroll 1
        for (int c = ch * H; c < (ch + 1) * H; c += 32) {
          float v[32];
          tmem_load_cols<32>(t_dk + (uint32_t)c, v);
#pragma unroll
          for (int i = 0; i < 32; ++i) dst[(c + i) * 128] = v[i];
          tmem_load_cols<32>(t_dv + (uint32_t)c, v);
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

// ---------------------------------------------------------------- partial sums of dK and dV
// Adds the partial sums of a key block's parts in part order, scales and rotates dK, rounds once.  A unit of this work is 32
// columns of a key block (16 of dK and their partners D / 2 further, or 32 of dV): a warp reads whole columns, 512 bytes each a
// part, every part's loads in flight at once; the sums pass through shared memory to threads that hold half a row of them
// each.  The units are taken by CTAs of the dQ kernel that have no tile (left), which need none of them: as a launch of its own
// behind it this cost 8 us.
struct Join {
  const float* partial;
  bf16* dqkv;
  const float *rope_cos, *rope_sin;
  float scale;
  int cut;  // key blocks with partial sums
  __host__ __device__ int units(const Plan& pl, int d) const { return cut * pl.all_groups * (d / 16); }
};
constexpr int JOIN_SMEM = 32 * 132 * 4;

// all THREADS of a CTA; s_sum: [column][key]
template <int D, int THREADS>
__device__ __forceinline__ void join_unit(const Join& jn, const Plan& pl, int unit, float (*s_sum)[132]) {
  constexpr int H = D / 2, K_UNITS = H / 16, WARPS = THREADS / 32, OWN = (32 + WARPS - 1) / WARPS;
  const int groups = pl.all_groups, S = pl.S, n_heads = pl.n_heads, n_kv = pl.n_kv;
  const int piece = unit % (D / 16), x = unit / (D / 16) / groups, grp = unit / (D / 16) % groups;
  const int np = pl.parts_of(x);
  if (np == 1) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool is_k = piece < K_UNITS;
  const int c0 = is_k ? piece * 16 : (piece - K_UNITS) * 32;
  const long long part_stride = (long long)groups * (2 * D * 128);
  const float* src = jn.partial + ((long long)pl.rank_of(x) * groups + grp) * (2 * D * 128) + lane * 4;
  float4 acc[OWN];
  int off[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int l = min(warp + i * WARPS, 31);  // of the unit's 32 columns
    off[i] = (is_k ? (l < 16 ? c0 + l : H + c0 + l - 16) : D + c0 + l) * 128;
    acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll 4
  for (int p = 0; p < np; ++p) {
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(src + p * part_stride + off[i]);
      acc[i].x += v.x; acc[i].y += v.y; acc[i].z += v.z; acc[i].w += v.w;
    }
  }
#pragma unroll
  for (int i = 0; i < OWN; ++i)
    if (warp + i * WARPS < 32) *reinterpret_cast<float4*>(&s_sum[warp + i * WARPS][lane * 4]) = acc[i];
  __syncthreads();
  const int kvh = grp % n_kv, b = grp / n_kv;
  for (int v = threadIdx.x; v < 256; v += THREADS) {
    const int r = v & 127, part = v >> 7, row = x * 128 + r;
    if (row >= S) continue;
    bf16* dst = jn.dqkv + ((long long)b * S + row) * (long long)((n_heads + 2 * n_kv) * D) + (n_heads + (is_k ? 0 : n_kv) + kvh) * D + c0;
    if (is_k) {
      float lo[8], hi[8];
      const int i0 = part * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        lo[i] = s_sum[i0 + i][r] * jn.scale;
        hi[i] = s_sum[16 + i0 + i][r] * jn.scale;
      }
      if (jn.rope_cos != nullptr) unrotate<8>(lo, hi, jn.rope_cos + (long long)row * H + c0 + i0, jn.rope_sin + (long long)row * H + c0 + i0);
      store_bf16_row<8>(dst + i0, lo);
      store_bf16_row<8>(dst + H + i0, hi);
    } else {
      float f[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = s_sum[part * 16 + i][r];
      store_bf16_row<16>(dst + part * 16, f);
    }
  }
  __syncthreads();  // s_sum is free again
}

// The same behind the dQ kernel that recomputes the scores.
template <int D>
__global__ void __launch_bounds__(256)
attn_window_join_kernel(const __grid_constant__ Join jn, const __grid_constant__ Plan pl) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s_sum[32][132];
  join_unit<D, 256>(jn, pl, (int)blockIdx.x, s_sum);
}

// ---------------------------------------------------------------- dQ from the stored dS^T
// dQ[i] = scale * sum over visible keys j of dS[i, j] K[j], rotated back: per 128-query tile one product over the keys of its
// band and the sink keys behind it.  Persistent: warp 0 TMA producer, warp 1 MMA issuer, warps 2..5 epilogue, accumulators
// double-buffered in TMEM, two CTAs an SM.  Both operands are mn-major (the contraction index is the row of dS^T and of K).
// The kernel is bound by the bytes of dS^T: S 16384, 16 / 8 heads of 128, window 1024: 0.66 GB in 125 us, 5.2 TB/s.
enum { DQ_THREADS = 192 };

template <int D>
struct DqCfg {
  static constexpr int A_BYTES = 64 * 128 * 2;  // one box of dS^T: 4 chunks of [64 keys][32 queries], 64-byte swizzle
  static constexpr int B_BYTES = 64 * D * 2;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int STAGES = D == 64 ? 3 : 2;
  static constexpr int OFF_OUT = STAGES * STAGE_BYTES;    // an epilogue warp's rows
  static constexpr int OFF_TABLE = OFF_OUT + 128 * D * 2;  // and its piece of the rotation tables
  static constexpr int OFF_BAR = OFF_TABLE + 4 * 4096;
  static constexpr int SMEM_BYTES = OFF_BAR + 128;
  static constexpr int TMEM_COLS = 2 * D;
};

template <int D>
__global__ void __launch_bounds__(DQ_THREADS, 2)
attn_window_dq_kernel(const bf16* __restrict__ ds_band, const __grid_constant__ CUtensorMap tm_sink,
                      const __grid_constant__ CUtensorMap tm_qkv, const __grid_constant__ CUtensorMap tm_out, const float* __restrict__ rope_cos,
                      const float* __restrict__ rope_sin, const __grid_constant__ Plan pl, const __grid_constant__ Join jn, float scale,
                      int* err) {
  using C = DqCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * C::STAGES + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * C::STAGES + 2 + a); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::STAGES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((sbase & 1023u) != 0u) {
    if (threadIdx.x == 0) atomicExch(err, (int)ERR_BAD_ALIGNMENT);
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull_bar(a), 1);
      mbar_init(tempty_bar(a), 4);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_sink);
    tma_prefetch_desc(&tm_qkv);
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
  pdl_wait();

  const int S = pl.S, n_rep = pl.n_heads / pl.n_kv;
  const int hq = pl.n_heads * D;
  const int nz = pl.groups * n_rep, ntiles = pl.nxb * nz;
  // tile t: query block qt of head z of this launch; 64-key steps: sink keys behind the band, then the band
  struct Tile {
    int qt, z, kvh, n, b, x_first, n_sink64, steps;
  };
  auto tile_of = [&](int t) {
    Tile r;
    r.qt = pl.nxb - 1 - t / nz;
    r.z = t % nz;
    const int grp = pl.group0 + r.z / n_rep;
    r.kvh = grp % pl.n_kv;
    r.b = grp / pl.n_kv;
    r.n = r.kvh * n_rep + r.z % n_rep;
    r.x_first = max(0, r.qt - pl.nb + 1);
    r.n_sink64 = (min(pl.sinks, r.x_first * 128) + 63) / 64;
    r.steps = r.n_sink64 + (r.qt - r.x_first + 1) * 2;
    return r;
  };

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
        const Tile r = tile_of(t);
        for (int i = 0; i < r.steps; ++i) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, err, kWaitLimitCycles, 0x81)) { ok = false; break; }
          const uint32_t fb = full_bar(stage);
          mbar_expect_tx(fb, C::STAGE_BYTES);
          const uint32_t a_dst = sbase + stage * C::STAGE_BYTES, b_dst = a_dst + C::A_BYTES;
          int key0;
          if (i < r.n_sink64) {
            key0 = i * 64;
            tma_load_4d(a_dst, &tm_sink, fb, 0, key0, r.qt * 4, r.z);  // keys past the last sink read as 0
          } else {
            const int j = i - r.n_sink64, x = r.x_first + (j >> 1);
            key0 = x * 128 + (j & 1) * 64;
            bulk_load(a_dst, ds_band + ((((long long)r.z * pl.nxb + x) * pl.nb + r.qt - x) * 2 + (j & 1)) * 8192, C::A_BYTES, fb);
          }
#pragma unroll
          for (int c = 0; c < D / 64; ++c) tma_load_3d(b_dst + c * 8192, &tm_qkv, fb, hq + r.kvh * D + 64 * c, key0, r.b);
          if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(D >> 3) << 17) |
                             ((uint32_t)(128 >> 4) << 24);  // both operands mn-major, N = D, M = 128
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
        const Tile r = tile_of(t);
        if (!mbar_wait(tempty_bar(acc), acc_phase ^ 1u, abort_flag, err, kWaitLimitCycles, 0x82)) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(acc * D);
        for (int i = 0; i < r.steps; ++i) {
          if (!mbar_wait(full_bar(stage), phase, abort_flag, err, kWaitLimitCycles, 0x83)) { ok = false; break; }
          tc_fence_after();
          const uint32_t a_addr = sbase + stage * C::STAGE_BYTES, b_addr = a_addr + C::A_BYTES;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma_bf16(d_tmem, umma_desc_sw64(a_addr + k * 1024, 4096, 512), umma_desc_sw128(b_addr + k * 2048, 8192, 1024), idesc,
                      (i | k) != 0 ? 1u : 0u);
          umma_commit(empty_bar(stage));
          if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        umma_commit(tfull_bar(acc));
        acc ^= 1;
        if (acc == 0) acc_phase ^= 1u;
      }
    }
  } else {
    const int q = warp & 3;
    int acc = 0;
    uint32_t acc_phase = 0;
    const uint32_t out = sbase + (uint32_t)(C::OFF_OUT + q * 32 * D * 2), table = sbase + (uint32_t)(C::OFF_TABLE + q * 4096);
    for (int t = blockIdx.x; t < ntiles; t += gridDim.x) {
      const Tile r = tile_of(t);
      bool ok = mbar_wait(tfull_bar(acc), acc_phase, abort_flag, err, kWaitLimitCycles, 0x84);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const int row0 = r.qt * 128 + q * 32;
      const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * D);
      if (lane == 0) bulk_wait_group_read0();  // the last tile's rows have left the staging buffer
      __syncwarp();
      if (rope_cos != nullptr) stage_rows_unrotated<D>(out, table, lane, taddr, scale, rope_cos, rope_sin, row0, S);
      else stage_rows<D>(out, lane, taddr, scale);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(tempty_bar(acc));
      send_rows<D>(&tm_out, out, lane, r.n * D, row0, r.b, S);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
    }
    if (lane == 0) bulk_wait_group0();
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
  // the tiles' loads and stores have left shared memory (waited for above); the CTAs with the fewest tiles begin with the units
  static_assert(JOIN_SMEM <= C::OFF_OUT, "the stages hold a unit's columns");
  const int units = jn.units(pl, D);
  for (int u = (int)(gridDim.x - 1 - blockIdx.x); u < units; u += (int)gridDim.x)
    join_unit<D, DQ_THREADS>(jn, pl, u, reinterpret_cast<float (*)[132]>(smem));
}

// ---------------------------------------------------------------- dQ without stored dS^T
// For sequences and windows whose dS^T would not fit the scratch even for one group: 128 queries (Q, dO) resident, 64-key
// blocks (K, V) streamed, S and dP computed again into one of two TMEM buffers, dQ += dS K.
// (S 8400, window 2000, 64 heads of 128: on one kv head, which takes this way, the backward pass is 2.58 ms with 29 MB of
// scratch; on two, whose dS^T is stored, 2.26 ms with 1.2 GB.)
enum { BB_XFULL = 0, BB_YFULL = 1, BB_YEMPTY = 5, BB_SDPFULL = 9, BB_TFULL = 11, BB_ACCDONE = 13, BB_COUNT = 14 };
constexpr int DQR_THREADS = 352;  // producer, 2 MMA issuers, 8 compute warps

template <int D>
struct DqrCfg {
  static constexpr int KC = D / 64;
  static constexpr int X_BYTES = 128 * D * 2;
  static constexpr int Y_BYTES = 64 * D * 2;
  static constexpr int NST = 4;
  static constexpr int OFF_X1 = 0, OFF_X2 = X_BYTES, OFF_Y = 2 * X_BYTES;
  static constexpr int OFF_BAR = OFF_Y + NST * 2 * Y_BYTES;
  static constexpr int SMEM_BYTES = OFF_BAR + 256;
  static constexpr int TMEM_COLS = 512;  // buffer b: S at b*128, dP at b*128+64; accumulator from column 256
  static constexpr int ACC0 = 256;
};

template <int D>
__global__ void __launch_bounds__(DQR_THREADS, 1)
attn_window_dq_recompute_kernel(const __grid_constant__ CUtensorMap tm_qkv128, const __grid_constant__ CUtensorMap tm_qkv64,
                                const __grid_constant__ CUtensorMap tm_do128, const float* __restrict__ lse,
                                const float* __restrict__ delta, bf16* __restrict__ dqkv, const float* __restrict__ rope_cos,
                                const float* __restrict__ rope_sin, const __grid_constant__ Plan pl, float scale,
                                float scale_log2, int* err) {
  using C = DqrCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + BB_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((sbase & 1023u) != 0u) {
    if (threadIdx.x == 0) atomicExch(err, (int)ERR_BAD_ALIGNMENT);
    return;
  }
  const int S = pl.S, n_heads = pl.n_heads, n_kv = pl.n_kv;
  const int hq = n_heads * D, hkv = n_kv * D;
  const long long ld = hq + 2 * hkv;
  const int all = pl.all_groups / n_kv * n_heads;
  const int rank = (int)blockIdx.x / all, grp = (int)blockIdx.x % all;
  const int x0 = (pl.nxb - 1 - rank) * 128;  // the first query blocks, with fewer keys, end the launch
  const int n_q = grp % n_heads, b = grp / n_heads, kvh = n_q / (n_heads / n_kv);
  const KeyRuns runs(x0, S, pl.window, pl.sinks);
  const int iters = runs.count;

  if (threadIdx.x == 0) {
    mbar_init(bar(BB_XFULL), 1);
    for (int i = 0; i < C::NST; ++i) {
      mbar_init(bar(BB_YFULL + i), 1);
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
        tma_load_3d(sbase + C::OFF_X1 + kc * 16384, &tm_qkv128, bar(BB_XFULL), n_q * D + kc * 64, x0, b);
        tma_load_3d(sbase + C::OFF_X2 + kc * 16384, &tm_do128, bar(BB_XFULL), n_q * D + kc * 64, x0, b);
      }
      for (int it = 0; it < iters; ++it) {
        const int st = it % C::NST, y0 = runs.block(it) * 64;
        if (!mbar_wait(bar(BB_YEMPTY + st), (((uint32_t)(it / C::NST)) & 1u) ^ 1u, abort_flag, err, kWaitLimitCycles, 0x91)) break;
        const uint32_t ydst = sbase + C::OFF_Y + st * 2 * C::Y_BYTES;
        mbar_expect_tx(bar(BB_YFULL + st), 2 * C::Y_BYTES);
#pragma unroll
        for (int kc = 0; kc < C::KC; ++kc) {
          tma_load_3d(ydst + kc * 8192, &tm_qkv64, bar(BB_YFULL + st), hq + kvh * D + kc * 64, y0, b);
          tma_load_3d(ydst + C::Y_BYTES + kc * 8192, &tm_qkv64, bar(BB_YFULL + st), hq + hkv + kvh * D + kc * 64, y0, b);
        }
      }
    }
  } else if (warp == 1 || warp == 10) {
    // ------------------------------------------------------------------ MMA issuers
    // two threads, because one cannot issue products this small fast enough: side 0 owns S, side 1 owns dP and dQ += dS K
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
      bool ok = mbar_wait(bar(BB_XFULL), 0, abort_flag, err, kWaitLimitCycles, 0x92) &&
                mbar_wait(bar(BB_YFULL), 0, abort_flag, err, kWaitLimitCycles, 0x93);
      if (ok) {
        tc_fence_after();
        issue_sdp(0);
      }
      for (int it = 0; it < iters && ok; ++it) {
        if (it + 1 < iters) {
          const int y1s = (it + 1) % C::NST;
          if (!mbar_wait(bar(BB_YFULL + y1s), ((uint32_t)((it + 1) / C::NST)) & 1u, abort_flag, err, kWaitLimitCycles, 0x94)) { ok = false; break; }
          // the TMEM columns this writes were last read by this same thread's accumulating MMAs of block it-1: in order
          tc_fence_after();
          issue_sdp(it + 1);
        }
        const int bf = it & 1;
        if (!mbar_wait(bar(BB_TFULL + bf), ((uint32_t)it >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x95)) { ok = false; break; }
        tc_fence_after();
        const int yst = it % C::NST;
        const uint32_t y1 = sbase + C::OFF_Y + yst * 2 * C::Y_BYTES;
        // A operands (bf16) sit in TMEM where S / dP were: 16 streamed rows (K = 16) = 8 columns; the two compute warps of
        // a lane quarter each wrote their 32 at the start of their own 32 fp32 columns
        const uint32_t ta = tmem_base + (uint32_t)(bf * 128 + side * 64);
        const uint32_t first = it > 0 ? 1u : 0u;
        if (side == 1) {
          const uint64_t by = umma_desc_sw128(y1, 8192, 1024);
          const uint32_t dacc = tmem_base + (uint32_t)C::ACC0;
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
    const int row = x0 + rloc;
    const uint32_t tlane = tmem_base + ((uint32_t)(q * 32) << 16);
    const int rmin = x0 + q * 32, rmax = rmin + 31;
    float lse2_row = 0.f, delta_row = 0.f;
    if (row < S) {
      const long long stat = ((long long)b * n_heads + n_q) * S;
      lse2_row = lse[stat + row] * kLog2e;
      delta_row = delta[stat + row];
    }
    bool ok = true;
    for (int it = 0; it < iters; ++it) {
      const int bf = it & 1;
      ok = mbar_wait(bar(BB_SDPFULL + bf), ((uint32_t)it >> 1) & 1u, abort_flag, err, kWaitLimitCycles, 0x96);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      uint32_t rs[32], rp[32];
      tmem_ld32(tlane + (uint32_t)(bf * 128 + ch * 32), rs);
      tmem_ld32(tlane + (uint32_t)(bf * 128 + 64 + ch * 32), rp);
      tmem_ld_wait();

      // single elements are only tested where the warp's tile touches an edge of the mask (warp-uniform)
      const int cmin = runs.block(it) * 64 + ch * 32;
      const bool full = cmin + 31 <= rmin && (rmax - cmin < pl.window || cmin + 32 <= pl.sinks);
      const int hi = row - cmin, lo = row - pl.window + 1 - cmin, sk = pl.sinks - cmin;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        float p = fast_exp2(fmaf(__uint_as_float(rs[i]), scale_log2, -lse2_row));
        if (!full && (i > hi || (i < lo && i >= sk))) p = 0.f;
        rp[i] = __float_as_uint(p * (__uint_as_float(rp[i]) - delta_row));
      }
      // bf16 pairs back into TMEM, over this warp's own (already loaded) fp32 columns
      uint32_t wd[16];
#pragma unroll
      for (int c = 0; c < 16; ++c) wd[c] = pack_bf16(__uint_as_float(rp[2 * c]), __uint_as_float(rp[2 * c + 1]));
      tmem_st16(tlane + (uint32_t)(bf * 128 + 64 + ch * 32), wd);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BB_TFULL + bf));
    }
    if (ok) {
      ok = mbar_wait(bar(BB_ACCDONE), 0, abort_flag, err, kWaitLimitCycles, 0x98);
      ok = __all_sync(0xffffffffu, ok);
    }
    if (ok) {
      tc_fence_after();
      constexpr int W = D / 4, H = D / 2;
      const int i0 = ch * W;
      // this warp owns columns [i0, i0+W) and their partners D/2 further
      float lo[W], hi[W];
      tmem_load_cols<W>(tlane + (uint32_t)(C::ACC0 + i0), lo);
      tmem_load_cols<W>(tlane + (uint32_t)(C::ACC0 + H + i0), hi);
#pragma unroll
      for (int i = 0; i < W; ++i) { lo[i] *= scale; hi[i] *= scale; }
      if (rope_cos != nullptr) {
        const int pos = min(row, S - 1);
        unrotate<W>(lo, hi, rope_cos + (long long)pos * H + i0, rope_sin + (long long)pos * H + i0);
      }
      if (row < S) {
        bf16* dst = dqkv + ((long long)b * S + row) * ld + n_q * D;
        store_bf16_row<W>(dst + i0, lo);
        store_bf16_row<W>(dst + H + i0, hi);
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


// Parts: where the launch has several times more streamed blocks than SMs, a part is as long as a window block's whole list
// (or an eighth of a slot's share, if that is longer), so that only sink blocks are cut.  Smaller launches are cut into one
// part per slot (of a CTA on an SM), of at least 4 blocks: the set-up and the partial sums of a part cost about as much as 2.
// Groups: dS^T is kept for as many (batch row, kv head) groups at a time as kDsBytes holds.
constexpr size_t kDsBytes = (size_t)1 << 30;

struct Scratch {
  size_t delta, partial, band, sink, total;  // byte offsets and size
  bool stored;                               // dS^T is stored (else dQ recomputes it)
};

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Query blocks that a key block meets through the window, at most.
int window_blocks(int S, int window) {
  const int nxb = (S + 127) / 128, nb = (127 + window + 127) / 128;
  return nb < nxb ? nb : nxb;
}

// Queries that a streamed block of the dK/dV kernel has.  Heads of 64: half blocks and two CTAs an SM, except in launches of
// no more than six whole blocks an SM, whose CTAs run alone and want to be quick (B 8, S 1024, 12 heads: 57 against 69 us at
// window 128, 67 against 79 at 256, 91 against 103 at 1024; B 3, S 1531, 6 heads on one: 41 against 37).  Those are launches of
// 1536 blocks and more and of 864; on which side those between are better was not measured.
int block_of(int B, int S, int nh, int d, int window) {
  return d == 64 && (long long)B * nh * ((S + 127) / 128) * window_blocks(S, window) > 6 * kSms ? 64 : 128;
}

Plan make_plan(int B, int S, int nh, int nkv, int window, int sinks, Scratch* l, int d, int block) {
  Plan p;
  p.S = S; p.n_heads = nh; p.n_kv = nkv; p.window = window; p.sinks = sinks;
  p.nxb = (S + 127) / 128;
  p.nb = window_blocks(S, window);
  p.n_sink = (sinks + 127) / 128;
  p.group0 = 0;
  p.all_groups = p.groups = nkv * B;
  const long long n_rep = nh / nkv;
  const long long sink_len = p.n_sink > 0 ? n_rep * p.nxb : 0;
  const long long window_len = p.n_sink < p.nxb ? n_rep * p.blocks_seen(p.n_sink) : 0;
  long long total = window_len * (p.nxb - p.n_sink);
  total += n_rep * ((long long)p.n_sink * p.nxb - (long long)p.n_sink * (p.n_sink - 1) / 2);  // sink block x: nxb - x
  total *= p.all_groups;
  const long long slots = kSms * (block == 64 ? 2 : 1);  // CTAs that run at a time
  const long long per_slot = (total + slots - 1) / slots;
  const long long longest = window_len > 0 ? window_len : sink_len;
  long long chunk = per_slot < longest ? per_slot : longest;
  if (chunk < 4) chunk = 4;
  if (per_slot >= longest && chunk < (per_slot + 7) / 8) chunk = (per_slot + 7) / 8;
  p.chunk = (int)(chunk < INT_MAX ? chunk : INT_MAX);
  p.parts = window_len > chunk ? (int)((window_len + chunk - 1) / chunk) : 1;
  p.parts_sink = sink_len > chunk ? (int)((sink_len + chunk - 1) / chunk) : 1;

  const size_t part_slots = p.parts > 1 ? (size_t)p.ranks() : p.parts_sink > 1 ? (size_t)p.n_sink * p.parts_sink : 0;
  l->delta = 0;
  l->partial = round256((size_t)B * nh * S * sizeof(float));
  l->band = l->partial + part_slots * p.all_groups * (2 * d * 128) * sizeof(float);
  const size_t band = (size_t)n_rep * p.nxb * p.nb * 32768;  // of one group
  const size_t sink = p.nxb > p.nb ? (size_t)n_rep * p.nxb * 4 * sinks * 64 : 0;
  l->stored = band + sink <= 2 * kDsBytes;
  l->sink = l->total = l->band;
  if (l->stored) {
    size_t fit = kDsBytes / (band + sink);
    if (fit < 1) fit = 1;
    const int rounds = (int)((p.all_groups + fit - 1) / fit);
    p.groups = (p.all_groups + rounds - 1) / rounds;
    l->sink = l->band + round256(p.groups * band);
    l->total = l->sink + round256(p.groups * sink);
  }
  return p;
}

template <int D, int BLOCK>
cudaError_t bwd_t(const bf16* qkv, const bf16* o, const bf16* d_o, const float* lse, bf16* dqkv, const float* cs, const float* sn,
                  uint8_t* scratch, int B, int S, int nh, int nkv, int window, int sinks, int* err, cudaStream_t st, int& launches) {
  Scratch l;
  Plan pl = make_plan(B, S, nh, nkv, window, sinks, &l, D, BLOCK);
  static unsigned long long set_kv = 0, set_q = 0, set_r = 0;
  cudaError_t e = ensure_dynamic_smem(attn_window_dkv_kernel<D, BLOCK>, DkvCfg<D, BLOCK>::SMEM_BYTES, set_kv);
  if (e == cudaSuccess && l.stored) e = ensure_dynamic_smem(attn_window_dq_kernel<D>, DqCfg<D>::SMEM_BYTES, set_q);
  if (e == cudaSuccess && !l.stored) e = ensure_dynamic_smem(attn_window_dq_recompute_kernel<D>, DqrCfg<D>::SMEM_BYTES, set_r);
  if (e != cudaSuccess) return e;
  float* delta = reinterpret_cast<float*>(scratch + l.delta);
  float* partial = reinterpret_cast<float*>(scratch + l.partial);
  bf16* band = l.stored ? reinterpret_cast<bf16*>(scratch + l.band) : nullptr;
  bf16* sink = l.stored ? reinterpret_cast<bf16*>(scratch + l.sink) : nullptr;
  const int hq = nh * D, nqkv = (nh + 2 * nkv) * D, n_rep = nh / nkv;
  const bool has_sink = sinks > 0 && pl.nxb > pl.nb;
  CUtensorMap tq128, tq64, td128, tsink, tout, tdo;
  if (!make_tmap_3d(&tq128, qkv, nqkv, S, B, nqkv, 128) || !make_tmap_3d(&tq64, qkv, nqkv, S, B, nqkv, 64) ||
      !make_tmap_3d(&tout, dqkv, nqkv, S, B, nqkv, 32) || !make_tmap_3d(&tdo, d_o, hq, S, B, hq, DkvCfg<D, BLOCK>::BQ))
    return cudaErrorInvalidValue;
  if (!l.stored && !make_tmap_3d(&td128, d_o, hq, S, B, hq, 128)) return cudaErrorInvalidValue;
  if (l.stored) {
    if (!has_sink) tsink = tq64;  // not read
    else if (!make_tmap_ds(&tsink, sink, sinks, (uint64_t)pl.nxb * 4, (uint64_t)pl.groups * n_rep)) return cudaErrorInvalidValue;
  }
  const float scale = (float)(1.0 / sqrt((double)D));
  const float scale_log2 = (float)((1.0 / sqrt((double)D)) * 1.4426950408889634);
  int dev = 0, sms = kSms;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  e = attention_delta(o, d_o, delta, B, S, nh, D, st);
  launches = 1;
  const int per_round = pl.groups;
  Join jn{partial, dqkv, cs, sn, scale, pl.parts > 1 ? pl.nxb : pl.parts_sink > 1 ? pl.n_sink : 0};
  const Join none{partial, dqkv, cs, sn, scale, 0};
  for (int g0 = 0; g0 < pl.all_groups && e == cudaSuccess; g0 += per_round) {
    pl.group0 = g0;
    pl.groups = pl.all_groups - g0 < per_round ? pl.all_groups - g0 : per_round;
    e = launch_pdl(attn_window_dkv_kernel<D, BLOCK>, dim3((unsigned)pl.ranks() * pl.groups), dim3(DKV_THREADS), DkvCfg<D, BLOCK>::SMEM_BYTES, st,
                   tq128, DkvCfg<D, BLOCK>::BQ == 128 ? tq128 : tq64, tdo, tout, lse, delta, partial, band, sink, cs, sn, pl, scale, scale_log2, err);
    ++launches;
    if (e != cudaSuccess || !l.stored) continue;
    const bool last = g0 + per_round >= pl.all_groups;
    const long long ctas = (long long)pl.nxb * pl.groups * n_rep + (last ? jn.units(pl, D) : 0);
    e = launch_pdl(attn_window_dq_kernel<D>, dim3((unsigned)(ctas < 2 * sms ? ctas : 2 * sms)), dim3(DQ_THREADS), DqCfg<D>::SMEM_BYTES, st,
                   (const bf16*)band, tsink, tq64, tout, cs, sn, pl, last ? jn : none, scale, err);
    ++launches;
  }
  if (e != cudaSuccess) return e;
  if (!l.stored) {
    e = launch_pdl(attn_window_dq_recompute_kernel<D>, dim3((unsigned)(pl.nxb * nh * B)), dim3(DQR_THREADS), DqrCfg<D>::SMEM_BYTES, st,
                   tq128, tq64, td128, lse, delta, dqkv, cs, sn, pl, scale, scale_log2, err);
    if (e != cudaSuccess) return e;
    ++launches;
  }
  if (l.stored || jn.cut == 0) return cudaSuccess;
  ++launches;
  return launch_pdl(attn_window_join_kernel<D>, dim3((unsigned)jn.units(pl, D)), dim3(256), 0, st, jn, pl);
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
  Scratch l;
  make_plan(B, S, nh, nkv, window, sinks, &l, d, block_of(B, S, nh, d, window));
  return l.total;
}

// Not monotonic in S: a window or a number of sinks that S does not exceed is cut to it.  Within a 128-token block nothing but the
// size of what is kept per token changes with S, upwards, on either side of S = window (up to it there are no sinks); while S is
// within the sinks, the rows kept of them grow with S too, and the heads kept at a time step down: every S counts.
size_t attention_window_most_scratch_bytes(int max_batch, int max_seq, int nh, int nkv, int d, int window, int sinks) {
  if (window > max_seq) window = max_seq;
  if (sinks > max_seq) sinks = max_seq;
  size_t most = 0;
  auto count = [&](int B, int S) {
    const size_t n = attention_window_scratch_bytes(B, S, nh, nkv, d, window, sinks);
    if (n > most) most = n;
  };
  for (int B = 1; B <= max_batch; ++B)
    for (int S0 = 1; S0 <= max_seq; S0 += 128) {
      const int S1 = max_seq - S0 < 127 ? max_seq : S0 + 127;
      if (S0 <= window && window < S1) count(B, window);
      const int every = S0 > window ? S0 : window + 1;  // the sinks count from here on
      for (int S = every; S <= sinks && S < S1; ++S) count(B, S);
      count(B, S1);
    }
  return most;
}

cudaError_t attention_window_bwd(const bf16* qkv, const bf16* o, const bf16* d_o, const float* lse, bf16* dqkv, const float* cs,
                                 const float* sn, void* scratch, int B, int S, int nh, int nkv, int d, int window, int sinks, int* err,
                                 cudaStream_t st, int* launches) {
  if (!shape_ok(B, S, nh, nkv, d, window, sinks) || !err || (cs == nullptr) != (sn == nullptr)) return cudaErrorInvalidValue;
  clamp_mask(S, window, sinks);
  uint8_t* s = reinterpret_cast<uint8_t*>(scratch);
  int unused = 0;
  int& n = launches != nullptr ? *launches : unused;
  if (block_of(B, S, nh, d, window) == 64) return bwd_t<64, 64>(qkv, o, d_o, lse, dqkv, cs, sn, s, B, S, nh, nkv, window, sinks, err, st, n);
  if (d == 64) return bwd_t<64, 128>(qkv, o, d_o, lse, dqkv, cs, sn, s, B, S, nh, nkv, window, sinks, err, st, n);
  return bwd_t<128, 128>(qkv, o, d_o, lse, dqkv, cs, sn, s, B, S, nh, nkv, window, sinks, err, st, n);
}

}  // namespace fs

// =============================================================================== entry points
namespace {
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}
// bytes of the packed q, k, v (and of their gradients), of o (and dO) and of lse
struct Sizes {
  size_t qkv, o, lse;
  Sizes(int32_t B, int32_t S, int32_t nh, int32_t nkv, int32_t d) {
    const size_t rows = (size_t)B * S;
    qkv = rows * (nh + 2 * nkv) * d * 2;
    o = rows * nh * d * 2;
    lse = rows * nh * 4;
  }
};
ft_status status_of(cudaError_t e) { return e == cudaSuccess ? FT_OK : e == cudaErrorInvalidValue ? FT_EINVAL : FT_ECUDA; }
}  // namespace

extern "C" ft_status ft_k_attention_window_fwd(const void* dev_qkv, void* dev_o, float* dev_lse, int32_t B, int32_t S, int32_t n_heads,
                                               int32_t n_kv_heads, int32_t head_dim, int32_t window, int32_t n_sinks, void* stream) {
  if (!dev_qkv || !dev_o || !dev_lse || !aligned16(dev_qkv) || !aligned16(dev_o) || !aligned4(dev_lse)) return FT_EINVAL;
  if (fs::attention_window_scratch_bytes(B, S, n_heads, n_kv_heads, head_dim, window, n_sinks) == 0) return FT_EINVAL;
  const Sizes n(B, S, n_heads, n_kv_heads, head_dim);
  if (overlap(dev_o, n.o, dev_qkv, n.qkv) || overlap(dev_lse, n.lse, dev_qkv, n.qkv) || overlap(dev_lse, n.lse, dev_o, n.o)) return FT_EINVAL;
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
      !aligned16(dev_sin) || !aligned4(dev_lse) || (reinterpret_cast<uintptr_t>(dev_scratch) & 255u) != 0)
    return FT_EINVAL;
  const size_t need = fs::attention_window_scratch_bytes(B, S, n_heads, n_kv_heads, head_dim, window, n_sinks);
  if (need == 0) return FT_EINVAL;
  if (scratch_bytes < need) return FT_ENOMEM;
  const Sizes n(B, S, n_heads, n_kv_heads, head_dim);
  const size_t table = (size_t)S * (head_dim / 2) * sizeof(float);
  const struct { const void* p; size_t bytes; } inputs[] = {{dev_qkv, n.qkv}, {dev_o, n.o}, {dev_do, n.o}, {dev_lse, n.lse},
                                                            {dev_cos, table}, {dev_sin, table}};
  for (const auto& in : inputs)
    if (in.p && (overlap(dev_dqkv, n.qkv, in.p, in.bytes) || overlap(dev_scratch, need, in.p, in.bytes))) return FT_EINVAL;
  if (overlap(dev_dqkv, n.qkv, dev_scratch, need)) return FT_EINVAL;
  int* status = fs::attention_status_word();
  if (!status) return FT_ECUDA;
  return status_of(fs::attention_window_bwd(
      reinterpret_cast<const fs::bf16*>(dev_qkv), reinterpret_cast<const fs::bf16*>(dev_o), reinterpret_cast<const fs::bf16*>(dev_do),
      dev_lse, reinterpret_cast<fs::bf16*>(dev_dqkv), dev_cos, dev_sin, dev_scratch, B, S, n_heads, n_kv_heads, head_dim, window,
      n_sinks, status, reinterpret_cast<cudaStream_t>(stream)));
}
