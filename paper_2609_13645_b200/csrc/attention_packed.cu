// Causal attention inside the documents of a packed batch, forward, on the 5th-generation tensor cores.
//
// Tiles of 128 queries are cut from the packed rows and not from the documents: short documents share tiles instead of leaving them
// half empty, and the number of tiles is known on the host.  Row i sees the rows from its document's first one to itself, so a
// tile streams the 128-key blocks from its first row's document on to its own diagonal.
//
// A CTA, one an SM, works on two tiles at a time: the same queries of two heads, which stream the same K and V if the heads share
// them and each its own if not, or, with an odd number of heads, two neighbouring blocks of queries of a head (each takes part
// only in the blocks it sees).  A tile has its scores S (128 columns, bf16 P
// over the first 64) and its output O in TMEM and four softmax warps, a query row a thread.  While one tile's warps take
// exponentials, the other tile's products run:
//   warp 0      producer: the next work item, Q of both tiles, K and V through rings of TMA copies
//   warp 1      MMA issuer, alternating between the tiles: O_t += P_t V_j (by halves of 64 keys, as P gets ready), S_t = Q_t K_{j+1}^T
//   warps 2-5, 6-9  softmax and output of tile 0, of tile 1
// Two tiles a CTA halve what K and V cost in shared memory, whose bandwidth bounds a CTA of one tile: a pair of blocks of
// 128 x 128 at D = 128 takes 1024 cycles of tensor pipe, of exponential unit and (with shared K and V) of shared memory each.
//
// The grid has a CTA a work item, the longest first; a CTA that has issued all loads of its item takes over the next one that has
// not started (clusterlaunchcontrol), so that the next item's loads go on while the last one ends, and items of any length even out.
//
// T 16384, 4 documents of up to 5622 rows, 16 / 8 heads of 128: 282 us in a short run, 1114 TFLOP/s of visible pairs, and 329 in a long one, whose
// clock the power cap lowers; the tensor pipe is 57 % and the exponential unit 58 % busy.  What bounds it is each tile's chain of about 3600 cycles a block: scores to registers 200, maxima 200,
// exponentials 1100, P to TMEM 150, then P V and the next S on the tensor cores, behind the other tile's (1100 and 650 of latencies); TMEM is
// full, so the next S cannot be formed before P V has read P.  Measured beside it, in short runs when this took 277: two warps a row with 64 keys each 338 us (twice
// the instructions around the exponentials), blocks of 64 keys with two score buffers a tile 359, the exponentials taken
// speculatively in one pass of 64 keys 337; with 12 heads of 64 the same.
#include <limits.h>
#include <math.h>

#include "attention.cuh"
#include "attention_tile.cuh"
#include "attention_window.cuh"
#include "tmap.cuh"

namespace fs {
namespace {

constexpr int THREADS = 320;
constexpr int kOrdered = 256;  // blocks of queries of a head (or pairs of them), at most, that are taken in the order of their lengths

template <int D>
struct Cfg {
  static constexpr int KC = D / 64;
  static constexpr int NK = D == 64 ? 4 : 2, NV = NK;
  static constexpr int Q_BYTES = 128 * D * 2, KV_BYTES = 128 * D * 2;
  static constexpr int OFF_K = 2 * Q_BYTES, OFF_V = OFF_K + NK * KV_BYTES;
  static constexpr int OFF_OUT = OFF_V + NV * KV_BYTES;  // 32 rows of 64 columns a softmax warp
  static constexpr int OFF_BAR = OFF_OUT + 8 * 4096;
  static constexpr int SMEM_BYTES = OFF_BAR + 512;
  static constexpr int TMEM_COLS = 512, O_COL = 256;  // S of tile t from column 128 t, O from 256 + 128 t
};
static_assert(Cfg<128>::SMEM_BYTES <= 232448, "shared memory of one SM");

enum { P_QFULL = 0, P_QEMPTY = 2, P_KFULL = 4, P_KEMPTY = 8, P_VFULL = 12, P_VEMPTY = 16, P_SFULL = 20, P_PFULL = 22, P_ODONE = 26,
       P_OFINAL = 28, P_OEMPTY = 30, P_INFO = 32, P_INFOEMPTY = 34, P_NEXT = 36, P_TAIL = 37, P_COUNT = 38 };

// What a work item is: the head and first query of each tile and the 128-key blocks [first, end) that it sees (none: an idle tile);
// split: the tiles' heads have K and V of their own (and see the same blocks).
struct Item {
  int valid, split, head[2], q0[2], first[2], end[2];
};

// Bit e: key e of 32 is seen, given that keys lo <= e <= hi are.
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t visible(int hi, int lo) { return below(hi + 1) & ~below(lo); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Hands over an item of the grid that has not started: 16 bytes of answer, counted on the barrier.
__device__ __forceinline__ void ask_next(uint32_t answer, uint32_t bar) {
  mbar_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
__device__ __forceinline__ int read_next(uint32_t answer) {  // -1: there is none left
  uint32_t got, x;
  asm volatile(
      "{\n .reg .b128 a;\n .reg .pred p;\n ld.shared.b128 a, [%2];\n"
      " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n selp.u32 %0, 1, 0, p;\n mov.u32 %1, 0;\n"
      " @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, a;\n}"
      : "=r"(got), "=r"(x) : "r"(answer) : "memory");
  fence_proxy_async_smem();  // the next answer is written behind this read
  return got != 0 ? (int)x : -1;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
attn_packed_fwd_kernel(const __grid_constant__ CUtensorMap tm_qkv, const __grid_constant__ CUtensorMap tm_out, bf16* __restrict__ o,
                       float* __restrict__ lse, int T, int n_heads, int n_kv, int n_qblocks, int by_head, const __grid_constant__ Docs docs,
                       float scale_log2, int* err) {
  using C = Cfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  const uint32_t bar0 = sbase + C::OFF_BAR;
  auto bar = [&](int i) { return bar0 + 8u * i; };
  Item* items = reinterpret_cast<Item*>(bars + P_COUNT);  // two, in turn
  constexpr int AFTER = (8 * P_COUNT + 2 * sizeof(Item) + 15) / 16 * 16;
  static_assert(AFTER % 16 == 0 && AFTER + 16 + 8 <= 512, "the answer is aligned, and all of it fits");
  const uint32_t answer = bar0 + AFTER;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_BAR + AFTER + 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if ((sbase & 1023u) != 0u) {  // the swizzled tiles need a 1024-byte aligned base
    if (threadIdx.x == 0) atomicExch(err, (int)ERR_BAD_ALIGNMENT);
    return;
  }
  const int hq = n_heads * D, hkv = n_kv * D, n_rep = n_heads / n_kv;
  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(bar(P_QFULL + t), 1);
      mbar_init(bar(P_QEMPTY + t), 1);
      mbar_init(bar(P_SFULL + t), 1);
      mbar_init(bar(P_PFULL + 2 * t), 4);
      mbar_init(bar(P_PFULL + 2 * t + 1), 4);
      mbar_init(bar(P_ODONE + t), 1);
      mbar_init(bar(P_OFINAL + t), 1);
      mbar_init(bar(P_OEMPTY + t), 4);
      mbar_init(bar(P_INFO + t), 1);
      mbar_init(bar(P_INFOEMPTY + t), 9);  // the MMA warp and the softmax warps
    }
    for (int i = 0; i < C::NK; ++i) {
      mbar_init(bar(P_KFULL + i), 1);
      mbar_init(bar(P_KEMPTY + i), 1);
      mbar_init(bar(P_VFULL + i), 1);
      mbar_init(bar(P_VEMPTY + i), 1);
    }
    mbar_init(bar(P_NEXT), 1);
    mbar_init(bar(P_TAIL), 1);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_qkv);
    tma_prefetch_desc(&tm_out);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();  // set-up done; from here on the kernel touches what its predecessor wrote
  // items: the same queries of two heads, or two blocks of queries of one; a place of the order of lengths is a block (or two)
  const int per = by_head ? n_heads / 2 : n_heads, places = by_head ? n_qblocks : (n_qblocks + 1) / 2, rows = by_head ? 128 : 256;
  const bool ordered = places <= kOrdered;
  Ordered<kOrdered> order{};
  if (ordered && warp == 0) order.read(places, lane, [&](int i) { return __ldg(docs.start + i * rows); });
  const int e_last = __ldg(docs.end + T - 1), rows_end = e_last < 0 ? 0 : e_last < T ? e_last : T;  // rows behind it are nobody's

  // The item that consumers work on next: waits for it, takes it over and gives its place back.
  auto take = [&](int k, Item& it, int site) {
    bool ok = mbar_wait(bar(P_INFO + (k & 1)), ((uint32_t)k >> 1) & 1u, abort_flag, err, kWaitLimitCycles, site);
    ok = __all_sync(0xffffffffu, ok);
    if (ok) {
      it = items[k & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(P_INFOEMPTY + (k & 1)));
    }
    return ok && it.valid != 0;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    int index = (int)blockIdx.x, kcount = 0, qcount[2] = {0, 0};
    uint32_t tail_parity = 0;
    bool ok = true;
    auto wait_all = [&](int i, uint32_t parity, int site) {
      const bool got = mbar_wait(bar(i), parity, abort_flag, err, kWaitLimitCycles, site);
      return __all_sync(0xffffffffu, got) != 0;
    };
    if (ordered)
      order.measure(places, lane, [&](int i, int start) {
        const int row = i * rows;
        return row < rows_end ? (min(row + rows, rows_end) + 127) / 128 - (min(max(start, 0), row) >> 7) : 0;
      });
    for (int k = 0; ok; ++k) {
      Item it;
      it.valid = index >= 0;
      const int rank = index / per, which = index % per;
      int place = places - 1 - rank;
      if (ordered && it.valid) {
        order.find(places, rank, lane);
        place = order.tile;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        it.head[t] = by_head ? 2 * which + t : which;
        it.q0[t] = place * rows + t * (rows - 128);
        it.first[t] = it.end[t] = 0;
        if (it.valid && it.q0[t] < rows_end) {
          const int a = __ldg(docs.start + it.q0[t]);
          it.first[t] = min(max(a, 0), it.q0[t]) >> 7;
          it.end[t] = (it.q0[t] >> 7) + 1;
        }
      }
      it.split = by_head && it.head[0] / n_rep != it.head[1] / n_rep;
      if (!(ok = wait_all(P_INFOEMPTY + (k & 1), (((uint32_t)k >> 1) & 1u) ^ 1u, 0xa1))) break;
      if (lane == 0) {
        items[k & 1] = it;
        mbar_arrive(bar(P_INFO + (k & 1)));
      }
      if (!it.valid) break;
      // blocks of both tiles, an idle one aside
      const bool use0 = it.end[0] > 0, use1 = it.end[1] > 0;
      const int b0 = use0 && use1 ? min(it.first[0], it.first[1]) : use0 ? it.first[0] : it.first[1];
      const int b1 = max(it.end[0], it.end[1]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (it.end[t] == 0) continue;
        if (!(ok = wait_all(P_QEMPTY + t, ((uint32_t)qcount[t] & 1u) ^ 1u, 0xa2))) break;
        ++qcount[t];
        if (lane == 0) {
          mbar_expect_tx(bar(P_QFULL + t), C::Q_BYTES);
#pragma unroll
          for (int kc = 0; kc < C::KC; ++kc)
            tma_load_3d(sbase + t * C::Q_BYTES + kc * 16384, &tm_qkv, bar(P_QFULL + t), it.head[t] * D + kc * 64, it.q0[t], 0);
        }
      }
      // K of a block, for both tiles or for each, then V
      for (int j = b0; j < b1 && ok; ++j) {
        for (int e = 0; e <= it.split && ok; ++e) {
          const int st = (kcount + e) % C::NK;
          if (!(ok = wait_all(P_KEMPTY + st, ((uint32_t)((kcount + e) / C::NK) & 1u) ^ 1u, 0xa3))) break;
          if (lane == 0) {
            mbar_expect_tx(bar(P_KFULL + st), C::KV_BYTES);
#pragma unroll
            for (int kc = 0; kc < C::KC; ++kc)
              tma_load_3d(sbase + C::OFF_K + st * C::KV_BYTES + kc * 16384, &tm_qkv, bar(P_KFULL + st), hq + it.head[e] / n_rep * D + kc * 64, j * 128, 0);
          }
        }
        for (int e = 0; e <= it.split && ok; ++e, ++kcount) {
          const int st = kcount % C::NV;
          if (!(ok = wait_all(P_VEMPTY + st, ((uint32_t)(kcount / C::NV) & 1u) ^ 1u, 0xa4))) break;
          // a block that reaches behind the last document: its V arrives on a barrier of its own and loses those rows first
          const bool tail = j * 128 + 128 > rows_end;
          const uint32_t v = sbase + C::OFF_V + st * C::KV_BYTES, full = bar(tail ? P_TAIL : P_VFULL + st);
          if (lane == 0) {
            mbar_expect_tx(full, C::KV_BYTES);
#pragma unroll
            for (int kc = 0; kc < C::KC; ++kc)
              tma_load_3d(v + kc * 16384, &tm_qkv, full, hq + hkv + it.head[e] / n_rep * D + kc * 64, j * 128, 0);
          }
          if (tail) {
            if (!(ok = wait_all(P_TAIL, tail_parity, 0xa5))) break;
            tail_parity ^= 1u;
            zero_rows<D, 128>(v, rows_end - j * 128, lane);
            if (lane == 0) mbar_arrive(bar(P_VFULL + st));
          }
        }
      }
      if (!ok) break;
      // not before all loads are on their way: an item that is taken over early waits here while another CTA has nothing to do
      if (lane == 0) ask_next(answer, bar(P_NEXT));
      if (!(ok = wait_all(P_NEXT, (uint32_t)k & 1u, 0xa6))) break;
      index = read_next(answer);
      __syncwarp();
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    const uint32_t elected = elect_one();
    const uint32_t idesc_base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);
    const uint32_t idesc_s = idesc_base | ((uint32_t)(128 >> 3) << 17);              // N = 128 keys, both K-major
    const uint32_t idesc_pv = idesc_base | (1u << 16) | ((uint32_t)(D >> 3) << 17);  // N = D, B (V) mn-major
    auto wait_all = [&](int i, uint32_t parity, int site) {
      const bool got = mbar_wait(bar(i), parity, abort_flag, err, kWaitLimitCycles, site);
      return __all_sync(0xffffffffu, got) != 0;
    };
    int kcount = 0, pcount[2] = {0, 0}, icount[2] = {0, 0};
    bool ok = true;
    Item it;
    for (int k = 0; ok && take(k, it, 0xb1); ++k) {
      const bool use0 = it.end[0] > 0, use1 = it.end[1] > 0;
      const int b0 = use0 && use1 ? min(it.first[0], it.first[1]) : use0 ? it.first[0] : it.first[1];
      const int b1 = max(it.end[0], it.end[1]);
      auto sees = [&](int t, int j) { return j >= it.first[t] && j < it.end[t]; };
      // Scores of tile t against the kc-th K block.  (Its second 64 keys, whose columns P leaves alone, ahead of the second half of P V: 333 us
      // at T 16384 where this takes 301; 64 columns take the tensor cores as long as 128.)
      auto scores = [&](int t, int kc) {
        tc_fence_after();
        const uint64_t dq = umma_desc_sw128(sbase + t * C::Q_BYTES, 0, 1024);
        const uint64_t dk = umma_desc_sw128(sbase + C::OFF_K + kc % C::NK * C::KV_BYTES, 0, 1024);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const uint64_t off = (uint64_t)(((i >> 2) * 16384 + (i & 3) * 32) >> 4);
          umma_bf16_if(elected, tmem_base + 128u * t, dq + off, dk + off, idesc_s, i > 0 ? 1u : 0u);
        }
      };
      auto wait_k = [&](int t, int j, int kc) {
        return (j != it.first[t] || wait_all(P_QFULL + t, (uint32_t)icount[t] & 1u, 0xb2)) &&
               wait_all(P_KFULL + kc % C::NK, (uint32_t)(kc / C::NK) & 1u, 0xb3);
      };
      auto scores_done = [&](int t, int j, int kc) {
        umma_commit_if(elected, bar(P_SFULL + t));
        if (it.split) umma_commit_if(elected, bar(P_KEMPTY + kc % C::NK));
        if (j + 1 == it.end[t]) umma_commit_if(elected, bar(P_QEMPTY + t));
      };
      const int step = 1 + it.split;
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (ok && sees(t, b0)) {
          const int kc = kcount + (it.split ? t : 0);
          if (!(ok = wait_k(t, b0, kc))) break;
          scores(t, kc);
          scores_done(t, b0, kc);
        }
      if (ok && b1 > b0 && !it.split) umma_commit_if(elected, bar(P_KEMPTY + kcount % C::NK));
      for (int j = b0; j < b1 && ok; ++j, kcount += step) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int vc = kcount + (it.split ? t : 0), st = vc % C::NV, next = vc + step;
          const bool more = j + 1 < b1 && sees(t, j + 1), now = sees(t, j);
          if (now) {
            const bool first = j == it.first[t];
            if (!(ok = wait_all(P_VFULL + st, (uint32_t)(vc / C::NV) & 1u, 0xb4))) break;
            if (first && !(ok = wait_all(P_OEMPTY + t, ((uint32_t)icount[t] & 1u) ^ 1u, 0xb5))) break;
            const uint64_t dv = umma_desc_sw128(sbase + C::OFF_V + st * C::KV_BYTES, 16384, 1024);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (!(ok = wait_all(P_PFULL + 2 * t + h, (uint32_t)pcount[t] & 1u, 0xb6))) break;
              tc_fence_after();
#pragma unroll
              for (int i = 0; i < 4; ++i)  // bf16 P: 16 keys = 8 columns
                umma_bf16_ts_if(elected, tmem_base + (uint32_t)(C::O_COL + 128 * t), tmem_base + (uint32_t)(128 * t + 32 * h + 8 * i),
                                dv + (uint64_t)(((4 * h + i) * 2048) >> 4), idesc_pv, first && h == 0 && i == 0 ? 0u : 1u);
            }
            if (!ok) break;
            umma_commit_if(elected, bar(P_ODONE + t));
            if (it.split) umma_commit_if(elected, bar(P_VEMPTY + st));
            ++pcount[t];
            if (j + 1 == it.end[t]) umma_commit_if(elected, bar(P_OFINAL + t));
          }
          if (more) {
            if (!(ok = wait_k(t, j + 1, next))) break;
            scores(t, next);
            scores_done(t, j + 1, next);
          }
        }
        if (!ok) break;
        if (!it.split) {
          umma_commit_if(elected, bar(P_VEMPTY + kcount % C::NV));
          if (j + 1 < b1) umma_commit_if(elected, bar(P_KEMPTY + (kcount + 1) % C::NK));
        }
      }
      icount[0] += use0;
      icount[1] += use1;
    }
  } else {
    // ------------------------------------------------------------------ softmax warps: one query row a thread = TMEM lane
    const int t = (warp - 2) >> 2, q = warp & 3;
    const uint32_t tlane = tmem_base + ((uint32_t)(q * 32) << 16);
    const uint32_t t_s = tlane + (uint32_t)(128 * t), t_o = tlane + (uint32_t)(C::O_COL + 128 * t);
    const uint32_t stage = sbase + (uint32_t)(C::OFF_OUT + (warp - 2) * 4096);
    uint32_t blocks = 0, icount = 0;  // blocks so far, items in which the tile took part
    bool ok = true;
    Item it;
    for (int k = 0; ok && take(k, it, 0xc1); ++k) {
      const int b_first = t == 0 ? it.first[0] : it.first[1], b_end = t == 0 ? it.end[0] : it.end[1], q0 = t == 0 ? it.q0[0] : it.q0[1];
      const int head = t == 0 ? it.head[0] : it.head[1];
      if (b_end == 0) continue;
      const int row = q0 + q * 32 + lane, wmin = q0 + q * 32;
      int own = T;  // first row of this row's document
      if (row < rows_end) own = min(max(__ldg(docs.start + row), 0), row);
      const int own_max = __shfl_sync(0xffffffffu, own, 31);
      // The row reference is an integer in the log2 domain: any such reference gives the same softmax, and bf16 rounding commutes with
      // powers of two.  It moves only if a block's maximum turns out more than 2^kRefSlack above it (or, for a row that has seen nothing, far
      // below it).
      // lsum is the sum of the exponentials; o is divided by nsum, in which blocks on an edge of the mask count with their rounded P:
      // the weights of a row that sees few keys then add up to 1, and a row that sees one key returns its value.
      float mref = 0.f, lsum = 0.f, nsum = 0.f;
      for (int j = b_first; j < b_end; ++j) {
        ok = mbar_wait(bar(P_SFULL + t), blocks & 1u, abort_flag, err, kWaitLimitCycles, 0xc2);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ++blocks;
        tc_fence_after();
        const int first = j * 128;
        // only blocks on an edge of the mask are tested key by key
        const bool all = first + 127 <= wmin && first >= own_max;
        uint32_t r[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(t_s + 32u * c, r[c]);
        tmem_ld_wait();
        if (!all) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t seen = visible(row - first - 32 * c, own - first - 32 * c);
#pragma unroll
            for (int e = 0; e < 32; ++e) r[c][e] = seen & (1u << e) ? r[c][e] : 0xff800000u;  // -inf
          }
        }
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; e += 2) m4[e >> 1 & 3] = max3(m4[e >> 1 & 3], __uint_as_float(r[c][e]), __uint_as_float(r[c][e + 1]));
        const float mx = max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]);
        const float mcand = ceilf(mx * scale_log2);  // scale_log2 > 0: the maximum commutes with it
        const bool move = mcand > mref + kRefSlack || (lsum == 0.f && mx > -INFINITY && mcand < mref - 2.f * kRefSlack);
        if (__any_sync(0xffffffffu, move)) {
          const float alpha = move && lsum > 0.f ? fast_exp2(mref - mcand) : 1.0f;  // an exact power of two
          if (move) mref = mcand;
          lsum *= alpha;
          nsum *= alpha;
          if (__any_sync(0xffffffffu, alpha != 1.0f)) {  // rescale O, behind the previous product
            ok = mbar_wait(bar(P_ODONE + t), (blocks - 2u) & 1u, abort_flag, err, kWaitLimitCycles, 0xc3);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t x[32];
              tmem_ld32(t_o + (uint32_t)c, x);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * alpha);
              tmem_st32(t_o + (uint32_t)c, x);
            }
          }
        }
        float2 psum[4] = {both(0.f), both(0.f), both(0.f), both(0.f)}, rsum = both(0.f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t pw[32];  // bf16 pairs: keys 2c, 2c+1 in word c
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            const float2 x = fma2(make_float2(__uint_as_float(r[2 * h + (e >> 5)][e & 31]), __uint_as_float(r[2 * h + (e >> 5)][(e & 31) + 1])),
                                  both(scale_log2), both(-mref));
            const float2 a = make_float2(fast_exp2(x.x), fast_exp2(x.y));
            psum[e >> 1 & 3] = add2(psum[e >> 1 & 3], a);
            pw[e >> 1] = pack_bf16(a.x, a.y);
          }
          tmem_st32(t_s + 32u * h, pw);  // over scores that are in registers
          if (!all) {
#pragma unroll
            for (int e = 0; e < 32; ++e) rsum = add2(rsum, make_float2(bf16_lo(pw[e]), bf16_hi(pw[e])));
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(P_PFULL + 2 * t + h));
        }
        psum[0] = add2(add2(psum[0], psum[1]), add2(psum[2], psum[3]));
        const float block_sum = psum[0].x + psum[0].y;
        lsum += block_sum;
        nsum += all ? block_sum : rsum.x + rsum.y;
      }
      if (ok) {
        ok = mbar_wait(bar(P_OFINAL + t), icount & 1u, abort_flag, err, kWaitLimitCycles, 0xc4);
        ok = __all_sync(0xffffffffu, ok);
      }
      if (!ok) break;
      ++icount;
      tc_fence_after();
      const float inv = 1.0f / nsum;
      if (row < rows_end) lse[(long long)head * T + row] = (mref + log2f(lsum)) * kLn2;
#pragma unroll 1
      for (int c = 0; c < C::KC; ++c) {
        if (lane == 0) bulk_wait_group_read0();  // what was staged last has left
        __syncwarp();
        stage_rows<64>(stage, lane, t_o + (uint32_t)(64 * c), inv);
        if (c + 1 == C::KC) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(P_OEMPTY + t));
        }
        send_rows_clipped<64>(&tm_out, o, hq, stage, lane, head * D + 64 * c, wmin, rows_end);
      }
      __syncwarp();
    }
    if (lane == 0) bulk_wait_group0();
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
cudaError_t fwd_t(const bf16* qkv, bf16* o, float* lse, const Docs& docs, int T, int nh, int nkv, int* err, cudaStream_t st) {
  using C = Cfg<D>;
  static unsigned long long smem_set = 0;
  cudaError_t e = ensure_dynamic_smem(attn_packed_fwd_kernel<D>, C::SMEM_BYTES, smem_set);
  if (e != cudaSuccess) return e;
  const int nqkv = (nh + 2 * nkv) * D;
  CUtensorMap tm_qkv, tm_out;
  if (!make_tmap_3d(&tm_qkv, qkv, nqkv, T, 1, nqkv, 128) || !make_tmap_3d(&tm_out, o, nh * D, T, 1, nh * D, 32)) return cudaErrorInvalidValue;
  const float scale_log2 = (float)((1.0 / sqrt((double)D)) * 1.4426950408889634);
  // Heads of 128 have room for one K and one V block a tile where each tile has its own: neighbouring queries share them instead.
  const int nqb = (T + 127) / 128, by_head = D == 64 ? nh % 2 == 0 : nh / nkv % 2 == 0;
  const long long items = by_head ? (long long)nqb * (nh / 2) : (long long)(nqb + 1) / 2 * nh;
  return launch_pdl(attn_packed_fwd_kernel<D>, dim3((unsigned)items), dim3(THREADS), C::SMEM_BYTES, st, tm_qkv, tm_out, o, lse, T, nh, nkv, nqb,
                    by_head, docs, scale_log2, err);
}

}  // namespace

cudaError_t attention_packed_fwd(const bf16* qkv, bf16* o, float* lse, const Docs& docs, int T, int nh, int nkv, int d, int* err, cudaStream_t st) {
  if (attention_packed_scratch_bytes(T, nh, nkv, d, 1) == 0 || !err) return cudaErrorInvalidValue;
  // Two tiles a CTA from six tiles an SM on; below, a CTA's start and end count, and two small ones an SM hide each other's.  us for
  // documents of 300 / 1000 / 4000 on average, in brackets with one tile a CTA:
  //   16 / 8 heads of 128   T 2048: 16.8 36.1 37.3 (15.2 26.9 29.5);  T 6144: 33.7 45.8 83.3 (32.9 47.4 85.2);  T 16384: 70 104 269 (78 113 291)
  //   12 heads of 64        T 2048: 15.8 33.8 33.7 (11.9 25.2 26.9);  T 8192: 29.7 42.6 98.6 (28.9 43.3 98.8);  T 16384: 52 76 178 (54 81 193)
  // With pairs of neighbouring blocks of queries (7 heads of 64 on one, T 20000) short documents lose, 41.5 (36.3) at 200, and longer ones
  // gain, 61 (68) and 135 (157); the host, which chooses, does not know the lengths.
  if ((long long)((T + 127) / 128) * nh < 6 * 148) return attention_packed_fwd_tile(qkv, o, lse, docs, T, nh, nkv, d, err, st);
  if (d == 64) return fwd_t<64>(qkv, o, lse, docs, T, nh, nkv, err, st);
  return fwd_t<128>(qkv, o, lse, docs, T, nh, nkv, err, st);
}

}  // namespace fs
