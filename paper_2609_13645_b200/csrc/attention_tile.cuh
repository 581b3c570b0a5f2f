// Pieces shared by the attention kernels on the tensor cores: TMEM rows to registers, rows of bf16 to memory.
#pragma once
#include "common.cuh"

namespace fs {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRefSlack = 8.0f;  // a softmax row's integer reference moves once the maximum has passed it by 2^8

__device__ __forceinline__ void store8_b32(void* dst, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

template <int W>
__device__ __forceinline__ void tmem_load_cols(uint32_t taddr, float (&out)[W]) {
  static_assert(W == 32 || W == 16, "chunk width");
  if constexpr (W == 32) {
    uint32_t t[32];
    tmem_ld32(taddr, t);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 32; ++i) out[i] = __uint_as_float(t[i]);
  } else {
    uint32_t t[16];
    tmem_ld16(taddr, t);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) out[i] = __uint_as_float(t[i]);
  }
}

template <int W>
__device__ __forceinline__ void store_bf16_row(bf16* dst, const float (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 8) {
    uint4 o;
    o.x = pack_bf16(v[i], v[i + 1]);
    o.y = pack_bf16(v[i + 2], v[i + 3]);
    o.z = pack_bf16(v[i + 4], v[i + 5]);
    o.w = pack_bf16(v[i + 6], v[i + 7]);
    *reinterpret_cast<uint4*>(dst + i) = o;
  }
}

// Backward of the rotation: its transpose, on pairs (i, i + d/2) of one row; cs, sn: the row's tables from column i on.
template <int W>
__device__ __forceinline__ void unrotate(float (&lo)[W], float (&hi)[W], const float* cs, const float* sn) {
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

// ---- output rows of a warp (thread = row, 32 rows of D columns in TMEM) on their way to memory.  They are staged in shared
// memory as D / 64 boxes of [32 rows][64 columns] bf16 under the 128-byte swizzle and leave as tensor stores of full
// lines, clipped at the end of the sequence.  (A thread that stores its own row, and reads its own row of the rotation tables,
// touches 32 lines an instruction: 13000 cycles for a 128 x 128 tile with rotation, a sixth of the dK/dV kernel.)
__device__ __forceinline__ void tma_store_3d(const void* tmap, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(tmap), "r"(src), "r"(x), "r"(y),
               "r"(z) : "memory");
}
// 8 columns from `col` on of row `lane` (16 bytes)
__device__ __forceinline__ void stage_piece(uint32_t out, int lane, int col, uint4 v) {
  st_shared_v4(out + (uint32_t)((col >> 6) * 4096 + lane * 128 + ((((col & 63) >> 3) ^ (lane & 7)) * 16)), v);
}
template <int W>
__device__ __forceinline__ void stage_cols(uint32_t out, int lane, int col, const float (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 8)
    stage_piece(out, lane, col + i, make_uint4(pack_bf16(v[i], v[i + 1]), pack_bf16(v[i + 2], v[i + 3]), pack_bf16(v[i + 4], v[i + 5]),
                                               pack_bf16(v[i + 6], v[i + 7])));
}
template <int D>
__device__ __forceinline__ void stage_rows(uint32_t out, int lane, uint32_t tmem_row, float scale) {
#pragma unroll 1
  for (int c = 0; c < D; c += 32) {
    float v[32];
    tmem_load_cols<32>(tmem_row + (uint32_t)c, v);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] *= scale;
    stage_cols<32>(out, lane, c, v);
  }
}
// The same for rows that are rotated back by the tables cs, sn (fp32 [S, D / 2]; row0: position of the warp's first row).
// 16 columns of the warp's 32 table rows at a time are read in whole 64-byte runs into `table` (4 KB of the warp's own: a row
// of 64 bytes each, its 16-byte pieces xor-ed with bits of the row against bank conflicts) and from there by row.
template <int D>
__device__ __forceinline__ void stage_rows_unrotated(uint32_t out, uint32_t table, int lane, uint32_t tmem_row, float scale,
                                                     const float* __restrict__ cs, const float* __restrict__ sn, int row0, int S) {
  constexpr int H = D / 2;
  float4 c4[4], s4[4];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long at = (long long)min(row0 + k * 8 + (lane >> 2), S - 1) * H + i0 + (lane & 3) * 4;
      c4[k] = *reinterpret_cast<const float4*>(cs + at);
      s4[k] = *reinterpret_cast<const float4*>(sn + at);
    }
  };
  auto slot = [&](int row, int piece) { return table + (uint32_t)(row * 64 + ((piece ^ ((row >> 1) & 3)) * 16)); };
  fetch(0);
#pragma unroll 1
  for (int i0 = 0; i0 < H; i0 += 16) {
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = k * 8 + (lane >> 2);
      st_shared_v4(slot(r, lane & 3), make_uint4(__float_as_uint(c4[k].x), __float_as_uint(c4[k].y), __float_as_uint(c4[k].z), __float_as_uint(c4[k].w)));
      st_shared_v4(slot(r, lane & 3) + 2048, make_uint4(__float_as_uint(s4[k].x), __float_as_uint(s4[k].y), __float_as_uint(s4[k].z), __float_as_uint(s4[k].w)));
    }
    if (i0 + 16 < H) fetch(i0 + 16);
    float lo[16], hi[16];
    tmem_load_cols<16>(tmem_row + (uint32_t)i0, lo);
    tmem_load_cols<16>(tmem_row + (uint32_t)(H + i0), hi);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint4 c = ld_shared_v4(slot(lane, k)), s = ld_shared_v4(slot(lane, k) + 2048);
      const uint32_t cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float y1 = lo[4 * k + u] * scale, y2 = hi[4 * k + u] * scale;
        const float co = __uint_as_float(cc[u]), si = __uint_as_float(ss[u]);
        lo[4 * k + u] = y1 * co + y2 * si;
        hi[4 * k + u] = y2 * co - y1 * si;
      }
    }
    stage_cols<16>(out, lane, i0, lo);
    stage_cols<16>(out, lane, H + i0, hi);
  }
}
// Sends the staged rows off: D columns from x on, 32 rows from y on of batch row z.
template <int D>
__device__ __forceinline__ void send_rows(const void* tmap, uint32_t out, int lane, int x, int y, int z, int S) {
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0 && y < S) {
#pragma unroll
    for (int c = 0; c < D / 64; ++c) tma_store_3d(tmap, out + (uint32_t)(c * 4096), x + 64 * c, y, z);
    bulk_commit_group();
  }
}

// Untiled bulk copies (both addresses and the size multiples of 16 bytes).
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}

// MMA issue from code that the whole warp runs: the operands stay warp-uniform and one elected lane issues.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t e;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
  return e;
}
__device__ __forceinline__ void umma_bf16_if(uint32_t elected, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 e, %5, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(elected)
      : "memory");
}
__device__ __forceinline__ void umma_bf16_ts_if(uint32_t elected, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                                uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 e, %5, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(elected)
      : "memory");
}
__device__ __forceinline__ void umma_commit_if(uint32_t elected, uint32_t bar) {
  asm volatile(
      "{\n .reg .pred e;\n setp.ne.b32 e, %1, 0;\n"
      " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(elected)
      : "memory");
}

}  // namespace fs
