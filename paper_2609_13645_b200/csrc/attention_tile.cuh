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
