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

}  // namespace fs
