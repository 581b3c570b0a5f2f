// Packed batches: documents of any length one behind the other in one buffer of T rows.  The bounds of every row's document
// (computed once a batch, read by every layer's attention and by the rotation) and the entry points of the attention inside them,
// whose kernels are instances of the windowed ones.
#include "../../include/forgestep.h"
#include "attention.cuh"
#include "attention_window.cuh"

namespace fs {
namespace {

// bounds [3][T]: first row of the row's document, the row behind its last, position in it.  A row takes a binary search in the
// offsets, whose few lines stay in L1.  Offsets that do not ascend from 0 to at most T, or a document longer than `longest`, are
// reported in the status word; the bounds stay within [0, T] whatever the offsets hold.
__global__ void __launch_bounds__(256)
packed_bounds_kernel(const int* __restrict__ cu, int n, int T, int longest, int* __restrict__ bounds, int* err) {
  pdl_trigger();
  pdl_wait();
  const int t = (int)(blockIdx.x * 256 + threadIdx.x);
  const int total = n > 0 ? min(max(__ldg(cu + n), 0), T) : 0;  // no documents: nobody's rows, whatever the one offset holds
  if (t < T) {
    int start = T, end = total, pos = 0;
    if (t < total) {
      int lo = 0, hi = n;  // the first offset beyond t lies in (lo, hi]
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(cu + mid + 1) > t) hi = mid;
        else lo = mid + 1;
      }
      const int i = min(lo, n - 1);
      start = min(max(__ldg(cu + i), 0), t);
      end = min(max(__ldg(cu + i + 1), t + 1), total);
      pos = t - start;
    }
    bounds[t] = start;
    bounds[(long long)T + t] = end;
    bounds[2ll * T + t] = pos;
  }
  bool bad = t == 0 && (__ldg(cu) != 0 || __ldg(cu + n) > T);
  for (long long i = t; i < n; i += (long long)gridDim.x * 256) {
    const long long len = (long long)__ldg(cu + i + 1) - __ldg(cu + i);
    bad = bad || len < 0 || len > longest;
  }
  if (bad) atomicCAS(err, (int)ERR_NONE, (int)ERR_BAD_INDEX);
}

}  // namespace
}  // namespace fs

namespace {
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}
ft_status status_of(cudaError_t e) { return e == cudaSuccess ? FT_OK : e == cudaErrorInvalidValue ? FT_EINVAL : FT_ECUDA; }
struct Sizes {
  size_t qkv, o, lse, bounds;
  Sizes(int32_t T, int32_t nh, int32_t nkv, int32_t d) {
    qkv = (size_t)T * (nh + 2 * nkv) * d * 2;
    o = (size_t)T * nh * d * 2;
    lse = (size_t)T * nh * 4;
    bounds = (size_t)T * 12;
  }
};
fs::Docs docs_of(const int32_t* bounds, int32_t T) { return fs::Docs{bounds, bounds + T, bounds + 2 * (size_t)T}; }
}  // namespace

extern "C" ft_status ft_k_packed_bounds(const int32_t* dev_offsets, int32_t n_docs, int32_t T, int32_t longest, int32_t* dev_bounds,
                                        void* stream) {
  if (!dev_offsets || !dev_bounds || n_docs < 0 || n_docs == INT32_MAX || T <= 0 || T > (1 << 28) || longest < 1) return FT_EINVAL;
  if (!aligned(dev_offsets, 4) || !aligned(dev_bounds, 4)) return FT_EINVAL;
  if (overlap(dev_offsets, ((size_t)n_docs + 1) * 4, dev_bounds, (size_t)T * 12)) return FT_EINVAL;
  int* status = fs::attention_status_word();
  if (!status) return FT_ECUDA;
  return status_of(fs::launch_pdl(fs::packed_bounds_kernel, dim3((unsigned)((T + 255) / 256)), dim3(256), 0, reinterpret_cast<cudaStream_t>(stream),
                                  (const int*)dev_offsets, n_docs, T, longest, (int*)dev_bounds, status));
}

extern "C" ft_status ft_k_attention_packed_fwd(const void* dev_qkv, void* dev_o, float* dev_lse, const int32_t* dev_bounds, int32_t T,
                                               int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, void* stream) {
  if (!dev_qkv || !dev_o || !dev_lse || !dev_bounds) return FT_EINVAL;
  if (!aligned(dev_qkv, 16) || !aligned(dev_o, 16) || !aligned(dev_lse, 4) || !aligned(dev_bounds, 4)) return FT_EINVAL;
  if (fs::attention_packed_scratch_bytes(T, n_heads, n_kv_heads, head_dim, 1) == 0) return FT_EINVAL;
  const Sizes n(T, n_heads, n_kv_heads, head_dim);
  if (overlap(dev_o, n.o, dev_qkv, n.qkv) || overlap(dev_lse, n.lse, dev_qkv, n.qkv) || overlap(dev_lse, n.lse, dev_o, n.o) ||
      overlap(dev_o, n.o, dev_bounds, n.bounds) || overlap(dev_lse, n.lse, dev_bounds, n.bounds))
    return FT_EINVAL;
  int* status = fs::attention_status_word();
  if (!status) return FT_ECUDA;
  return status_of(fs::attention_packed_fwd(reinterpret_cast<const fs::bf16*>(dev_qkv), reinterpret_cast<fs::bf16*>(dev_o), dev_lse,
                                            docs_of(dev_bounds, T), T, n_heads, n_kv_heads, head_dim, status,
                                            reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" size_t ft_k_attention_packed_scratch_bytes(int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t longest) {
  return fs::attention_packed_scratch_bytes(T, n_heads, n_kv_heads, head_dim, longest);
}

extern "C" ft_status ft_k_attention_packed_bwd(const void* dev_qkv, const void* dev_o, const void* dev_do, const float* dev_lse,
                                               void* dev_dqkv, const int32_t* dev_bounds, const float* dev_cos, const float* dev_sin,
                                               void* dev_scratch, uint64_t scratch_bytes, int32_t T, int32_t n_heads, int32_t n_kv_heads,
                                               int32_t head_dim, int32_t longest, void* stream) {
  if (!dev_qkv || !dev_o || !dev_do || !dev_lse || !dev_dqkv || !dev_bounds || !dev_scratch) return FT_EINVAL;
  if (!aligned(dev_qkv, 16) || !aligned(dev_o, 16) || !aligned(dev_do, 16) || !aligned(dev_dqkv, 16) || !aligned(dev_cos, 16) ||
      !aligned(dev_sin, 16) || !aligned(dev_lse, 4) || !aligned(dev_bounds, 4) || !aligned(dev_scratch, 256) || !dev_cos != !dev_sin)
    return FT_EINVAL;
  const size_t need = fs::attention_packed_scratch_bytes(T, n_heads, n_kv_heads, head_dim, longest);
  if (need == 0) return FT_EINVAL;
  if (scratch_bytes < need) return FT_ENOMEM;
  const Sizes n(T, n_heads, n_kv_heads, head_dim);
  const size_t table = (size_t)longest * (head_dim / 2) * sizeof(float);
  const struct { const void* p; size_t bytes; } inputs[] = {{dev_qkv, n.qkv}, {dev_o, n.o}, {dev_do, n.o}, {dev_lse, n.lse},
                                                            {dev_cos, table}, {dev_sin, table}, {dev_bounds, n.bounds}};
  for (const auto& in : inputs)
    if (in.p && (overlap(dev_dqkv, n.qkv, in.p, in.bytes) || overlap(dev_scratch, need, in.p, in.bytes))) return FT_EINVAL;
  if (overlap(dev_dqkv, n.qkv, dev_scratch, need)) return FT_EINVAL;
  int* status = fs::attention_status_word();
  if (!status) return FT_ECUDA;
  return status_of(fs::attention_packed_bwd(
      reinterpret_cast<const fs::bf16*>(dev_qkv), reinterpret_cast<const fs::bf16*>(dev_o), reinterpret_cast<const fs::bf16*>(dev_do),
      dev_lse, reinterpret_cast<fs::bf16*>(dev_dqkv), dev_cos, dev_sin, docs_of(dev_bounds, T), dev_scratch, T, n_heads, n_kv_heads,
      head_dim, longest, status, reinterpret_cast<cudaStream_t>(stream)));
}
