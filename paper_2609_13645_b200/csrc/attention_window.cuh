// Host-side interface of causal attention over a sliding window with sink keys (tcgen05 tensor cores).
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.cuh"

namespace fs {

// Query i sees key j iff j <= i and (i - j < window or j < sinks); window >= 1, sinks >= 0.  Layouts as in attention.cuh.
cudaError_t attention_window_fwd(const bf16* qkv, bf16* o, float* lse, int B, int S, int n_heads, int n_kv, int d, int window,
                                 int sinks, int* err, cudaStream_t st);

// scratch: attention_window_scratch_bytes() bytes, 256-byte aligned; contents on entry do not matter.  launches (may be null):
// kernels enqueued (delta; dK/dV and dQ once a round of heads; without stored dS^T one dQ, and one that adds partial sums).
size_t attention_window_scratch_bytes(int B, int S, int n_heads, int n_kv, int d, int window, int sinks);
// The most that any batch of up to max_batch rows of up to max_seq tokens needs.
size_t attention_window_most_scratch_bytes(int max_batch, int max_seq, int n_heads, int n_kv, int d, int window, int sinks);
cudaError_t attention_window_bwd(const bf16* qkv, const bf16* o, const bf16* d_o, const float* lse, bf16* dqkv, const float* cos,
                                 const float* sin, void* scratch, int B, int S, int n_heads, int n_kv, int d, int window, int sinks,
                                 int* err, cudaStream_t st, int* launches = nullptr);

// Attention inside the documents of a packed batch of T rows: row i sees the rows from its document's first one to itself.
// start, end: first row of a row's document and the one behind its last (rows behind the last document: T and the number of rows
// in front of them); pos: row - start, the row of the rotation tables.
struct Docs {
  const int *start, *end, *pos;
};
// attention_packed_fwd_tile: its kernel of one tile a CTA, for small calls (attention_packed_fwd chooses).
cudaError_t attention_packed_fwd_tile(const bf16* qkv, bf16* o, float* lse, const Docs& docs, int T, int n_heads, int n_kv, int d, int* err,
                                      cudaStream_t st);
cudaError_t attention_packed_fwd(const bf16* qkv, bf16* o, float* lse, const Docs& docs, int T, int n_heads, int n_kv, int d, int* err,
                                 cudaStream_t st);
// longest: rows of the longest document, at most; cos, sin: fp32 [longest, d / 2] or null.
size_t attention_packed_scratch_bytes(int T, int n_heads, int n_kv, int d, int longest);
cudaError_t attention_packed_bwd(const bf16* qkv, const bf16* o, const bf16* d_o, const float* lse, bf16* dqkv, const float* cos,
                                 const float* sin, const Docs& docs, void* scratch, int T, int n_heads, int n_kv, int d, int longest,
                                 int* err, cudaStream_t st);

}  // namespace fs
