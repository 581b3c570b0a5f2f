// One AdamW step over many tensors in one launch, with moments in 32 bits or in 8.
//
// A plan lists the tensors once: the host cuts them into chunks of 2048 elements and writes both lists into a blob that the
// caller copies to the device, so that a step costs one launch whatever the number and sizes of the tensors.  A block walks over
// chunks; a thread holds 8 consecutive elements of each array.  Every array is read and written once: bound by memory (30
// bytes an element with fp32 moments and gradients and a bf16 copy, 16.1 with 8-bit moments and bf16 gradients).
//
// Moments in 8 bits: runs of 256 elements share a scale, the run's greatest magnitude / 448; an element is a signed 8-bit float
// (4 exponent and 3 mantissa bits, at most 448) times it.  The second moment is kept as its square root, which halves the
// range that the codes have to span.  A moment moves by a fraction 1 - beta of its distance to the gradient's in a step, far less
// than the 6 to 12 % between two codes: rounded to nearest it would never move again.  So codes are rounded up or down at
// random, with probabilities that keep the mean, by 16 bits of a counter-based generator (the dropout masks' one):
//   key = mix(mix(seed) ^ step C2),   word of elements 2 k and 2 k + 1 = mix(key ^ k C3)
// whose 16-bit parts, lowest first, serve m and sqrt(v) of the first and of the second; elements count through the tensors in the
// plan's order, each tensor rounded up to 256.  A second moment that is not 0 never becomes 0, which would let the next update
// divide by epsilon alone.  The codes and scales are, bit for bit, those of this definition in 64 bits: fp32 decides where it can, and what it
// leaves open is formed again in 64 bits.
#include <cuda_fp8.h>
#include <float.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>
#include <utility>
#include <vector>

#include "../../include/forgestep.h"
#include "adamw_math.cuh"
#include "common.cuh"

namespace fs {
namespace {

constexpr int kChunk = 2048, kThreads = 256, kRun = 256;
// Second moments in 8 bits are worked on in roots times 2^16: fp32 holds the squares of roots from 2^-79 to 2^48.  (Roots outside formed in 64 bits
// too: 4 % more instructions, 579 -> 614 us.)
constexpr float kUp = 65536.f, kDown = 1.f / 65536.f;
constexpr uint32_t kMagic = 0x41445750u;
constexpr unsigned long long kStepKey = 0xA24BAED4963EE407ull, kGroupKey = 0x8CB92BA72F3D8DD7ull;

struct PlanHeader {
  uint32_t magic;
  int32_t n_tensors, n_chunks, param16, grad16, bits, pad0, pad1;
  uint64_t bytes, chunk_offset;  // of the blob; of the chunk list in it
};
struct PlanTensor {
  void* p;
  const void* g;
  void *m, *v;
  float *ms, *vs;
  bf16* copy;
  long long n;
  long long base;  // elements of the tensors before, each rounded up to 256
  float wd;
  int aligned;  // whole threads' elements can be moved as vectors
};
struct PlanChunk {
  int tensor, index;
};

struct StepArgs {
  float lr, eps;
  double beta1, omb1, beta2, omb2, log_beta1, log_beta2;  // omb = 1 - beta
  float b1[2], o1[2], b2[2], o2[2];                       // the first four in two fp32 parts
  const long long* step;
  const float *dev_lr, *grad_scale;
  unsigned long long seed;
};

// ---- 8 consecutive elements of a thread
__device__ __forceinline__ void load32(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
               "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void load8(const float* p, int n, bool vec, float (&f)[8]) {
  if (vec) {
    uint32_t w[8];
    load32(p, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load8(const bf16* p, int n, bool vec, float (&f)[8]) {
  if (vec) {
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void store8(float* p, int n, bool vec, const float (&f)[8]) {
  if (vec) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(f[i]);
    store32(p, w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = f[i];
  }
}
__device__ __forceinline__ void store8(bf16* p, int n, bool vec, const float (&f)[8]) {
  if (vec) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = __float2bfloat16_rn(f[i]);
  }
}
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int n, bool vec) {
  if (vec) return *reinterpret_cast<const uint2*>(p);
  uint8_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = i < n ? p[i] : 0;
  uint2 r;
  memcpy(&r, b, 8);
  return r;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int n, bool vec, uint2 w) {
  if (vec) {
    *reinterpret_cast<uint2*>(p) = w;
  } else {
    uint8_t b[8];
    memcpy(b, &w, 8);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = b[i];
  }
}

// The values of 8 codes over a scale.
__device__ __forceinline__ void decode(uint2 w, float scale, float (&f)[8]) {
  const uint32_t h[2] = {w.x, w.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 v = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(h[i >> 1] >> (16 * (i & 1))), __NV_E4M3));
    const float2 x = __half22float2(v);
    f[2 * i] = x.x * scale;
    f[2 * i + 1] = x.y * scale;
  }
}
__device__ __forceinline__ float code_value(uint2 w, int i) {
  const uint32_t code = (i < 4 ? w.x >> (8 * i) : w.y >> (8 * (i - 4))) & 0xffu;
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}
__device__ __forceinline__ void put_code(uint2& w, int i, uint32_t code) {
  const uint32_t at = 8 * (i & 3), keep = ~(0xffu << at);
  if (i < 4) w.x = (w.x & keep) | code << at;
  else w.y = (w.y & keep) | code << at;
}

// ---- numbers of two fp32 parts, about 45 bits
struct Two {
  float h, l;
};
__device__ __forceinline__ Two product(float a, float b) {
  const float h = __fmul_rn(a, b);
  return {h, __fmaf_rn(a, b, -h)};
}
__device__ __forceinline__ Two product(Two a, Two b) {
  const Two p = product(a.h, b.h);
  return {p.h, __fmaf_rn(a.h, b.l, __fmaf_rn(a.l, b.h, p.l))};
}
__device__ __forceinline__ Two sum(Two a, Two b) {
  const float s = __fadd_rn(a.h, b.h), t = __fsub_rn(s, a.h);
  const float e = __fadd_rn(__fadd_rn(__fsub_rn(a.h, __fsub_rn(s, t)), __fsub_rn(b.h, t)), __fadd_rn(a.l, b.l));
  const float h = __fadd_rn(s, e);
  return {h, __fsub_rn(e, __fsub_rn(h, s))};
}
__device__ __forceinline__ Two root(Two a) {  // a.h > 0
  float r, inv;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(a.h));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(r));
  const float e = __fmul_rn(__fadd_rn(__fmaf_rn(-r, r, a.h), a.l), 0.5f * inv), h = __fadd_rn(r, e);
  return {h, __fsub_rn(e, __fsub_rn(h, r))};
}

// A moment (ROOT: the second one's root) of an element from its code, scale and gradient, as the definition orders the operations.
template <bool ROOT>
__device__ __forceinline__ double moment_64(const StepArgs& a, float code, float scale, float g, float clip) {
  const double kept = __dmul_rn((double)code, (double)scale), d = __dmul_rn((double)g, (double)clip);
  if (!ROOT) return __dadd_rn(__dmul_rn(a.beta1, kept), __dmul_rn(a.omb1, d));
  return __dsqrt_rn(__dadd_rn(__dmul_rn(a.beta2, __dmul_rn(kept, kept)), __dmul_rn(__dmul_rn(a.omb2, d), d)));
}

// ---- rounding: floor(|y| / step + bits / 65536) steps; from 2^-6 on a step is the last of 3 mantissa bits, below it is 2^-9
// y 2^-120 has its code in bits 20 to 26 (below 2^-6 it is a denormal number, whose bits count the same steps), and what is cut off behind
// them.  Here all that lies 4 places further up, so that the code ends at the top byte without y's sign, and `random` (16 bits, 8
// places up) is added.
__device__ __forceinline__ uint32_t with_random(float small, uint32_t random) { return __float_as_uint(small) * 16u + random; }
// Whether what lies behind the code is within off / 2^20 steps of a border; off, under 2^19, in the low 23 bits of its argument.
__device__ __forceinline__ bool at_border(uint32_t sum, uint32_t off) { return sum * 256u + off * 4096u <= off * 8192u; }
__device__ __forceinline__ uint32_t round_random(double a, uint32_t bits) {
  const int e = a < 0.015625 ? 0 : (__double2hiint(a) >> 20) - 1023 + 6;  // binades above 2^-6
  const double steps = a * __hiloint2double((1023 + 9 - e) << 20, 0);     // 8 to 16 of them in a binade, up to 8 below
  return min((uint32_t)((int)floor(steps + (double)bits * (1.0 / 65536.0)) + 8 * e), 126u);
}

// A run's greatest element: fp32 bits (infinities and NaN are the greatest), and its scale.
struct RunTop {
  uint32_t own, top;  // of the lane, with the element's number in place of the last 3 bits; of the run, without them
  int lane;           // that holds it
  bool whole;         // the run is formed in 64 bits: others are only a few roundings below and may be it, or `terms` are far greater than it
  float scale;        // 0: the run is 0
  __device__ __forceinline__ bool coded() const { return top >= 0x0d800000u; }  // from 2^-100 on
};
// grad_top: the lane's greatest gradient; terms: its term in the elements, if they are sums that may cancel.
__device__ __forceinline__ RunTop greatest(const float (&x)[8], float grad_top, float terms) {
  RunTop t;
  uint32_t key[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) key[i] = (__float_as_uint(x[i]) & 0x7ffffff8u) | (uint32_t)i;
  t.own = max(max(max(key[0], key[1]), max(key[2], key[3])), max(max(key[4], key[5]), max(key[6], key[7])));
  t.top = __reduce_max_sync(0xffffffffu, t.own) & ~7u;
  const bool may_win = t.own >= t.top - 64u;
  const uint32_t who = __ballot_sync(0xffffffffu, may_win);
  uint32_t second = 0;  // 2^32 less its distance to the lane's greatest
#pragma unroll
  for (int i = 0; i < 8; ++i) second = __viaddmax_u32(key[i], 0u - t.own, second);
  t.lane = __ffs(who) - 1;
  const bool near = may_win && second >= 0u - 72u;  // the 64, and the numbers in the last bits
  // without gradients in the run, elements that are near each other have one code and are equal
  t.whole = ((who & (who - 1)) != 0 || __any_sync(0xffffffffu, near || terms > 4.f * __uint_as_float(t.top))) && __any_sync(0xffffffffu, grad_top != 0.f);
  t.scale = 0.f;
  return t;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float magnitude(const float (&g)[8]) {
  return max3(max3(fabsf(g[0]), fabsf(g[1]), fabsf(g[2])), max3(fabsf(g[3]), fabsf(g[4]), fabsf(g[5])), fmaxf(fabsf(g[6]), fabsf(g[7])));
}
// The number of the lane's greatest, of 8.
__device__ __forceinline__ float pick(const float (&g)[8], uint32_t number) {
  const bool b0 = number & 1u, b1 = number & 2u, b2 = number & 4u;
  const float g01 = b0 ? g[1] : g[0], g23 = b0 ? g[3] : g[2], g45 = b0 ? g[5] : g[4], g67 = b0 ? g[7] : g[6];
  return b2 ? (b1 ? g67 : g45) : (b1 ? g23 : g01);
}
// The scales of both moments: the winners' values in two parts, m's on the lower lanes and the root of v's on the upper ones.  Returns in
// bits 0 and 16 whether they lie half way between two fp32 numbers but for the last places of 64 bits (one run in a thousand: the betas are
// decimal fractions, whose multiples of fp32 numbers land there).
__device__ __forceinline__ uint32_t run_scales(RunTop& m, RunTop& v, const StepArgs& a, uint2 old_m, uint2 old_v, float scale_m, float scale_v,
                                               float clip_up, const float (&g)[8]) {
  const float gm = __shfl_sync(0xffffffffu, pick(g, m.own), m.lane), cm = __shfl_sync(0xffffffffu, code_value(old_m, m.own & 7), m.lane);
  const float gv = __shfl_sync(0xffffffffu, pick(g, v.own), v.lane), cv = __shfl_sync(0xffffffffu, code_value(old_v, v.own & 7), v.lane);
  const bool second = (threadIdx.x & 16u) != 0;
  Two kept = product(second ? cv : cm, second ? scale_v : scale_m);
  const Two d = product(second ? gv : gm, second ? clip_up : clip_up * kDown);
  Two grown = product(second ? Two{a.o2[0], a.o2[1]} : Two{a.o1[0], a.o1[1]}, d);
  const Two square = product(kept, kept), twice = product(grown, d);
  if (second) { kept = square; grown = twice; }
  Two x = sum(product(second ? Two{a.b2[0], a.b2[1]} : Two{a.b1[0], a.b1[1]}, kept), grown);
  const Two r = root(x);
  if (second) x = r;
  x = product(x, Two{1.f / 448.f, (float)(1.0 / 448.0 - (double)(1.f / 448.f))});
  const float scale = __fadd_rn(x.h, x.l), half_step = __uint_as_float(__float_as_uint(scale) & 0x7f800000u) * 5.9604645e-8f;
  const uint32_t tie = __ballot_sync(0xffffffffu, fabsf(fabsf(__fadd_rn(__fsub_rn(x.h, scale), x.l)) - half_step) < half_step * 1e-3f);
  const float sm = fabsf(__shfl_sync(0xffffffffu, scale, 0)), sv = __shfl_sync(0xffffffffu, scale, 16);
  if (m.coded()) m.scale = sm;
  if (v.coded()) v.scale = sv;
  return tie;
}
// The scale of a run and the codes of its open lanes in 64 bits; the greatest is looked for among the elements [from, to) of every lane.
// x, y: the codes, z: the scale.  A run that is not finite in fp32 has codes of 1, which are what the scale is.
template <bool ROOT, typename G>
__device__ __noinline__ uint3 settle(uint2 codes, bool open, int n, int from, int to, const StepArgs& a, uint2 old, float scale, float clip, const G* grad,
                                     unsigned long long key, unsigned long long first) {
  double most = 0.0;
  bool nan = false;
  for (int i = from; i < to; ++i) {
    const double e = fabs(moment_64<ROOT>(a, code_value(old, i), scale, (float)grad[i], clip));
    most = fmax(most, e);
    nan |= !(e >= 0.0);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, o));
  nan = __any_sync(0xffffffffu, nan);
  if (nan || most > FLT_MAX) return make_uint3(0x38383838u, 0x38383838u, nan ? 0x7fffffffu : 0x7f800000u);
  if (most < 0x1p-100) return make_uint3(0u, 0u, 0u);
  const double unit = __dmul_rn(most, 1.0 / 448.0);
  for (int i = 0; i < (open ? n : 0); ++i) {
    const unsigned long long word = splitmix64(key ^ ((first + (unsigned long long)(i >> 1)) * kGroupKey));
    const uint32_t bits = (uint32_t)(word >> (32 * (i & 1) + (ROOT ? 16 : 0))) & 0xffffu;
    const double e = moment_64<ROOT>(a, code_value(old, i), scale, (float)grad[i], clip);
    uint32_t code = round_random(__ddiv_rn(fabs(e), unit), bits);
    if (ROOT && e > 0.0) code = max(code, 1u);
    if (!ROOT && e < 0.0) code |= 0x80u;
    put_code(codes, i, code);
  }
  return make_uint3(codes.x, codes.y, __float_as_uint((float)unit));
}

__device__ __forceinline__ float approx_root(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float approx_inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// 8 elements a thread, a run a warp.  Bound by instructions: 830 a run (104 an element), of which those of the integer unit (396; 68 % of all
// issue slots are taken) matter most: codes are shifted and added by multiplications, and pairs of fp32 numbers share an
// instruction.  Of 134M parameters' 571 us, the random bits take about 110, the scales in two parts 60, codes settled in 64
// bits 30; the bytes would take 334.
// c.omb1 / 2^16; clip_up, root_down: the scale of the gradients times 2^16 and the root of v's correction over it.
template <bool PARAM16, bool GRAD16>
__device__ __forceinline__ void step8(const PlanTensor& w, long long at, int n, bool vec, const StepArgs& a, const AdamCoef& c, float clip_up,
                                      float root_down, unsigned long long key) {
  typedef typename std::conditional<PARAM16, bf16, float>::type P;
  typedef typename std::conditional<GRAD16, bf16, float>::type G;
  P* pp = reinterpret_cast<P*>(w.p) + at;
  const G* gp = reinterpret_cast<const G*>(w.g) + at;
  uint8_t *mp = reinterpret_cast<uint8_t*>(w.m) + at, *vp = reinterpret_cast<uint8_t*>(w.v) + at;
  float g[8], m[8], r[8];
  const uint2 old_m = load_codes(mp, n, vec), old_v = load_codes(vp, n, vec);
  const float scale_m = w.ms[at / kRun], scale_v = w.vs[at / kRun];
  load8(gp, n, vec, g);
  const float grad_top = magnitude(g);
  decode(old_m, scale_m, m);
  decode(old_v, scale_v * kUp, r);
  {
    float p[8];
    load8(pp, n, vec, p);
    const float wd = w.wd;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 d = mul2(make_float2(g[i], g[i + 1]), both(clip_up)), r0 = make_float2(r[i], r[i + 1]), p0 = make_float2(p[i], p[i + 1]);
      const float2 m1 = fma2(both(c.beta1), make_float2(m[i], m[i + 1]), mul2(both(c.omb1), d));
      const float2 v1 = fma2(both(c.beta2), mul2(r0, r0), mul2(mul2(both(c.omb2), d), d));
      const float2 r1 = make_float2(approx_root(v1.x), approx_root(v1.y));
      const float2 den = fma2(r1, both(root_down), both(c.eps));
      const float2 quot = mul2(mul2(m1, both(c.rbc1)), make_float2(approx_inverse(den.x), approx_inverse(den.y)));  // within 2^-21
      const float2 p1 = fma2(both(-c.lr), fma2(both(wd), p0, quot), p0);
      m[i] = m1.x; m[i + 1] = m1.y;
      r[i] = r1.x; r[i + 1] = r1.y;
      p[i] = p1.x; p[i + 1] = p1.y;
    }
    store8(pp, n, vec, p);
    if (w.copy != nullptr) store8(w.copy + at, n, vec, p);
  }
  if (n < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= n) m[i] = r[i] = 0.f;
  }
  // m's terms may cancel.  Up to gradients' terms of 4 times the greatest element, an element's fp32 error, of up to 3 roundings of its own and 5
  // of the gradient's term, stays under 23 of the greatest's, and two elements that may be the greatest are within 64 last places.
  RunTop tm = greatest(m, grad_top, c.omb1 * fabsf(clip_up) * grad_top), tv = greatest(r, grad_top, 0.f);
  tm.whole = tm.whole || tm.top - 0x0d000000u < 0x01000000u || tm.top >= 0x7f000000u;  // next to 2^-100, and at fp32's end
  // v: but for roots from 2^-61 to 2^46, the low parts of whose squares are normal numbers
  if (tv.top - 0x29000000u >= 0x5e800000u - 0x29000000u)
    tv.whole = tv.top != 0u || __any_sync(0xffffffffu, grad_top != 0.f || (scale_v != 0.f && ((old_v.x | old_v.y) & 0x7f7f7f7fu) != 0u));
  const uint32_t ties = run_scales(tm, tv, a, old_m, old_v, scale_m, scale_v * kUp, clip_up, g);
  const float inv_m = tm.coded() ? approx_inverse(tm.scale) : 0.f, inv_v = tv.coded() ? approx_inverse(tv.scale) : 0.f;
  const unsigned long long first = (unsigned long long)(w.base + at) / 2;
  uint2 cm, cv;
  bool open_m = false, open_v = false;
  // An element's fp32 error in 2^-20 steps, which are the last places of what the floor is taken of (a rounding is up to one of them, in the
  // upper half of a binade): under 14 for the roundings of the element (5 at most), the scale (1), its inverse (4) and the product (1), and 2.5
  // of the terms' that it was added up from, |beta1 m| <= |sum| + |gradient's|.  The latter are at most 4 * 448 / 2^-6 in codes that are kept,
  // which is under half a step, what at_border() holds.
  const float grads = 4.f * c.omb1 * fabsf(clip_up) * inv_m;
  const uint32_t off_v = 14u;
  uint32_t sm[8], sv[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const unsigned long long word = splitmix64(key ^ ((first + (unsigned long long)(i >> 1)) * kGroupKey));
    const float2 ym = mul2(make_float2(m[i], m[i + 1]), both(inv_m)), yv = mul2(make_float2(r[i], r[i + 1]), both(inv_v));
    const float2 fm = mul2(ym, both(7.52316385e-37f)), fv = mul2(yv, both(7.52316385e-37f));
    const float2 t = mul2(make_float2(fabsf(g[i]), fabsf(g[i + 1])), both(grads));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t bits = (uint32_t)(word >> (32 * k));
      const float y = k == 0 ? ym.x : ym.y;
      // 2^-e of the binade that the number, or 2^-6 where that is more, lies in; the sum's low bits are the number of places
      const float binade = __uint_as_float(0x7f000000u - (__float_as_uint(fmaxf(fabsf(y), 0.015625f)) & 0x7f800000u));
      const float places = fmaf(k == 0 ? t.x : t.y, binade, 8388608.f + 14.f);
      sm[i + k] = with_random(k == 0 ? fm.x : fm.y, __byte_perm(bits, 0u, 0x4104));
      open_m |= at_border(sm[i + k], __float_as_uint(places));
      sm[i + k] = (sm[i + k] & 0x7fffffffu) | (__float_as_uint(m[i + k]) & 0x80000000u);
      sv[i + k] = with_random(k == 0 ? fv.x : fv.y, __byte_perm(bits, 0u, 0x4324));
      open_v |= at_border(sv[i + k], off_v);
      if (r[i + k] > 0.f) sv[i + k] = max(sv[i + k], 0x01000000u);
      else sv[i + k] = 0u;
    }
  }
  auto top_bytes = [](const uint32_t* x) { return __byte_perm(__byte_perm(x[0], x[1], 0x0073), __byte_perm(x[2], x[3], 0x0073), 0x5410); };
  cm = make_uint2(top_bytes(sm), top_bytes(sm + 4));
  cv = make_uint2(top_bytes(sv), top_bytes(sv + 4));
  auto settled = [&](auto root, const RunTop& t, float& stored, uint2 codes, bool tie, bool open, uint2 old, float scale) {
    if (tie || t.whole || __any_sync(0xffffffffu, open)) {
      const int winner = t.own & 7, end = (int)(threadIdx.x & 31) == t.lane ? winner + 1 : 0;
      const uint3 s = settle<decltype(root)::value, G>(codes, open || t.whole, n, t.whole ? 0 : winner, t.whole ? n : end, a, old, scale, clip_up * kDown, gp, key, first);
      codes = make_uint2(s.x, s.y);
      stored = __uint_as_float(s.z);
    }
    return codes;
  };
  float new_m = tm.scale, new_v = tv.scale * kDown;
  if (!tm.coded() && !tm.whole) cm = make_uint2(0u, 0u);
  else cm = settled(std::false_type{}, tm, new_m, cm, (ties & 1u) != 0, open_m, old_m, scale_m);
  if (tv.top == 0u && !tv.whole) cv = make_uint2(0u, 0u);
  else cv = settled(std::true_type{}, tv, new_v, cv, (ties & 0x10000u) != 0, open_v, old_v, scale_v);
  store_codes(mp, n, vec, cm);
  store_codes(vp, n, vec, cv);
  __syncwarp();  // every lane has read the scales
  if ((threadIdx.x & 31) == 0) {
    w.ms[at / kRun] = new_m;
    w.vs[at / kRun] = new_v;
  }
}

__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}
// Asks for a whole chunk's arrays, by one thread, so that a block that gets to them finds them in L2.  It pays with 8-bit moments, whose
// kernel has registers for 3 blocks an SM (599 us without, 573 with it), and not with fp32 ones (647 and 670).
template <bool PARAM16, bool GRAD16, int BITS>
__device__ __forceinline__ void prefetch_chunk(const PlanTensor& w, int index) {
  const long long at = (long long)index * kChunk;
  if (w.aligned == 0 || at + kChunk > w.n) return;
  constexpr int P = PARAM16 ? 2 : 4, G = GRAD16 ? 2 : 4, M = BITS / 8;
  prefetch_l2(reinterpret_cast<const uint8_t*>(w.p) + at * P, kChunk * P);
  prefetch_l2(reinterpret_cast<const uint8_t*>(w.g) + at * G, kChunk * G);
  prefetch_l2(reinterpret_cast<const uint8_t*>(w.m) + at * M, kChunk * M);
  prefetch_l2(reinterpret_cast<const uint8_t*>(w.v) + at * M, kChunk * M);
}

template <bool PARAM16, bool GRAD16, int BITS>
__global__ void __launch_bounds__(kThreads, BITS == 8 ? 3 : 4)
adamw_kernel(const uint8_t* __restrict__ plan, int n_chunks, unsigned long long chunk_offset, const __grid_constant__ StepArgs a) {
  typedef typename std::conditional<PARAM16, bf16, float>::type P;
  typedef typename std::conditional<GRAD16, bf16, float>::type G;
  __shared__ float s_bc[2];
  pdl_trigger();
  pdl_wait();
  const long long t = max(__ldg(a.step), 1ll);
  if (threadIdx.x < 2) s_bc[threadIdx.x] = (float)-expm1((double)t * (threadIdx.x == 0 ? a.log_beta1 : a.log_beta2));
  __syncthreads();
  AdamCoef c = make_adam_coef(a.dev_lr != nullptr ? __ldg(a.dev_lr) : a.lr, (float)a.beta1, (float)a.beta2, a.eps, s_bc[0], s_bc[1]);
  c.omb1 = (float)a.omb1;
  c.omb2 = (float)a.omb2;
  float clip = a.grad_scale != nullptr ? __ldg(a.grad_scale) : 1.f;
  const unsigned long long key = BITS == 8 ? splitmix64(splitmix64(a.seed) ^ ((unsigned long long)t * kStepKey)) : 0;
  float root_rbc2 = sqrtf(c.rbc2);
  if (BITS == 8) {
    c.omb1 *= kDown;
    clip *= kUp;
    root_rbc2 *= kDown;
  }
  const PlanTensor* tensors = reinterpret_cast<const PlanTensor*>(plan + sizeof(PlanHeader));
  const PlanChunk* chunks = reinterpret_cast<const PlanChunk*>(plan + chunk_offset);
  for (int k = blockIdx.x; k < n_chunks; k += gridDim.x) {
    const PlanChunk ch = chunks[k];
    const PlanTensor& w = tensors[ch.tensor];
    if (BITS == 8 && threadIdx.x == 0 && k + (int)gridDim.x < n_chunks) {
      const PlanChunk next = chunks[k + gridDim.x];
      prefetch_chunk<PARAM16, GRAD16, BITS>(tensors[next.tensor], next.index);
    }
    const long long at = (long long)ch.index * kChunk + threadIdx.x * 8;
    const long long left = w.n - at;
    const int n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    if (BITS == 32 ? n == 0 : at / kRun * kRun >= w.n) continue;  // with 8 bits a run's 32 threads stay together
    const bool vec = n == 8 && w.aligned != 0;
    if constexpr (BITS == 8) {
      step8<PARAM16, GRAD16>(w, at, n, vec, a, c, clip, root_rbc2, key);
    } else {
      float p[8], g[8], m[8], v[8];
      load8(reinterpret_cast<const P*>(w.p) + at, n, vec, p);
      load8(reinterpret_cast<const G*>(w.g) + at, n, vec, g);
      load8(reinterpret_cast<const float*>(w.m) + at, n, vec, m);
      load8(reinterpret_cast<const float*>(w.v) + at, n, vec, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) adamw_elem(__fmul_rn(g[i], clip), w.wd, c, p[i], m[i], v[i]);
      store8(reinterpret_cast<P*>(w.p) + at, n, vec, p);
      if (w.copy != nullptr) store8(w.copy + at, n, vec, p);
      store8(reinterpret_cast<float*>(w.m) + at, n, vec, m);
      store8(reinterpret_cast<float*>(w.v) + at, n, vec, v);
    }
  }
}

template <bool PARAM16, bool GRAD16>
cudaError_t launch(const PlanHeader& h, const uint8_t* plan, const StepArgs& a, cudaStream_t st) {
  // Blocks that come and go even out what SMs and memory partitions do to each other: 134M parameters with fp32 moments take 672 us in
  // 4 blocks an SM that stay, 647 in 8, 612 in 24, 600 in 64 (595 in 128); with 8-bit ones 577 in 3, 567 in 6, 557 in 27, 571 in 90.
  const unsigned blocks = (unsigned)std::min(h.n_chunks, 148 * (h.bits == 8 ? 27 : 64));
  if (h.bits == 8) return launch_pdl(adamw_kernel<PARAM16, GRAD16, 8>, dim3(blocks), dim3(kThreads), 0, st, plan, h.n_chunks, (unsigned long long)h.chunk_offset, a);
  return launch_pdl(adamw_kernel<PARAM16, GRAD16, 32>, dim3(blocks), dim3(kThreads), 0, st, plan, h.n_chunks, (unsigned long long)h.chunk_offset, a);
}

// Bytes of an array's n elements, by what it is.
struct Kinds {
  int param, grad, moment;
};

// FT_OK, and the number of chunks, for a list that the kernels can take.
ft_status check(const ft_adamw_tensor* list, int32_t n, int32_t param_dtype, int32_t grad_dtype, int32_t bits, long long* chunks) {
  if (!list || n <= 0 || (param_dtype & ~1) || (grad_dtype & ~1) || (bits != 8 && bits != 32)) return FT_EINVAL;
  const Kinds k{param_dtype == 0 ? 2 : 4, grad_dtype == 0 ? 2 : 4, bits / 8};
  long long total = 0;
  std::vector<std::pair<uintptr_t, uintptr_t>> written, read;
  for (int i = 0; i < n; ++i) {
    const ft_adamw_tensor& t = list[i];
    if (t.numel < 0 || t.numel > (1ll << 40) || !isfinite(t.weight_decay)) return FT_EINVAL;
    if (t.numel == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v || (bits == 8) != (t.m_scale != nullptr) || (bits == 8) != (t.v_scale != nullptr)) return FT_EINVAL;
    if (t.copy && param_dtype == 0) return FT_EINVAL;  // a bf16 parameter is its own copy
    const uintptr_t odd = ((uintptr_t)t.param % k.param) | ((uintptr_t)t.grad % k.grad) | ((uintptr_t)t.m % k.moment) | ((uintptr_t)t.v % k.moment) |
                          ((uintptr_t)t.copy % 2) | ((uintptr_t)t.m_scale % 4) | ((uintptr_t)t.v_scale % 4);
    if (odd) return FT_EINVAL;
    const size_t e = (size_t)t.numel, runs = (e + kRun - 1) / kRun;
    auto add = [](std::vector<std::pair<uintptr_t, uintptr_t>>& to, const void* p, size_t bytes) {
      if (p) to.emplace_back((uintptr_t)p, (uintptr_t)p + bytes);
    };
    add(written, t.param, e * k.param);
    add(written, t.m, e * k.moment);
    add(written, t.v, e * k.moment);
    add(written, t.copy, e * 2);
    add(written, t.m_scale, runs * 4);
    add(written, t.v_scale, runs * 4);
    add(read, t.grad, e * k.grad);
    total += (t.numel + kChunk - 1) / kChunk;
    if (total > INT32_MAX / 2) return FT_EINVAL;
  }
  // what the step writes is written by one thread, and not read as a gradient
  std::sort(written.begin(), written.end());
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].first < written[i - 1].second) return FT_EINVAL;
  for (const auto& r : read) {
    auto next = std::lower_bound(written.begin(), written.end(), std::make_pair(r.second, (uintptr_t)0));
    if (next != written.begin() && std::prev(next)->second > r.first) return FT_EINVAL;
  }
  *chunks = total;
  return FT_OK;
}

size_t chunk_list_at(int32_t n) { return (sizeof(PlanHeader) + (size_t)n * sizeof(PlanTensor) + 15) / 16 * 16; }

}  // namespace
}  // namespace fs

extern "C" size_t ft_k_adamw_plan_bytes(const ft_adamw_tensor* tensors, int32_t n_tensors, int32_t param_dtype, int32_t grad_dtype,
                                        int32_t state_bits) {
  try {
    long long chunks = 0;
    if (fs::check(tensors, n_tensors, param_dtype, grad_dtype, state_bits, &chunks) != FT_OK) return 0;
    return fs::chunk_list_at(n_tensors) + (size_t)chunks * sizeof(fs::PlanChunk);
  } catch (...) {
    return 0;
  }
}

extern "C" ft_status ft_k_adamw_plan(const ft_adamw_tensor* tensors, int32_t n_tensors, int32_t param_dtype, int32_t grad_dtype,
                                     int32_t state_bits, void* host_plan, uint64_t bytes) {
  try {
    long long chunks = 0;
    const ft_status s = fs::check(tensors, n_tensors, param_dtype, grad_dtype, state_bits, &chunks);
    if (s != FT_OK) return s;
    if (!host_plan || (reinterpret_cast<uintptr_t>(host_plan) & 7u) != 0) return FT_EINVAL;
    const size_t need = fs::chunk_list_at(n_tensors) + (size_t)chunks * sizeof(fs::PlanChunk);
    if (bytes < need) return FT_ENOMEM;
    memset(host_plan, 0, need);
    uint8_t* blob = reinterpret_cast<uint8_t*>(host_plan);
    fs::PlanHeader* h = reinterpret_cast<fs::PlanHeader*>(blob);
    fs::PlanTensor* list = reinterpret_cast<fs::PlanTensor*>(blob + sizeof(fs::PlanHeader));
    fs::PlanChunk* ch = reinterpret_cast<fs::PlanChunk*>(blob + fs::chunk_list_at(n_tensors));
    h->magic = fs::kMagic;
    h->n_tensors = n_tensors;
    h->n_chunks = (int32_t)chunks;
    h->param16 = param_dtype == 0;
    h->grad16 = grad_dtype == 0;
    h->bits = state_bits;
    h->bytes = need;
    h->chunk_offset = fs::chunk_list_at(n_tensors);
    long long base = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
      const ft_adamw_tensor& t = tensors[i];
      // a thread moves 8 elements of an array at once: 32 bytes of fp32, 16 of bf16, 8 of codes; chunks are prefetched in units of 16
      const uintptr_t odd = ((uintptr_t)t.param & (h->param16 ? 15u : 31u)) | ((uintptr_t)t.grad & (h->grad16 ? 15u : 31u)) |
                            (((uintptr_t)t.m | (uintptr_t)t.v) & (state_bits == 8 ? 15u : 31u)) | ((uintptr_t)t.copy & 15u);
      list[i] = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, reinterpret_cast<fs::bf16*>(t.copy), t.numel, base, t.weight_decay, odd == 0};
      for (long long k = 0; k < (t.numel + fs::kChunk - 1) / fs::kChunk; ++k) *ch++ = {i, (int)k};
      base += (t.numel + fs::kRun - 1) / fs::kRun * fs::kRun;
    }
    return FT_OK;
  } catch (...) {
    return FT_ENOMEM;
  }
}

extern "C" ft_status ft_k_adamw(const void* host_plan, const void* dev_plan, uint64_t plan_bytes, double lr, double beta1, double beta2, double eps,
                                const int64_t* dev_step, const float* dev_lr, const float* dev_grad_scale, uint64_t seed, void* stream) {
  if (!host_plan || !dev_plan || !dev_step || (reinterpret_cast<uintptr_t>(host_plan) & 7u) || (reinterpret_cast<uintptr_t>(dev_plan) & 15u)) return FT_EINVAL;
  if (((uintptr_t)dev_step & 7u) || ((uintptr_t)dev_lr & 3u) || ((uintptr_t)dev_grad_scale & 3u)) return FT_EINVAL;
  if (!isfinite((float)lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !isfinite((float)eps)) return FT_EINVAL;
  const fs::PlanHeader& h = *reinterpret_cast<const fs::PlanHeader*>(host_plan);
  if (plan_bytes < sizeof(h) || h.magic != fs::kMagic || h.bytes != plan_bytes) return FT_EINVAL;
  if (h.bits == 8 && eps < 0x1p-64) return FT_EINVAL;  // next to which roots that fp32 does not hold are nothing
  if (h.n_chunks == 0) return FT_OK;
  auto low = [](double v) { return (float)(v - (double)(float)v); };
  const double omb1 = 1.0 - beta1, omb2 = 1.0 - beta2;
  const fs::StepArgs a{(float)lr, (float)eps, beta1, omb1, beta2, omb2, log(beta1), log(beta2),
                       {(float)beta1, low(beta1)}, {(float)omb1, low(omb1)}, {(float)beta2, low(beta2)}, {(float)omb2, low(omb2)}, reinterpret_cast<const long long*>(dev_step), dev_lr, dev_grad_scale, seed};
  const uint8_t* plan = reinterpret_cast<const uint8_t*>(dev_plan);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (h.param16) e = h.grad16 ? fs::launch<true, true>(h, plan, a, st) : fs::launch<true, false>(h, plan, a, st);
  else e = h.grad16 ? fs::launch<false, true>(h, plan, a, st) : fs::launch<false, false>(h, plan, a, st);
  return e == cudaSuccess ? FT_OK : FT_ECUDA;
}
