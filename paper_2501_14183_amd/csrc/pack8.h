// The format of an activation in 8 bits, and the activations of the feed-forward block: device helpers of pack8.hip, ffn.hip and
// int8.hip.
//
// A row is cut into blocks of 32 channels.  A block has one exponent byte E and a signed byte for each channel, which stands for
// code * 2^(E - 127): the step is the smallest power of two (of at least 2^-126) of which the block's largest magnitude is, rounded,
// at most 127 steps, and a code is the nearest whole number, ties to even.  A power of two, and not the largest value over 127,
// because code * step then is a bf16 number: what the backward pass multiplies is the checkpoint itself, with no rounding of its
// own.  It costs half a bit on average: a value is off by at most half a step, 1/127.5 of the block's largest (which is 63.75 to 127.5
// steps).  Two exceptions: a block whose largest is below 63.75 * 2^-126 has the least step, and its values are off by up to 2^-127;
// magnitudes from 127.5 * 2^121 on count as 127 * 2^121, off by less than a step.  A block that holds an infinity or NaN has E = 255 and
// stands for NaN.
#ifndef VARDROP_PACK8_H
#define VARDROP_PACK8_H
#include "bf16_mfma.h"

namespace {

constexpr int kPackBlock = 32;
__host__ __device__ inline int pack_blocks(int d) { return (d + kPackBlock - 1) / kPackBlock; }
// Codes [rows][d], then exponents [rows][blocks].
__host__ __device__ inline size_t pack_exponents_at(long long rows, int d) { return vd_align_up((size_t)rows * d, 256); }
inline size_t pack_bytes(long long rows, int d) { return pack_exponents_at(rows, d) + vd_align_up((size_t)rows * pack_blocks(d), 256); }

__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// E of a block whose largest magnitude has these bits (127.5 / 64 is the mantissa that 0x10000 carries into the exponent)
__device__ inline uint32_t pack_exponent(uint32_t most) {
  if (most >= 0x7f800000u) return 255u;
  const uint32_t e = (most + 0x10000u) >> 23;
  return min(max(e, 7u) - 6u, 248u);
}
__device__ inline float pack_up(uint32_t e) { return __uint_as_float((254u - min(e, 253u)) << 23); }
__device__ inline float pack_step(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }
// Code of v in the low byte: 1.5 * 2^23 has steps of one, and the product with a power of two is exact.  (Only the largest exponent's can
// be above 127.)
__device__ inline uint32_t pack_code(float v, float up) { return __float_as_uint(fmaf(v, up, 12582912.f)); }
__device__ inline float pack_limit(float v) { return __builtin_amdgcn_fmed3f(v, -127.f * 0x1p121f, 127.f * 0x1p121f); }
// the larger of two magnitudes, NaN if one is
__device__ inline float most_of(float a, float b) { return __builtin_elementwise_maximum(__builtin_fabsf(a), __builtin_fabsf(b)); }
__device__ inline uint32_t pack_four(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
  return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}
// Codes of eight neighbouring values; the four lanes of a block come together, `e` is the block's.
__device__ inline u32x2 pack_eight(const float (&v)[8], uint32_t& e) {
  float top = most_of(most_of(most_of(v[0], v[1]), most_of(v[2], v[3])), most_of(most_of(v[4], v[5]), most_of(v[6], v[7])));
  top = most_of(top, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(top), 0xb1, 0xf, 0xf, true)));      // lanes ^ 1
  top = most_of(top, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(top), 0x4e, 0xf, 0xf, true)));      // lanes ^ 2
  e = pack_exponent(__float_as_uint(top));
  const float up = pack_up(e);
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = pack_code(v[i], up);
  if (e >= 248u) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = pack_code(pack_limit(v[i]), up);
  }
  return u32x2{pack_four(c[0], c[1], c[2], c[3]), pack_four(c[4], c[5], c[6], c[7])};
}
// Values of four codes (one conversion with sign extension and one product each)
__device__ inline void unpack_four(uint32_t w, float step, float* v) {
  v[0] = (float)(int8_t)w * step;
  v[1] = (float)(int8_t)(w >> 8) * step;
  v[2] = (float)(int8_t)(w >> 16) * step;
  v[3] = (float)((int)w >> 24) * step;
}
__device__ inline void unpack_eight(u32x2 codes, uint32_t e, float (&v)[8]) {
  const float step = pack_step(e);
  unpack_four(codes.x, step, v);
  unpack_four(codes.y, step, v + 4);
}

// ---- GELU(x) = x Phi(x), and its derivative Phi(x) + x phi(x).  With u = |x| and the upper tail Q = 1 - Phi,
//   GELU = max(x, 0) - u Q(u),   GELU' = 1/2 +- (1/2 - S(u)),   S = Q - u phi = Q R
// where log2 Q and R are smooth: polynomials of degrees 6 and 5 fitted to them over 0 <= u <= 5.5 (Q to 2.7e-5 of itself, u Q to
// 3.9e-6, S to 1.5e-5; from 5.5 on u Q is below 1.1e-7).  One exponential, no reciprocal: 13 and 22 vector issues an
// element; by the formula 7.1.26 of Abramowitz and Stegun 22 and 30, which the products cannot hide.  For results in bf16.
__device__ inline float tail_of(float u) {
  float p = 2.6153800718020648e-05f;
  p = fmaf(p, u, -0.0006609821575693786f);
  p = fmaf(p, u, 0.007488316390663385f);
  p = fmaf(p, u, -0.05197042599320412f);
  p = fmaf(p, u, -0.46032944321632385f);
  p = fmaf(p, u, -1.1505839824676514f);
  p = fmaf(p, u, -1.0000361204147339f);
  return fast_exp2(p);
}
__device__ inline float slope_factor(float u) {
  float r = -0.0016836859285831451f;
  r = fmaf(r, u, 0.01988912560045719f);
  r = fmaf(r, u, -0.1082354485988617f);
  r = fmaf(r, u, -0.6373599171638489f);
  r = fmaf(r, u, -0.7977257370948792f);
  return fmaf(r, u, 0.9999952912330627f);
}
// |x|, at most 5.5 (NaN stays)
__device__ inline float tail_argument(float x) { return __builtin_elementwise_minimum(__builtin_fabsf(x), 5.5f); }
enum { kActNone = VARDROP_ACT_NONE, kActRelu = VARDROP_ACT_RELU, kActGelu = VARDROP_ACT_GELU };
// For results in fp32: Q = exp(-u^2 / 2) R(t), t = 1 / (1 + u / 4), R a polynomial of degree 9 fitted over 0 <= u <= 14 (1.5e-8 of Q; from 14 on
// u Q is below 2^-140); u phi comes from the same exponential.  Value and derivative are off by at most 2 and 7 times 2^-24 (1 + u).  With the
// library's erfc and exp the gradient of the activation of 999 x 321 x 449 took 15.8 us, and not 13.6.
__device__ inline float fine_tail(float u, float& power) {
  const float t = __builtin_amdgcn_rcpf(fmaf(u, 0.25f, 1.f));
  power = fast_exp2(u * u * -0.72134752044448170f);
  float p = 0.03394695743918419f;
  p = fmaf(p, t, -0.19617852568626404f);
  p = fmaf(p, t, 0.3950040936470032f);
  p = fmaf(p, t, -0.3334725499153137f);
  p = fmaf(p, t, 0.3044894337654114f);
  p = fmaf(p, t, -0.02038533240556717f);
  p = fmaf(p, t, 0.12156835198402405f);
  p = fmaf(p, t, 0.09482017159461975f);
  p = fmaf(p, t, 0.10022900998592377f);
  return power * fmaf(p, t, -2.1600530089926906e-05f);
}
__device__ inline float fine_argument(float x) { return __builtin_elementwise_minimum(__builtin_fabsf(x), 14.f); }
// `fine`: for fp32 results
template <int ACT, bool FINE>
__device__ inline float act_value(float x) {
  if constexpr (ACT == kActNone) return x;
  if constexpr (ACT == kActRelu) return x < 0.f ? 0.f : x;              // (NaN stays)
  float power;
  const float u = FINE ? fine_argument(x) : tail_argument(x);
  return fmaf(-u, FINE ? fine_tail(u, power) : tail_of(u), __builtin_elementwise_maximum(x, 0.f));
}
// value and derivative
template <int ACT, bool FINE>
__device__ inline float act_both(float x, float& slope) {
  if constexpr (ACT == kActRelu) {
    slope = x > 0.f ? 1.f : (x <= 0.f ? 0.f : x);
    return x < 0.f ? 0.f : x;
  }
  if constexpr (FINE) {
    float power;
    const float u = fine_argument(x), q = fine_tail(u, power), s = fmaf(u * -0.39894228040143268f, power, q);
    slope = x > 0.f ? 1.f - s : s;
    return fmaf(-u, q, __builtin_elementwise_maximum(x, 0.f));
  }
  const float u = tail_argument(x), q = tail_of(u);
  const float t = fmaf(-slope_factor(u), q, 0.5f);
  slope = 0.5f + __uint_as_float(__float_as_uint(t) ^ (__float_as_uint(x) & 0x80000000u));
  return fmaf(-u, q, __builtin_elementwise_maximum(x, 0.f));
}

// eight neighbouring elements
template <typename T> __device__ inline void load_eight(const T* p, float (&v)[8]);
template <> __device__ inline void load_eight<bf16_t>(const bf16_t* p, float (&v)[8]) {
  const u32x4 q = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    v[2 * w] = __uint_as_float(q[w] << 16);
    v[2 * w + 1] = __uint_as_float(q[w] & 0xffff0000u);
  }
}
template <> __device__ inline void load_eight<float>(const float* p, float (&v)[8]) {
  const u32x4 a = reinterpret_cast<const u32x4*>(p)[0], b = reinterpret_cast<const u32x4*>(p)[1];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    v[w] = __uint_as_float(a[w]);
    v[4 + w] = __uint_as_float(b[w]);
  }
}
__device__ inline u32x4 eight_bf16(const float (&v)[8]) {
  return u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}
// `past`: past the caches.  A result that no cache holds until it is read otherwise drives out what the tiles beside it read again, and
// is written back when the kernel ends.  us, 65 536 x 768 x 1536: activation 250 -> 211, its gradient 280 -> 216 (128 x 128 tiles), dx 146 -> 137
// (256 x 256).  From kPastCaches on, as the block norms.
constexpr long long kPastCaches = 16 << 20;
template <typename V>
__device__ inline void store_past(V* p, const V& v, bool past) {
  if (past) {
    asm volatile("");            // (keeps the compiler from making one store, a plain one, of the two)
    __builtin_nontemporal_store(v, p);
    asm volatile("");
  } else {
    *p = v;
  }
}
__device__ inline void store_eight(bf16_t* p, const float (&v)[8], bool past = false) { store_past(reinterpret_cast<u32x4*>(p), eight_bf16(v), past); }
__device__ inline void store_eight(float* p, const float (&v)[8], bool past = false) {
  store_past(reinterpret_cast<u32x4*>(p), u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, past);
  store_past(reinterpret_cast<u32x4*>(p) + 1, u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])}, past);
}
__device__ inline float to_float(bf16_t v) { return bf2f(v); }
__device__ inline float to_float(float v) { return v; }
__device__ inline void from_float(bf16_t* p, float v) { *p = f2bf(v); }
__device__ inline void from_float(float* p, float v) { *p = v; }

}  // namespace
#endif  // VARDROP_PACK8_H
