// 8-bit rows: e4m3 (OCP: 4 bits of exponent, 3 of mantissa, largest value 448, no infinity) with one scale for each block of
// 128 values of a row, or for each 128 x 128 block of a weight.  A scale is a power of two, kept as its exponent's byte b: 2^(b - 127).
// Powers of two because they cost nothing: dividing by one and multiplying by one round nothing, a stored value times its scale
// is exact in bf16, and the matrix instruction takes the byte as it is.
#pragma once
#include "common.h"
#include "mfma_util.h"

namespace mb {

constexpr int kFp8Block = 128;
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__host__ __device__ inline int fp8_blocks(int width) { return (width + kFp8Block - 1) / kFp8Block; }

// Descriptor of `bytes` bytes from `base`, both the same in all lanes.  (Said to the compiler word by word: bounds that it works out
// on the vector unit would make a loop over the lanes of every access.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a), hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(hi << 32 | lo), 0,
                                           (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// |x|, or 0 for infinities and NaN (which a block's scale is not taken from).
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < __builtin_inff() ? a : 0.f;
}

// The scale of a block whose largest finite magnitude is `amax`: the smallest 2^e, e >= -126, with amax <= 448 * 2^e, as e + 127.
// (448 = 1.75 * 2^8: the addition carries into the exponent where the mantissa is over 1.75.)
__device__ __forceinline__ int scale_byte(float amax) {
  return max((int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8, 1);
}
// Whether a largest magnitude lies so near to 448 * 2^e that an error of `reach` 2^-23 of its power of two could decide between
// two scales, and the least magnitude that does.
__device__ __forceinline__ bool near_border(float amax, uint32_t reach) {
  return (__float_as_uint(amax) & 0x7fffffu) - (0x600000u - reach) < 2 * reach;
}
__device__ __forceinline__ float border_from(float amax, uint32_t reach) {
  return __uint_as_float((__float_as_uint(amax) & 0x7f800000u) | (0x600000u - reach));
}
// The scale itself; byte 255 stands for NaN.
__device__ __forceinline__ float scale_value(int byte) {
  return byte == 0 ? __uint_as_float(0x00400000u) : byte == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)byte << 23);
}

// Four values as e4m3 under a scale (round to nearest even; what is not finite becomes NaN).  Of `scale` the instruction takes
// the exponent: byte << 23 as a float.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d, float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ float scale_bits(int byte) { return __uint_as_float((uint32_t)byte << 23); }
// Four e4m3 values.
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float (&x)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}
// The same times a scale (its exponent, byte << 23 as a float).
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float scale, float (&x)[4]) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}

// Eight e4m3 values times a scale, as bf16; exact where the product is a normal number.  (Of `scale` the instruction takes the
// exponent: byte << 23 as a float.)
__device__ __forceinline__ bf16x8 to_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return as_bf16x8(r);
}

// The lane's number, counted afresh: what only rare code needs is not kept in registers for it.
__device__ __forceinline__ int lane_again() {
  uint32_t all = ~0u;
  asm volatile("" : "+s"(all));
  return __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0u));
}

// Largest of a value over groups of 8 consecutive lanes (the 8 lanes that hold a block of a row, 16 values each).
__device__ __forceinline__ float max_of_8_lanes(float x) {
  x = fmaxf(x, __shfl_xor(x, 1));
  x = fmaxf(x, __shfl_xor(x, 2));
  return fmaxf(x, __shfl_xor(x, 4));
}

// The GeLU with a small RELATIVE error, because a block whose gates are all far negative gets a scale of its own: there an absolute
// error of 1e-7, enough for a bf16 result next to larger ones, would be most of the value.  A stored result is rounded by 2^-4 of
// itself; where the error could decide the block's scale, 64 bits do.  (Phi the normal distribution function, phi its density.)
//
// GeLU(h) = h Phi(h) = max(h, 0) - |h| Phi(-|h|) alone, where the derivative's exp(-h^2 / 2) is not needed as well: Phi(-|h|) as
// 2^Q(|h|), Q of degree 9 fitted for the least error over |h| = 0 .. 13.4, 2.4e-5 of the value (with fp32's rounding 3.4e-5 up to
// 11 and 4.5e-5 beyond).  One transcendental instead of two, which take as long as four other instructions each.  (Q falls
// on beyond the fit.)
__device__ __forceinline__ float gelu_tail(float h) {
  const float x = fabsf(h);
  float q = fmaf(-1.8374048948999189e-09f, x, 1.3548363142490416e-07f);
  q = fmaf(q, x, -4.38907682109857e-06f);
  q = fmaf(q, x, 8.267235534731299e-05f);
  q = fmaf(q, x, -0.001013598870486021f);
  q = fmaf(q, x, 0.008634578436613083f);
  q = fmaf(q, x, -0.053876444697380066f);
  q = fmaf(q, x, -0.45889127254486084f);
  q = fmaf(q, x, -1.1509331464767456f);
  q = fmaf(q, x, -1.0000337362289429f);
  const float above = __uint_as_float((uint32_t)max((int)__float_as_uint(h), 0));   // max(h, 0), without quieting a NaN first
  return fmaf(-x, __builtin_amdgcn_exp2f(q), above);
}
// The same and the derivative Phi(h) + h phi(h).  With x = |h|, t = 1 / (1 + 0.305 x), m = t P(t), P of degree 5:
//   Phi(-x) = m exp(-x^2 / 2),   Phi(-x) - x phi(x) = (m - x / sqrt(2 pi)) exp(-x^2 / 2), the derivative at -x (at x it is 1 - that).
// P is fitted over x = 0 .. 13.4 for the least relative error of both at once, which makes m exact where the second one is 0, at
// x = 0.7518: a fit for the value alone was off by 0.8 % of the derivative at -0.75.  (Of all bf16 h down to -13, which hold all that a
// stored h can be: 8.2e-6 of the value, 8.6e-6 of the derivative, and 5.9e-5 of it within 0.02 of its zero, from fp32's rounding of m.)
__device__ __forceinline__ void gelu_tail_and_grad(float h, float& val, float& grad) {
  const float x = fabsf(h), t = __builtin_amdgcn_rcpf(fmaf(0.305f, x, 1.0f));
  float p = fmaf(-0.0770023167f, t, 0.201740488f);
  p = fmaf(p, t, -0.00384007534f);
  p = fmaf(p, t, 0.140364885f);
  p = fmaf(p, t, 0.116739348f);
  p = fmaf(p, t, 0.121997997f);
  const float m = p * t, e = __builtin_amdgcn_exp2f(h * (h * (-0.5f * kLog2e)));
  val = fmaf(-x, m * e, fmaxf(h, 0.0f));
  const float below = fmaf(-0.3989422804014327f, x, m) * e;
  grad = h < 0.f ? below : 1.0f - below;
}
// Largest finite magnitude of 16 values.
template <typename V>
__device__ __forceinline__ float largest_of_16(const V& v) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) a = fmaxf(a, fabsf(v[i]));   // (a NaN is passed over)
  if (__builtin_expect(__ballot(!(a < __builtin_inff())) != 0, 0)) {
    a = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) a = fmaxf(a, finite_abs(v[i]));
  }
  return a;
}

// Sum over the wave, without the detour through LDS that a shuffle takes: 16 lanes by data-parallel moves (xor 1, 2, then the
// mirror images of 8 and 16 lanes), then the row and half-wave swaps.
template <int kCtrl>
__device__ __forceinline__ double moved(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_mov_dpp((int)(uint32_t)u, kCtrl, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), kCtrl, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double joined(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }
__device__ __forceinline__ double wave_sum(double x) {
  x += moved<0xb1>(x);    // quad_perm 1, 0, 3, 2
  x += moved<0x4e>(x);    // quad_perm 2, 3, 0, 1
  x += moved<0x141>(x);   // mirrored within 8 lanes
  x += moved<0x140>(x);   // mirrored within 16 lanes
  uint64_t u = __builtin_bit_cast(uint64_t, x);
  const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
  const auto b = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  x = joined(a[0], b[0]) + joined(a[1], b[1]);
  u = __builtin_bit_cast(uint64_t, x);
  const auto c = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
  const auto d = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return joined(c[0], d[0]) + joined(c[1], d[1]);
}

// GeLU in 64 bits, and its derivative: Phi(-|h|) = t P(t) exp(-x^2) / 2 with x = |h| / sqrt 2, t = 1 / (1 + 0.3 x) and P of degree 10 (4e-10
// of the value, and of Phi in the derivative), to decide between scales.
__device__ __forceinline__ double gelu64(double h, double* grad = nullptr) {
  const double x = fabs(h) * 0.70710678118654752440, t = 1.0 / fma(0.3, x, 1.0);
  double p = 0.055734015794935123;
  p = fma(p, t, -0.33301687949411679);
  p = fma(p, t, 0.74512765630325928);
  p = fma(p, t, -0.84218931949770892);
  p = fma(p, t, 0.77589148990779011);
  p = fma(p, t, -0.28565462890504778);
  p = fma(p, t, 0.26894751688341517);
  p = fma(p, t, 0.10941256579431252);
  p = fma(p, t, 0.16781163040879243);
  p = fma(p, t, 0.16865276238932064);
  p = fma(p, t, 0.16928319008836501);
  const double e = exp(-x * x), tail = 0.5 * p * t * e, cdf = h < 0.0 ? tail : 1.0 - tail;
  if (grad) *grad = cdf + h * 0.39894228040143267794 * e;
  return h * cdf;
}
// A value as a float that lies on the same side of the scales' borders, 448 * 2^e, which belong to the smaller one.
__device__ __forceinline__ float round_beside_border(double v) {
  const float f = (float)v;
  const uint32_t bits = __float_as_uint(f);
  return (bits & 0x7fffffu) == 0x600000u && fabs(v) > (double)fabsf(f) ? __uint_as_float(bits + 1) : f;
}

}  // namespace mb
