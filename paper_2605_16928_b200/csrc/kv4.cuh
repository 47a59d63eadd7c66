// The 4-bit K/V cache (rtp_cache.kv_format == RTP_KV_FP4).  A group of 16 channels of a token holds 16 codes E2M1 and one
// scale, an unsigned 8-bit float with 5 exponent and 3 mantissa bits (bias 15): an fp16 without its sign and its lower
// seven mantissa bits, so that code << 7 IS the scale's fp16 pattern, subnormals included.  A code has at most two
// significant bits and a scale four, so their product has six: it is exact in bf16, and in fp16 as long as the scale is at
// most 10240 (6 * 10240 = 61440 < 65504), the largest one that is written.
#pragma once

#include "rtp_device.cuh"

namespace rtp {

constexpr int kKv4Group = 16;                              // channels that share a scale
constexpr int kKv4TokBytes = kHeadDim / 2;                 // codes of a token: 64 bytes of K, 64 of V
constexpr int kKv4ScaleBytes = 2 * kHeadDim / kKv4Group;   // scales of a token: 8 of K, then 8 of V
constexpr float kKv4MaxScale = 10240.0f;
constexpr float kKv4MaxValue = 6.0f * kKv4MaxScale;

// t >= 0 -> scale code, nearest, ties to even.  (t = amax / 6 of bf16 values is never so close to a tie, without being one,
// that its own fp32 rounding could matter: amax differs from six times the tie by 2^-9 of it at least.)
__device__ __forceinline__ uint32_t kv4_scale_code(float t) {
  if (t < 6.103515625e-05f) return (uint32_t)__float2int_rn(t * 131072.0f);   // below 2^-14: multiples of 2^-17
  const uint32_t b = __float_as_uint(t);
  return ((b + 0x7ffffu + ((b >> 20) & 1u)) >> 20) - ((127u - 15u) << 3);
}
__device__ __forceinline__ float kv4_scale_value(uint32_t code) {
  return code < 8u ? (float)code * 7.62939453125e-06f : __uint_as_float((code + ((127u - 15u) << 3)) << 20);
}

// Two E2M1 codes of a byte (low half first) -> fp16x2, four bytes at a time.
__device__ __forceinline__ void e2m1x8_to_f16x2(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n"
      ".reg .b8 b0, b1, b2, b3;\n"
      "mov.b32 {b0, b1, b2, b3}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n"
      "}\n"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// Four pairs -> four bytes; the first of a pair goes to the low half.  Nearest, ties to even, saturating at 6.
__device__ __forceinline__ uint32_t f32_to_e2m1x8(const float (&x)[8]) {
  uint32_t w;
  asm("{\n"
      ".reg .b8 b0, b1, b2, b3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
      "mov.b32 %0, {b0, b1, b2, b3};\n"
      "}\n"
      : "=r"(w) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return w;
}

// Sixteen bf16 channels -> their codes and their scale.  Values beyond 61440 in magnitude saturate, a NaN is stored as 0;
// `bad` is set for either.
__device__ __forceinline__ uint2 kv4_encode(const uint4& lo, const uint4& hi, uint32_t& scale, bool& bad) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  uint32_t mx = 0;   // the magnitudes' bit patterns order like the magnitudes, two at a time
#pragma unroll
  for (int i = 0; i < 8; ++i) mx = __vmaxu2(mx, w[i] & 0x7fff7fffu);
  mx = max(mx & 0xffffu, mx >> 16);
  if (mx > 0x4770u) {   // 61440; infinities and NaN lie above it
    bad = true;
    mx = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int h = 0; h < 32; h += 16) {
        const uint32_t mag = (w[i] >> h) & 0x7fffu, put = mag > 0x7f80u ? 0u : min(mag, 0x4770u);
        w[i] = (w[i] & ~(0x7fffu << h)) | (put << h);
        mx = max(mx, put);
      }
    }
  }
  scale = kv4_scale_code(__fdiv_rn(__uint_as_float(mx << 16), 6.0f));
  // x / s as x * (inv + err), inv + err the reciprocal to 48 bits: the product with inv alone is off a tie by one bit for
  // scales of 15/8 * 2^n, the one below is exact at every tie
  const float s = kv4_scale_value(scale), inv = s > 0.f ? __frcp_rn(s) : 0.f, err = fmaf(-inv, s, 1.0f) * inv;
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = __uint_as_float((i & 1) ? (w[i >> 1] & 0xffff0000u) : (w[i >> 1] << 16));
    const float y = __uint_as_float((i & 1) ? (w[4 + (i >> 1)] & 0xffff0000u) : (w[4 + (i >> 1)] << 16));
    a[i] = fmaf(x, inv, x * err);
    b[i] = fmaf(y, inv, y * err);
  }
  return make_uint2(f32_to_e2m1x8(a), f32_to_e2m1x8(b));
}

}  // namespace rtp
