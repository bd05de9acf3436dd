// The 4-bit form of the paged cache.  Per token, head and group of 32 features: codes 0 .. 15, a scale s and a zero z in bf16.  With
// lo and hi the group's extremes, s = bf16((hi - lo) x 1/15), z = bf16(lo - 16 s), code = rint((x - z) / s) - 16 clamped to 0 .. 15, and
// a code stands for bf16(s (16 + code) + z), rounded once.  16 + code is what the attention kernel finds most easily: 0x4180 | code << 3
// as bf16, so that two codes become two values by one logic instruction and one packed multiply-add.  Everything held is finite: NaN is
// stored as 0 and magnitudes above 2^124 as 2^124, so that a masked token cannot spoil a row (weight 0 times its value is 0).
//
// A page and kv head is one block of 20 head_dim bytes:
//   K codes   [16 tokens][head_dim / 8 words]   word: features 8i .. 8i+7, feature c at bits 3 + 4 (c / 2) + 16 (c % 2) on (mod 32): rotating
//                                               right by 4e leaves features 2e and 2e+1 at bits 3 .. 6 of the two halves
//   K scales  [16 tokens][head_dim / 32]        s | z << 16
//   V codes   [2][8][4][head_dim / 32 words]    token 8h + 2q + p, feature (head_dim / 8) g + 4w + e: word [h][g][q][w], bits 16p + 4e on
//   V scales  [head_dim / 32][4][2]             group, q, h: {s of p = 0, 1}, {z of p = 0, 1}
// which are the registers of a warp-level MMA's fragments (lane 4g + q) in the order that one wide load of a lane takes them.
#pragma once
#include "state.cuh"

namespace laser {

constexpr int kQ4Group = 32;
constexpr float kQ4Top = 0x1p124f, kQ4Least = 0x1p-100f;

__host__ __device__ constexpr int q4_block_bytes(int dh) { return 20 * dh; }
__host__ __device__ constexpr int q4_k_codes(int dh, int t, int word) { return t * (dh / 2) + 4 * word; }
__host__ __device__ constexpr int q4_k_scale(int dh, int t, int group) { return 8 * dh + (t * (dh / 32) + group) * 4; }
// the 16-bit piece of features 4 c4 .. 4 c4 + 3
__host__ __device__ constexpr int q4_v_codes(int dh, int t, int c4) {
  const int per = dh / 32, g = c4 / per, w = c4 % per;
  return 10 * dh + (((t >> 3) * 8 + g) * 4 + ((t & 7) >> 1)) * per * 4 + w * 4 + (t & 1) * 2;
}
// s; z is four bytes further
__host__ __device__ constexpr int q4_v_scale(int dh, int t, int group) {
  return 18 * dh + ((group * 4 + ((t & 7) >> 1)) * 2 + (t >> 3)) * 8 + (t & 1) * 2;
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t bf16_bits(float x) {
  const __nv_bfloat16 h = __float2bfloat16_rn(x);
  return uint32_t(*reinterpret_cast<const uint16_t*>(&h));
}
__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// Scale and zero of the group that eight lanes (aligned, four features each) hold.
struct Q4Scale { uint32_t s, z; };
// NaN to 0, magnitudes to 2^124; a warp that has neither passes by
__device__ __forceinline__ void q4_finite(float (&x)[4]) {
  const bool fine = fabsf(x[0]) <= kQ4Top && fabsf(x[1]) <= kQ4Top && fabsf(x[2]) <= kQ4Top && fabsf(x[3]) <= kQ4Top;
  if (__all_sync(0xffffffffu, fine)) return;
#pragma unroll
  for (int u = 0; u < 4; ++u) x[u] = x[u] == x[u] ? fminf(fmaxf(x[u], -kQ4Top), kQ4Top) : 0.f;
}
__device__ __forceinline__ Q4Scale q4_scale(const float (&x)[4]) {
  float lo = fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), hi = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
#pragma unroll
  for (int o = 1; o <= 4; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  Q4Scale q;
  q.s = bf16_bits(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f));      // (the step is part of the format: one product, not a division)
  if (bf16_value(q.s) < kQ4Least) q.s = 0;
  q.z = bf16_bits(__fsub_rn(lo, 16.f * bf16_value(q.s)));
  return q;
}
// 16 + the codes of four values.  The quotient is the rounded one's neighbour at most (31 x 2^-22); where that could decide between two
// codes the division itself is made.  Rounded by adding 1.5 x 2^23 (quotients are below 2^20: a group's range is a few of its largest
// magnitude's 2^-24 at least, z is off by 2^-9 of it): conversions have a quarter of the other instructions' rate, and with three a value
// they took half of the time of an append.
__device__ __forceinline__ void q4_codes(const float (&x)[4], const Q4Scale& q, float (&at)[4]) {
  constexpr float kRound = 12582912.f;
  const float s = bf16_value(q.s), z = bf16_value(q.z);
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  bool clear = true;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float v = __fmul_rn(__fsub_rn(x[u], z), inv);
    at[u] = __fsub_rn(__fadd_rn(v, kRound), kRound);
    clear = clear && fabsf(__fsub_rn(v, at[u])) < 0.5f - 4e-5f;
  }
  if (!clear) {
#pragma unroll
    for (int u = 0; u < 4; ++u) at[u] = __fsub_rn(__fadd_rn(__fdiv_rn(__fsub_rn(x[u], z), s), kRound), kRound);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) at[u] = q.s == 0 ? 16.f : fminf(fmaxf(at[u], 16.f), 31.f);
}
// two codes c, d given as 16 + c, 16 + d: c | d << 4 in the low byte, nothing in the next
__device__ __forceinline__ uint32_t q4_two(float c, float d) { return __float_as_uint(__fmaf_rn(16.f, d, c + (8388608.f - 272.f))); }
// What two codes c, d stand for, given as 16 + c, 16 + d: the bf16 numbers that the attention kernel makes of them, by the same instruction
// (rounded once: in fp32 first, a z far below s is lost where s (16 + c) is halfway between two bf16 numbers).
__device__ __forceinline__ uint32_t q4_held2(float c, float d, const Q4Scale& q) {
  const __nv_bfloat162 at = __floats2bfloat162_rn(c, d);                   // (whole numbers below 32)
  uint32_t v;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v) : "r"(*reinterpret_cast<const uint32_t*>(&at)), "r"(q.s | q.s << 16), "r"(q.z | q.z << 16));
  return v;
}
#endif

}  // namespace laser
