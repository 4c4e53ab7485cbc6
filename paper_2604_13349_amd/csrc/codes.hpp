// The row code: a lane's part of a row, 16 consecutive columns, to codes and back.
//
// Every row carries an asymmetric code of its own and two half-precision numbers, zero = fp16(min x), scale = fp16((max x - min x) / L), L = 2^bits - 1,
// q = clamp(rint((x - zero) / scale), 0, L), and stands for zero + scale q.  The integer decision is taken in single precision with individually rounded
// subtract, divide and round-to-even.
#pragma once
#include <hip/hip_fp16.h>
#include "common.hpp"
#include "wave_ops.hpp"

namespace obf {

constexpr int QT_THREADS = 256;
constexpr int QT_COLS = 16;              // columns per lane

// 16 consecutive elements (16-byte aligned) as floats.
__device__ __forceinline__ void load16(const uint16_t* __restrict__ p, float (&o)[QT_COLS]) {
  const uint4 v[2] = {((const uint4*)p)[0], ((const uint4*)p)[1]};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { o[8 * i + 2 * k] = __uint_as_float(w[k] << 16); o[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
  }
}
__device__ __forceinline__ void load16(const float* __restrict__ p, float (&o)[QT_COLS]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float4 v = ((const float4*)p)[i]; o[4 * i] = v.x; o[4 * i + 1] = v.y; o[4 * i + 2] = v.z; o[4 * i + 3] = v.w; }
}
// Eight consecutive ones.
__device__ __forceinline__ void store8(uint16_t* __restrict__ p, const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = (uint32_t)float_to_bf16_bits(x[2 * k]) | ((uint32_t)float_to_bf16_bits(x[2 * k + 1]) << 16);
  *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* __restrict__ p, const float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) ((float4*)p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
}

// Smallest and largest of the LPR neighbouring lanes of a row, in all of them.
template <int LPR> __device__ __forceinline__ void row_range(float& lo, float& hi) {
  static_assert(LPR == 4 || LPR == 8, "lanes of a row");
  const auto meet = [&](const uint32_t l, const uint32_t h) { lo = fminf(lo, __uint_as_float(l)); hi = fmaxf(hi, __uint_as_float(h)); };
  meet(OBF_DPP_MOV(__float_as_uint(lo), 0xB1), OBF_DPP_MOV(__float_as_uint(hi), 0xB1));                        // lane ^ 1
  meet(OBF_DPP_MOV(__float_as_uint(lo), 0x4E), OBF_DPP_MOV(__float_as_uint(hi), 0x4E));                        // lane ^ 2
  if (LPR == 8) meet(OBF_DPP_MOV(__float_as_uint(lo), 0x141), OBF_DPP_MOV(__float_as_uint(hi), 0x141));        // the other four of eight
}

// Codes of the 16 columns x of a row that LPR neighbouring lanes share, scale and zero as half-precision bits (the same in all of them).
template <int LPR, int BITS>
__device__ __forceinline__ void encode16(const float (&x)[QT_COLS], uint32_t (&w)[QT_COLS * BITS / 32], uint16_t& scale, uint16_t& zero) {
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < QT_COLS; ++i) { lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]); }
  row_range<LPR>(lo, hi);
  constexpr float L = (float)((1 << BITS) - 1);
  const __half zh = __float2half_rn(lo), sh = __float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), L));
  const float z = __half2float(zh), s = __half2float(sh);
  float q[QT_COLS];
  if (s > 0.f && s < INFINITY && fabsf(z) < INFINITY) {
    // The correctly rounded quotient t / s from r = RN(1 / s), in one step: y = RN(t r) is off by less than 2 ulp, t - y s is exact, since s has 11 significant bits, and
    // y + (t - y s) r is off by 2^-23 ulp.  From the middle between two floats t / s keeps 2^-12 ulp at least: it is a fraction over an integer below 2^11, and none itself,
    // since an odd number of 25 bits does not divide one of 24.  (Taking the product alone where it lies far enough from a tie, and two steps
    // elsewhere, which is often, since bf16 rows have many ties: 38.5 us for 37.7 to 4 bits, int4 rows 22.6 for 21.3.)
    const float r = __frcp_rn(s);
#pragma unroll
    for (int i = 0; i < QT_COLS; ++i) {
      const float t = __fsub_rn(x[i], z), y = __fmul_rn(t, r);
      q[i] = rintf(__builtin_amdgcn_fmed3f(__fmaf_rn(__fmaf_rn(-y, s, t), r, y), 0.f, L));
    }
  } else {                                                     // a constant row, or values past the half-precision range
#pragma unroll
    for (int i = 0; i < QT_COLS; ++i) q[i] = (s > 0.f) ? fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[i], z), s)), 0.f), L) : 0.f;
  }
#pragma unroll
  for (int k = 0; k < QT_COLS * BITS / 32; ++k) {              // little-endian: the even column of an int4 pair in the low half
    w[k] = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float byte = BITS == 8 ? q[4 * k + i] : fmaf(q[8 * k + 2 * i + 1], 16.f, q[8 * k + 2 * i]);
      w[k] = __builtin_amdgcn_cvt_pk_u8_f32(byte, i, w[k]);
    }
  }
  scale = __half_as_ushort(sh); zero = __half_as_ushort(zh);
}
template <int BITS>
__device__ __forceinline__ void decode16(const uint32_t (&w)[QT_COLS * BITS / 32], const uint16_t scale, const uint16_t zero, float (&x)[QT_COLS]) {
  const float s = __half2float(__ushort_as_half(scale)), z = __half2float(__ushort_as_half(zero));
#pragma unroll
  for (int i = 0; i < QT_COLS; ++i) x[i] = fmaf(s, (float)((w[i * BITS / 32] >> (i * BITS % 32)) & ((1u << BITS) - 1u)), z);
}

// A lane's codes of 16 consecutive columns, in one piece of 16 (8 bits) or 8 bytes.
template <int BITS> __device__ __forceinline__ void store_codes16(uint8_t* __restrict__ p, const uint32_t (&w)[QT_COLS * BITS / 32]) {
  if constexpr (BITS == 8) *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
  else *(uint2*)p = make_uint2(w[0], w[1]);
}

// The way back takes eight columns from 8 part on and eight of the row's other half, so that the lanes of a row store whole lines at a time (16 columns a lane in one piece
// leave every other 16 bytes of a line to the next store: 61 us for 52, codes of 8 bits 27 for 24; to codes it makes no difference).
template <int D, int BITS> __device__ __forceinline__ void load_codes_part(const uint8_t* __restrict__ row, const int part, uint32_t (&w)[QT_COLS * BITS / 32]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* p = row + i * (D / 2 * BITS / 8) + part * BITS;
    if constexpr (BITS == 8) { const uint2 v = *(const uint2*)p; w[2 * i] = v.x; w[2 * i + 1] = v.y; }
    else w[i] = *(const uint32_t*)p;
  }
}
template <int D, typename T> __device__ __forceinline__ void store_part(T* __restrict__ row, const int part, const float (&x)[QT_COLS]) {
  store8(row + 8 * part, x);
  store8(row + D / 2 + 8 * part, x + 8);
}

}  // namespace obf
