// Operands of a tile of 32 keys for the kernels whose waves read the caches straight into registers.
#pragma once
#include "attend.hpp"

namespace obf {

// Place of entry v of a span; entries behind it repeat the last one.
template <int D> __device__ __forceinline__ size_t few_row(const AttendSpan s, const int v) { return (size_t)attend_key(s, min(v, s.count - 1)) * D; }

template <typename ET, int D> struct FewTile;

// bf16: operands of v_mfma_f32_16x16x32_bf16, lane l: row l % 16, elements 8 (l / 16) .. + 7 of 32
template <int D> struct FewTile<uint16_t, D> {
  static constexpr int KV = D / 32;            // 16-byte pieces of a key (or query) row per lane
  static constexpr int DB = D / 16;            // blocks of 16 channels in O
  typedef __attribute__((__vector_size__(DB / 2 * sizeof(uint32_t)))) uint32_t vrow;   // channels DB i .. + DB - 1 of a row
  union Frag { uint4 u; bf16x8 v; };
  struct Keys { Frag k[2][KV]; };
  struct Vals { vrow v[2][4]; };
  struct Query { Frag q[KV]; };

  static __device__ __forceinline__ void load_query(Query& q, const uint16_t* row, const int lane) {
    const uint4* p = (const uint4*)row + (lane >> 4);
#pragma unroll
    for (int c = 0; c < KV; ++c) q.q[c].u = p[4 * c];
  }
  static __device__ __forceinline__ void load_keys(Keys& f, const uint16_t* K, const AttendSpan span, const int base, const int lane) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint4* p = (const uint4*)(K + few_row<D>(span, base + 16 * b + (lane & 15))) + (lane >> 4);
#pragma unroll
      for (int c = 0; c < KV; ++c) f.k[b][c].u = p[4 * c];
    }
  }
  static __device__ __forceinline__ void load_vals(Vals& f, const uint16_t* V, const AttendSpan span, const int base, const int lane) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        f.v[b][r] = *(const vrow*)(V + few_row<D>(span, base + 16 * b + 4 * (lane >> 4) + r) + DB * (lane & 15));
  }
  static __device__ __forceinline__ void scores(f32x4 (&x)[2], const Keys& k, const Query& q) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      x[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KV; ++c) x[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.k[b][c].v, q.q[c].v, x[b], 0, 0, 0);
    }
  }
  // O^T += V^T P^T of NB blocks of 16 query rows; p[nb][b][r]: key 16 b + 4 (lane / 16) + r
  template <int NB>
  static __device__ __forceinline__ void values(f32x4 (&o)[NB][DB], const Vals& f, const float (&p)[NB][2][4]) {
    bf16x8 hi[NB], lo[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = p[nb][e >> 2][e & 3];
        hi[nb][e] = (__bf16)x;
        lo[nb][e] = (__bf16)(x - (float)hi[nb][e]);
      }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const uint32_t sel = (db & 1) ? 0x07060302u : 0x05040100u;
      union { uint32_t u[4]; bf16x8 v; } a;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        a.u[2 * b] = __builtin_amdgcn_perm(f.v[b][1][db >> 1], f.v[b][0][db >> 1], sel);
        a.u[2 * b + 1] = __builtin_amdgcn_perm(f.v[b][3][db >> 1], f.v[b][2][db >> 1], sel);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, hi[nb], o[nb][db], 0, 0, 0);
        o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, lo[nb], o[nb][db], 0, 0, 0);
      }
    }
  }
  // an exponent of all ones among the lane's values
  static __device__ __forceinline__ bool not_finite(const Vals& f) {
    bool bad = false;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < DB / 2; ++i) bad |= ((f.v[b][r][i] & 0x7f80u) == 0x7f80u) | ((f.v[b][r][i] & 0x7f800000u) == 0x7f800000u);
    return bad;
  }
  static __device__ __forceinline__ float value(const uint16_t* row, const int c) { return __uint_as_float((uint32_t)row[c] << 16); }
  static __device__ __forceinline__ int channel(const int quad, const int db, const int r) { return DB * (4 * quad + r) + db; }
};

// fp32: operands of v_mfma_f32_16x16x4_f32, lane l: row l % 16, element l / 16 of 4
template <int D> struct FewTile<float, D> {
  static constexpr int KV = D / 16, DB = D / 16, VV = D / 64;
  struct Keys { f32x4 k[2][KV]; };
  struct Vals { f32x4 v[2][4][VV]; };
  struct Query { f32x4 q[KV]; };

  static __device__ __forceinline__ void load_query(Query& q, const float* row, const int lane) {
#pragma unroll
    for (int c = 0; c < KV; ++c) q.q[c] = *(const f32x4*)(row + 16 * c + 4 * (lane >> 4));
  }
  static __device__ __forceinline__ void load_keys(Keys& f, const float* K, const AttendSpan span, const int base, const int lane) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float* p = K + few_row<D>(span, base + 16 * b + (lane & 15)) + 4 * (lane >> 4);
#pragma unroll
      for (int c = 0; c < KV; ++c) f.k[b][c] = *(const f32x4*)(p + 16 * c);
    }
  }
  static __device__ __forceinline__ void load_vals(Vals& f, const float* V, const AttendSpan span, const int base, const int lane) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float* p = V + few_row<D>(span, base + 16 * b + 4 * (lane >> 4) + r) + 4 * (lane & 15);
#pragma unroll
        for (int c = 0; c < VV; ++c) f.v[b][r][c] = *(const f32x4*)(p + 64 * c);
      }
  }
  static __device__ __forceinline__ void scores(f32x4 (&x)[2], const Keys& k, const Query& q) {
#pragma unroll
    for (int b = 0; b < 2; ++b) x[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KV; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int b = 0; b < 2; ++b) x[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.k[b][c][e], q.q[c][e], x[b], 0, 0, 0);
  }
  template <int NB>
  static __device__ __forceinline__ void values(f32x4 (&o)[NB][DB], const Vals& f, const float (&p)[NB][2][4]) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.v[b][r][db >> 2][db & 3], p[nb][b][r], o[nb][db], 0, 0, 0);
  }
  static __device__ __forceinline__ bool not_finite(const Vals& f) {
    bool bad = false;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < VV; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) bad |= (__float_as_uint(f.v[b][r][c][e]) & 0x7f800000u) == 0x7f800000u;
    return bad;
  }
  static __device__ __forceinline__ float value(const float* row, const int c) { return row[c]; }
  static __device__ __forceinline__ int channel(const int quad, const int db, const int r) { return 64 * (db >> 2) + 4 * (4 * quad + r) + (db & 3); }
};

__device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4]) {
  union { __bf16 h[4]; uint2 u; } x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x.h[i] = (__bf16)v[i];
  *(uint2*)p = x.u;
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }

}  // namespace obf
