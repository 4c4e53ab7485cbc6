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

// What the waves of a workgroup leave for their join.
template <int D, int NB, int NW> struct FewShared { float o[NW][16 * NB][D]; float m[NW][16 * NB], l[NW][16 * NB]; };

// Workgroup `block` of those of one set of keys; with_logits: the logits are kept if a.logits asks for it.
template <typename ET, int D, int NB, int NW>
__device__ __forceinline__ void attend_few(const AttendArgs& a, const AttendKeys& k, int block, const bool with_logits, FewShared<D, NB, NW>& sm) {
  typedef FewTile<ET, D> Tile;
  constexpr int DB = Tile::DB, ROWS = 16 * NB;
  // which set of keys, tile of rows and range of keys
  const int split = block % k.nsplit;
  block /= k.nsplit;
  const int row_tile = block % k.row_tiles, set = block / k.row_tiles;
  const int h = set % a.H, ks = set / a.H;
  const int set_rows = k.row_samples * a.T * a.g;
  const int row0 = row_tile * ROWS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quad = lane >> 4;
  const int n = attend_len(k, ks, h), sink = attend_sink(k, ks, h);
  // (a message is not causal: its queries have no positions)
  const int pmin = n - a.T + row0 / a.g, pmax = n - a.T + (min(row0 + ROWS, set_rows) - 1) / a.g;
  const AttendSpan span = attend_span(k, n, sink, pmin, pmax);
  const int tiles = (span.count + 31) / 32, per = max(NW, (tiles + k.nsplit - 1) / k.nsplit);   // (a short head does not use all its ranges)
  const int first = split * per, behind = min(tiles, first + per);
  const bool joined = a.ranges > 1;
  const ET* K = (const ET*)k.K + ((size_t)ks * k.sample_rows + (size_t)h * k.stride) * D;
  const ET* V = (const ET*)k.V + ((size_t)ks * k.sample_rows + (size_t)h * k.stride) * D;

  typename Tile::Query q[NB];
  int pos[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const AttendRow w = attend_row(a, k, ks, min(row0 + 16 * nb + (lane & 15), set_rows - 1));
    Tile::load_query(q[nb], (const ET*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt, lane);
    pos[nb] = n - a.T + w.t;
  }
  f32x4 o[NB][DB];
  float m[NB], l[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = -INFINITY; l[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // A tile's logits are stored behind the next one's loads: the counter of outstanding accesses runs in order, and a wait for loads behind stores would wait
  // for those too.  (A message's weights are not asked for.)
  float* logits = a.logits && with_logits ? a.logits + ((size_t)set * a.logit_tiles * set_rows + (lane & 15)) * 32 + 4 * quad : nullptr;
  f32x4 held[NB][2];
  const auto keep = [&](const int i) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      if (16 * nb + (lane & 15) < set_rows) {
        float* at = logits + ((size_t)i * set_rows + 16 * nb) * 32;
        *(f32x4*)at = held[nb][0];
        *(f32x4*)(at + 16) = held[nb][1];
      }
  };
  int i = first + wave;
  for (; i < behind; i += NW) {
    const int base = 32 * i;
    typename Tile::Keys kf;
    typename Tile::Vals vf;
    Tile::load_keys(kf, K, span, base, lane);
    Tile::load_vals(vf, V, span, base, lane);
    if (logits && i > first + wave) keep(i - NW);
    const bool cut = attend_cut(k, span, sink, pmin, pmax, base, 32);
    float p[NB][2][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      f32x4 x[2];
      Tile::scores(x, kf, q[nb]);
      const AttendView view = attend_view(k, span, sink, pos[nb], base + 4 * quad);
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = x[b][r] * a.scale2;
          if (cut) v = attend_sees(view, 16 * b + r) ? v : -INFINITY;
          x[b][r] = v;
          mx = fmaxf(mx, v);
        }
      held[nb][0] = x[0]; held[nb][1] = x[1];
      if (__any(mx > m[nb] + kAttendSlack)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float next = fmaxf(m[nb], mx);
        const float f = next > -INFINITY ? attend_exp2(m[nb] - next) : 1.f;
        m[nb] = next;
        l[nb] *= f;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[nb][db] *= f;
      }
      const float ref = m[nb] > -INFINITY ? m[nb] : 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) { p[nb][b][r] = attend_exp2(x[b][r] - ref); l[nb] += p[nb][b][r]; }
    }
    // A product takes 0 times a hidden value; where that value is not finite, the tile's terms are added one by one instead.
    if (cut && k.causal && a.T > 1 && __any(Tile::not_finite(vf))) {
#pragma unroll 1
      for (int v = base; v < min(span.count, base + 32); ++v) {
        const ET* krow = K + few_row<D>(span, v);
        const ET* row = V + few_row<D>(span, v);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const AttendRow w = attend_row(a, k, ks, min(row0 + 16 * nb + (lane & 15), set_rows - 1));
          const ET* qrow = (const ET*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt;
          float dot = 0.f;
#pragma unroll 1
          for (int c = 0; c < D; ++c) dot = fmaf(Tile::value(krow, c), Tile::value(qrow, c), dot);
          if (attend_sees(attend_view(k, span, sink, pos[nb]), v)) {
            const float wt = attend_exp2(fmaf(dot, a.scale2, -(m[nb] > -INFINITY ? m[nb] : 0.f)));
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int c = 0; c < 4; ++c) o[nb][db][c] = fmaf(wt, Tile::value(row, Tile::channel(quad, db, c)), o[nb][db][c]);
          }
        }
      }
    } else {
      Tile::template values<NB>(o, vf, p);
    }
  }
  if (logits && i > first + wave) keep(i - NW);

  // the waves' parts
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    l[nb] += __shfl_xor(l[nb], 16);
    l[nb] += __shfl_xor(l[nb], 32);
    const int r = 16 * nb + (lane & 15);
    if (quad == 0) { sm.m[wave][r] = m[nb]; sm.l[wave][r] = l[nb]; }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) sm.o[wave][r][Tile::channel(quad, db, c)] = o[nb][db][c];
  }
  __syncthreads();
  constexpr int PIECES = D / 4;
  for (int e = threadIdx.x; e < ROWS * PIECES; e += NW * 64) {
    const int r = e / PIECES, c = (e % PIECES) * 4;
    if (row0 + r >= set_rows) break;
    float top = sm.m[0][r];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, sm.m[w][r]);
    const float ref = top > -INFINITY ? top : 0.f;
    float sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = attend_exp2(sm.m[w][r] - ref);
      sum = fmaf(f, sm.l[w][r], sum);
      const float4 x = *(const float4*)&sm.o[w][r][c];
      v[0] = fmaf(f, x.x, v[0]); v[1] = fmaf(f, x.y, v[1]); v[2] = fmaf(f, x.z, v[2]); v[3] = fmaf(f, x.w, v[3]);
    }
    // (a sum of 0: no key is visible; a sum that is no number: some visible logit is none, whatever `top` is)
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= inv;
    const float lse2 = sum != 0.f ? top + attend_log2(sum) : -INFINITY;
    const AttendRow w = attend_row(a, k, ks, row0 + r);
    const size_t number = attend_row_number(a, h, w);
    if (joined) {
      const size_t at = (size_t)(k.split0 + split) * a.rows + number;
      if (c == 0) a.part_lse[at] = lse2;
      if (sum != 0.f) *(float4*)(a.part_O + at * D + c) = make_float4(v[0], v[1], v[2], v[3]);   // (nobody reads the others)
    } else {
      if (c == 0 && a.lse) a.lse[number] = lse2 * 0.69314718055994531f;
      store4((ET*)a.O + (size_t)w.s * a.os + (size_t)(h * a.g + w.gi) * a.oh + (size_t)w.t * a.ot + c, v);
    }
  }
}

}  // namespace obf
