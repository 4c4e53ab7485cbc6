// Operands and places in LDS of the bf16 kernels of many query rows (v_mfma_f32_32x32x16_bf16, lane l: row l % 32, elements 8 (l / 32) .. + 7 of 16).
#pragma once
#include "attend.hpp"
#include "lds_load.hpp"

namespace obf {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t TilePiece;

union TileFrag { TilePiece u; bf16x8 v; s16x4 h[2]; uint32_t w[4]; };

// Places in a tile of rows of 2 D bytes.
template <int D> __device__ __forceinline__ int place_k(const int row, const int piece) {       // 16-byte pieces
  return row * 2 * D + ((piece ^ (D == 128 ? row & 15 : (row >> 1) & 7)) << 4);
}
template <int D> __device__ __forceinline__ int swap_v(const int row) { return D == 128 ? row & 3 : (row >> 1) & 1; }   // of 64-byte pieces

constexpr int AT_WAVES = 4, AT_THREADS = AT_WAVES * 64, AT_ROWS = AT_WAVES * 32, AT_KEYS = 64;
static_assert(AT_ROWS == kAttendTileRows, "rows of a workgroup's tile");

// Entries v .. v + 63 of a span (those behind it repeat the last one) of K, or of V, to LDS.
template <int D, bool VALUES>
__device__ __forceinline__ void tile_fill(const uint32_t lds, const uint16_t* X, const AttendSpan span, const int v, const int wave, const int lane) {
  constexpr int PIECES = D / 8, LOADS = AT_KEYS * PIECES / AT_THREADS, ROWS = AT_THREADS / PIECES;   // rows per load of the workgroup
  // offsets from the first entry: 32 bits without a sign, what the rows of a head span
  const int start = attend_uniform(attend_key(span, v)), jump = attend_uniform(v < span.split ? span.split - v : AT_KEYS);
  const int last = attend_uniform(span.count - 1 - v);
  const void* base = attend_uniform(X + (size_t)start * D);
  uint32_t off[LOADS];
  int rows[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int at = wave * 64 + lane, row = i * ROWS + at / PIECES, place = at % PIECES;
    off[i] = (VALUES ? place ^ (swap_v<D>(row) << 2) : place ^ (D == 128 ? row & 15 : (row >> 1) & 7)) * 16;
    rows[i] = row;
  }
  if (jump < AT_KEYS || last < AT_KEYS - 1) {
    const int skip = attend_uniform(span.skip);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) { const int r = min(rows[i], last); rows[i] = r + (r >= jump ? skip : 0); }
  }
#pragma unroll
  for (int i = 0; i < LOADS; ++i) off[i] += (uint32_t)rows[i] * (2u * D);
  load_to_lds(lds + wave * 1024, off, base);
}

template <bool CUT> struct TileCut { static constexpr bool value = CUT; };

// The larger one; where one is no number, whatever (its row is none then).  One instruction: fmaxf would first make its operands quiet.
__device__ __forceinline__ float tile_max(const float a, const float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }

template <int D> constexpr int attend_tile_bytes() { return 4 * AT_KEYS * D * 2; }     // K, K, V, V

// Workgroup `block` of those of one set of keys (with a.fused: the message's, then the own).  PARTS: bf16 parts of a weight in the product with V.
template <int D, int PARTS>
__device__ __forceinline__ void attend_tile(const AttendArgs& a, const AttendKeys& k, const int block, char* sm) {
  constexpr int KK = D / 16, DB = D / 32, TILE = AT_KEYS * D * 2;
  // set of keys, tile of rows and range of keys; the rows with the most keys first
  int within;
  const int set = attend_set(block, k.samples * a.H, k.row_tiles * k.nsplit, within);
  const int split = within % k.nsplit, row_tile = k.row_tiles - 1 - within / k.nsplit;
  const int h = set % a.H, ks = set / a.H;
  const int set_rows = k.row_samples * a.T * a.g;
  const int row0 = row_tile * AT_ROWS;
  const int lane = threadIdx.x & 63, wave = attend_uniform(threadIdx.x >> 6), half = lane >> 5;
  const int n = attend_uniform(attend_len(k, ks, h)), sink = attend_uniform(attend_sink(k, ks, h));
  const int pmin = n - a.T + row0 / a.g, pmax = n - a.T + (min(row0 + AT_ROWS, set_rows) - 1) / a.g;
  const AttendSpan span = attend_span(k, n, sink, pmin, pmax);
  const int front = a.fused ? attend_uniform(attend_len(a.keys[0], 0, h)) : 0, front_tiles = (front + AT_KEYS - 1) / AT_KEYS;
  const int tiles = front_tiles + (span.count + AT_KEYS - 1) / AT_KEYS, per = (tiles + k.nsplit - 1) / k.nsplit;
  const int first = split * per, behind = min(tiles, first + per);
  const uint16_t* K = (const uint16_t*)k.K + ((size_t)ks * k.sample_rows + (size_t)h * k.stride) * D;
  const uint16_t* V = (const uint16_t*)k.V + ((size_t)ks * k.sample_rows + (size_t)h * k.stride) * D;
  const uint16_t* FK = a.fused ? (const uint16_t*)a.keys[0].K + (size_t)h * a.keys[0].stride * D : K;
  const uint16_t* FV = a.fused ? (const uint16_t*)a.keys[0].V + (size_t)h * a.keys[0].stride * D : V;

  const int r = row0 + wave * 32 + (lane & 31);
  const AttendRow w = attend_row(a, k, ks, min(r, set_rows - 1));
  const uint16_t* qrow = (const uint16_t*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt;
  const int pos = n - a.T + w.t;
  TileFrag q[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) q[kk].u = *(const TilePiece*)(qrow + 16 * kk + 8 * half);

  f32x16 o[DB];
  float m, l;
  // A product takes 0 times a hidden value: one that is not finite makes a row's O no number, and the pass is repeated with care for those.
  int careful = 0;

  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)sm;
  // lane's places
  int at_k[KK], at_v[DB];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) at_k[kk] = place_k<D>(lane & 31, 2 * kk + half);
  const int vrow = 4 * half + ((lane & 15) >> 2);
#pragma unroll
  for (int db = 0; db < DB; ++db) at_v[db] = vrow * 2 * D + ((db ^ swap_v<D>(vrow)) << 6) + ((lane & 16) << 1) + ((lane & 3) << 3);

  // One tile.  CUT: with the masks.
  const auto take = [&](const auto tag, const char* tk, const char* tv, const AttendKeys& kt, const AttendSpan st, const int base) {
    constexpr bool CUT = decltype(tag)::value;
    f32x16 x[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      TileFrag kf[KK];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[kk].u = *(const TilePiece*)(tk + b * 32 * 2 * D + at_k[kk]);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[b][e] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk].v, q[kk].v, x[b], 0, 0, 0);
    }
    const AttendView view = attend_view(kt, st, sink, pos, base + 4 * half);
    if (CUT) {
      // (attend_sees in two steps, the second only where the window begins inside the tile)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[b][e] = 32 * b + 8 * (e >> 2) + (e & 3) <= view.hi ? x[b][e] : -INFINITY;
      if (kt.causal && kt.window > 0 && base <= pmax - kt.window - st.skip)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int j = 32 * b + 8 * (e >> 2) + (e & 3);
            x[b][e] = ((j > view.lo) | (j < view.first)) ? x[b][e] : -INFINITY;
          }
    }
    float top[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) top[c] = x[c >> 1][8 * (c & 1)];
#pragma unroll
    for (int e = 1; e < 8; ++e)
#pragma unroll
      for (int c = 0; c < 4; ++c) top[c] = tile_max(top[c], x[c >> 1][8 * (c & 1) + e]);
    const float mx = tile_max(tile_max(top[0], top[1]), tile_max(top[2], top[3])) * a.scale2;
    if (__any(mx > m + kAttendSlack)) {
      const float next = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32)));
      const float scale = next > -INFINITY ? attend_exp2(m - next) : 1.f;
      m = next;
      l *= scale;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] *= scale;
    }
    const float ref = m > -INFINITY ? m : 0.f;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      x[0][e] = attend_exp2(fmaf(x[0][e], a.scale2, -ref));
      x[1][e] = attend_exp2(fmaf(x[1][e], a.scale2, -ref));
      s0 += x[0][e]; s1 += x[1][e];
    }
    l += s0 + s1;
    if (CUT && careful && kt.causal) {
      // where a value is not finite, the tile's terms are added one by one
      bool bad = false;
      for (int e = lane; e < TILE / 16; e += 64) {
        const TilePiece y = *(const TilePiece*)(tv + e * 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) bad |= ((y[c] & 0x7f80u) == 0x7f80u) | ((y[c] & 0x7f800000u) == 0x7f800000u);
      }
      if (__any(bad)) {
#pragma unroll 1
        for (int e = base; e < min(st.count, base + AT_KEYS); ++e) {
          const uint16_t* krow = K + (size_t)attend_key(st, e) * D;
          const uint16_t* row = V + (size_t)attend_key(st, e) * D;
          float dot = 0.f;
#pragma unroll 1
          for (int c = 0; c < D; ++c) dot = fmaf(__uint_as_float((uint32_t)krow[c] << 16), __uint_as_float((uint32_t)qrow[c] << 16), dot);
          if (attend_sees(view, e - base - 4 * half)) {
            const float wt = attend_exp2(fmaf(dot, a.scale2, -ref));
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int c = 0; c < 16; ++c)
                o[db][c] = fmaf(wt, __uint_as_float((uint32_t)row[32 * db + 8 * (c >> 2) + 4 * half + (c & 3)] << 16), o[db][c]);
          }
        }
        return;
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      TileFrag p, rest;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = x[t >> 1][8 * (t & 1) + e];
        p.v[e] = (__bf16)w;
        if (PARTS == 2) rest.v[e] = (__bf16)(w - (float)p.v[e]);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        TileFrag v;
        v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tv + at_v[db] + t * 16 * 2 * D));
        v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tv + at_v[db] + (t * 16 + 8) * 2 * D));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v, p.v, o[db], 0, 0, 0);
        if (PARTS == 2) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v, rest.v, o[db], 0, 0, 0);
      }
    }
  };

  // Tile i: 64 entries of the message (the first front_tiles), then of the own span.  Every row of the workgroup sees all of the tiles from 0 to front_whole and
  // from whole0 to whole1; the others are taken with their masks.
  const AttendSpan front_span = {front, 0, 0};
  const int front_whole = front / AT_KEYS;
  int whole0 = front_tiles, whole1 = front_tiles + span.count / AT_KEYS;
  if (k.causal) {
    whole1 = min(whole1, front_tiles + max(0, pmin - span.skip + 1) / AT_KEYS);
    if (k.window > 0) whole0 += max(0, pmax - k.window - span.skip + AT_KEYS) / AT_KEYS;
  }
  const auto fill = [&](const int buf, const int i) {
    const uint16_t *from_k = K, *from_v = V;
    AttendSpan from = span;
    int v = (i - front_tiles) * AT_KEYS;
    if (i < front_tiles) { from_k = FK; from_v = FV; from = front_span; v = i * AT_KEYS; }
    tile_fill<D, false>(lds + buf * TILE, from_k, from, v, wave, lane);
    tile_fill<D, true>(lds + (2 + buf) * TILE, from_v, from, v, wave, lane);
  };
  int i, buf;
  // Tile i is there, nobody reads the other one any more: the loads of tile i + 1.
  const auto begin = [&]() {
    wait_loads<0>();
    __syncthreads();
    if (i + 1 < behind) fill(buf ^ 1, i + 1);
  };
  for (;; careful = 1) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
    m = -INFINITY; l = 0.f;
    i = first; buf = 0;
    if (first < behind) fill(0, first);
    // (two loops, so that the common one has the registers to itself)
    while (i < behind) {
      const int whole = min(behind, i < front_whole ? front_whole : i >= whole0 ? whole1 : i);
      for (; i < whole; ++i, buf ^= 1) {
        begin();
        take(TileCut<false>(), sm + buf * TILE, sm + (2 + buf) * TILE, k, span, 0);
      }
      // (none with masks where the message's whole tiles end at the first whole one of the own rows)
      const int cut = min(behind, i < front_tiles ? front_tiles : i < whole0 ? whole0 : i < whole1 ? i : behind);
      for (; i < cut; ++i, buf ^= 1) {
        AttendKeys kt = k;
        AttendSpan st = span;
        int v = (i - front_tiles) * AT_KEYS;
        if (i < front_tiles) { kt.causal = 0; kt.window = 0; st = front_span; v = i * AT_KEYS; }
        begin();
        take(TileCut<true>(), sm + buf * TILE, sm + (2 + buf) * TILE, kt, st, v);
      }
    }
    if (careful || !k.causal) break;
    bool bad = false;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) bad |= !(fabsf(o[db][e]) < INFINITY);
    if (!__syncthreads_or(bad)) break;                 // (also: nobody reads the tiles any more)
  }

  l += __shfl_xor(l, 32);
  if (r >= set_rows) return;
  const bool any = l != 0.f;                           // some key is visible (or some visible logit no number)
  const float inv = any ? 1.f / l : 0.f;
  const float lse2 = any ? m + attend_log2(l) : -INFINITY;
  const size_t number = attend_row_number(a, h, w);
  if (a.ranges > 1) {
    const size_t at = (size_t)(k.split0 + split) * a.rows + number;
    if (half == 0) a.part_lse[at] = lse2;
    if (!any) return;                                  // (nobody reads the others)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *(float4*)(a.part_O + at * D + 32 * db + 8 * c + 4 * half) =
            make_float4(o[db][4 * c] * inv, o[db][4 * c + 1] * inv, o[db][4 * c + 2] * inv, o[db][4 * c + 3] * inv);
  } else {
    if (half == 0 && a.lse) a.lse[number] = lse2 * 0.69314718055994531f;
    uint16_t* out = (uint16_t*)a.O + (size_t)w.s * a.os + (size_t)(h * a.g + w.gi) * a.oh + (size_t)w.t * a.ot;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        union { __bf16 b[4]; uint2 u; } y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y.b[e] = (__bf16)(any ? o[db][4 * c + e] * inv : 0.f);
        *(uint2*)(out + 32 * db + 8 * c + 4 * half) = y.u;
      }
  }
}

}  // namespace obf
