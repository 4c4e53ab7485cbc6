// Attention of many query rows per KV head over a cache held in codes, bf16: prompts.
//
// The scheme is that of attend_tile: 128 query rows a workgroup, 32 a wave, tiles of 64 rows in LDS, K Q^T, the terms 2^(x - m), V^T P^T with P as the first
// product left it.  What comes from memory are codes: a thread takes a quarter of a row, makes half-precision numbers of them and stores those where the kernel of rows has
// its rows; the next tile's codes are on their way while one is multiplied.  A code n becomes a number as 1024 + n, an OR, from which the rest is taken.
//   K: whole numbers n, code less the middle one c, which the products take exactly; x = scale (q . n) + (zero + c scale) sum(q): a multiplication per logit, and the
//      second term by one more product, of zero and scale with three parts of sum(q), 33 bits.  So logits, and lse, are single precision (values rounded to half
//      precision would be 2^-11 off, lse 1e-3).
//   V: values zero + scale * code, rounded once, 2^-11 of the value, where the result is rounded to 2^-8.
// With 4 bits the eight channels of a word lie in LDS in the order 0 4 1 5 2 6 3 7, in which the masks leave them; Q follows it, and O's rows are put in order at the end.
// Q enters as half-precision numbers under a power of two per row, bf16 exactly but for elements 2^-39 of the largest; the weights as half-precision numbers
// of 11 bits, the largest between 2^7 and 2^15.
// A row of V whose numbers are none is stored as zeros and its tile marked: whoever sees it gets no number, whoever does not, nothing of it.
//
// Every workgroup of a head makes the numbers anew.  Where there are many (ROWS), a kernel of its own makes them once, and the tiles come straight to LDS.
//
// Bound by power with long prompts: 4096 queries of 32 heads over 8 heads of 13517 rows of 128, 4 bits, 789 us at best and 841 on average of 30 in a row (0.92 to 0.98 PFLOP/s, the
// matrix pipe busy for 0.48 and the vector pipe for 0.55 of the time, together 0.83, at 1.8 to 1.9 GHz) and 18 for the rows' numbers (73 MB, 4.0 TB/s); with a window of 1024, 2000
// queries of 32 heads over 4 x 8 heads of 4000 to 6000 rows, 4 bits, 202 to 220 us (0.61 to 0.67 PFLOP/s of visible pairs) and 16 for the numbers.  By the longest heads where their
// lengths differ: 500 queries of 40 heads over 3 x 8 heads of 700 to 2139 rows of 64, 8 bits, 51 us, one wave a SIMD on average, and 8 for the numbers.  No gain: the logits a tile
// ahead of the weights (815 - 810 us; 32 row tiles over 8 heads of 8000 rows 192 - 212); two groups of waves on alternate tiles, joined in LDS (829 - 864; 59 - 60; 192 - 163).
#include "attend_codes.hpp"
#include "attend_tile.hpp"

namespace obf {

constexpr float kTileTop = 7.f;               // the reference's weight is 2^7

// Eight codes less `less` as half-precision numbers.
template <int BITS>
__device__ __forceinline__ void code_numbers(CodeFrag& f, const uint32_t* w, const float less) {
  const _Float16 b = (_Float16)(-1024.f - less);
  const f16x2 bias = {b, b};
  if constexpr (BITS == 4) {
    const _Float16 b16 = (_Float16)(-64.f - less);
    const f16x2 up = {(_Float16)0.0625f, (_Float16)0.0625f}, bias16 = {b16, b16};
    const uint32_t x = w[0], y = x >> 8;
    f.w[0] = (x & 0x000f000fu) | 0x64006400u; f.w[1] = (x & 0x00f000f0u) | 0x64006400u;
    f.w[2] = (y & 0x000f000fu) | 0x64006400u; f.w[3] = (y & 0x00f000f0u) | 0x64006400u;
    f.h[0] += bias; f.h[2] += bias;
    f.h[1] = __builtin_elementwise_fma(f.h[1], up, bias16);
    f.h[3] = __builtin_elementwise_fma(f.h[3], up, bias16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f.w[i] = __builtin_amdgcn_perm(0x64646464u, w[i >> 1], (i & 1) ? 0x04030402u : 0x04010400u);
      f.h[i] += bias;
    }
  }
}
__device__ __forceinline__ _Float16 half_of(const uint16_t x) { union { uint16_t u; _Float16 f; } y; y.u = x; return y.f; }
// What a logit takes of a row of K: its scale with kTileUnit taken out, and its zero and scale as they are.  An infinite one makes the first none: by itself it would hide the key
// from the queries whose sums have one sign.
constexpr float kTileUnit = 16384.f;          // sum(q) under q's power of two, 2^22 at most, times the middle code is a half-precision number with this taken out
__device__ __forceinline__ uint2 key_numbers(const uint16_t scale, const uint16_t zero) {
  const float s = (float)half_of(scale), z = (float)half_of(zero);
  return make_uint2(__float_as_uint(fmaf(0.f, s + z, s * (1.f / kTileUnit))), (uint32_t)scale << 16 | zero);
}

// Eight of V's values, zero + scale * code.
template <int BITS>
__device__ __forceinline__ void code_values(CodeFrag& f, const uint32_t* w, const _Float16 scale, const _Float16 zero) {
  code_numbers<BITS>(f, w, 0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) f.h[i] = __builtin_elementwise_fma(f.h[i], f16x2{scale, scale}, f16x2{zero, zero});
}
// The same past the half-precision range, as its ends, and of a row without numbers, as zeros.
__device__ __forceinline__ void code_clamp(CodeFrag& f, const bool none) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = none ? (_Float16)0.f : (_Float16)fminf(fmaxf((float)f.v[e], -65504.f), 65504.f);
}
// Largest magnitude that a row's numbers allow, or none.
template <int BITS> __device__ __forceinline__ float code_reach(const _Float16 scale, const _Float16 zero) {
  return fmaf(fabsf((float)scale), (float)((1 << BITS) - 1), fabsf((float)zero));
}

// The numbers of all rows that some query sees, 16 columns a lane, in the order of code_numbers.
constexpr int CR_THREADS = 256;
template <int D, int BITS>
__global__ __launch_bounds__(CR_THREADS) void k_codes_rows(const AttendCodesArgs args) {
  constexpr int LANES = D / 16, BYTES = D * BITS / 8, PER = CR_THREADS / LANES, PASSES = kCodeFlagRows / PER, WORDS = BITS / 2;
  static_assert(PER * PASSES == kCodeFlagRows, "a flag per workgroup");
  const AttendArgs& a = args.a;
  const AttendKeys& k = a.keys[0];
  const int set = blockIdx.x / args.flags, block = blockIdx.x % args.flags, h = set % a.H, s = set / a.H;
  const int n = attend_len(k, s, h), sink = attend_sink(k, s, h), part = threadIdx.x % LANES;
  if (block * kCodeFlagRows >= n) return;
  const size_t head = (size_t)s * k.sample_rows + (size_t)h * k.stride;
  bool bad = false;
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    const int j = block * kCodeFlagRows + pass * PER + threadIdx.x / LANES;
    if (j >= n || (k.causal && k.window > 0 && j <= n - a.T - k.window && j >= sink)) continue;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const CodeRows& c = which ? args.v : args.k;
      const uint8_t* from = c.codes + (head + j) * BYTES + part * (BYTES / LANES);
      uint32_t w[WORDS];
      if constexpr (WORDS == 2) { const uint2 x = *(const uint2*)from; w[0] = x.x; w[1] = x.y; }
      else { const uint4 x = *(const uint4*)from; w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w; }
      const _Float16 scale = half_of(c.scale[head + j]), zero = half_of(c.zero[head + j]);
      const float reach = code_reach<BITS>(scale, zero);
      const bool none = !(reach < INFINITY);
      const size_t row = (size_t)set * k.stride + j;
      if (which) bad |= none;
      else if (part == 0) args.numbers[row] = key_numbers(c.scale[head + j], c.zero[head + j]);
      uint16_t* to = (which ? args.rows_v : args.rows_k) + row * D + part * 16;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        CodeFrag f;
        if (which) {
          code_values<BITS>(f, w + p * (BITS / 4), scale, zero);
          if (!(reach < 65504.f)) code_clamp(f, none);
        } else code_numbers<BITS>(f, w + p * (BITS / 4), code_middle(BITS));
        *(uint4*)(to + 8 * p) = make_uint4(f.w[0], f.w[1], f.w[2], f.w[3]);
      }
    }
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) args.bad[(size_t)set * args.flags + block] = bad;
}

// As attend_set, but the tiles of one number of all sets follow one another: where causal heads have many of them, the last and longest of all heads run first and share their
// compute units with the first ones (us, set after set and tile after tile: 3 x 8 heads of 2139 rows of 64, 32 tiles, 86 - 75, 2 x 8 of 128 92 - 84, 4 x 8 of 1000 to 2000
// 95 - 80; heads of few tiles lose their second-level cache: 16 x 8 of 600 to 8000 rows, 7 tiles, 465 - 513).  A die's 32 compute units take its workgroups in turn, so that
// where its sets divide them they move on by one a turn: tiles of one set, of which a head may be longer than the others, would meet on the same ones (138 - 146 - 131).
constexpr int kDieCU = 32;
__device__ __forceinline__ int attend_set_by_tile(const int block, const int sets, int& within) {
  const int round = sets & 7 ? sets & -sets : 8, groups = sets / round, at = block / round;
  const int group = (at + (kDieCU % groups ? 0 : at / kDieCU)) % groups;
  within = at / groups;
  return group * round + (block + group) % round;
}

template <int D> struct CodeTileShared {
  char rows[4 * AT_KEYS * D * 2];             // K, K, V, V
  float scale[2][AT_KEYS];                    // of K, key_numbers
  uint32_t both[2][AT_KEYS];
  int marked[2];                              // the tile, plus one, that a buffer last held a row of V without numbers in
};

template <int D, int BITS, bool ROWS>
__global__ __launch_bounds__(AT_THREADS, D == 64 && (ROWS || BITS == 4) ? 3 : 2) void k_attend_codes_tile(const AttendCodesArgs args) {
  constexpr int KK = D / 16, DB = D / 32, TILE = AT_KEYS * D * 2, BYTES = D * BITS / 8, WORDS = BYTES / 16, PIECES = D / 32;
  static_assert(AT_THREADS == 4 * AT_KEYS, "a quarter of a row per thread");
  __shared__ __attribute__((aligned(1024))) CodeTileShared<D> sm;
  const AttendArgs& a = args.a;
  const AttendKeys& k = a.keys[0];
  int within;
  const int set = ROWS ? attend_set_by_tile(blockIdx.x, k.samples * a.H, within) : attend_set(blockIdx.x, k.samples * a.H, k.row_tiles * k.nsplit, within);
  const int split = within % k.nsplit, row_tile = k.row_tiles - 1 - within / k.nsplit;
  const int h = set % a.H, s = set / a.H;
  const int set_rows = a.T * a.g, row0 = row_tile * AT_ROWS;
  const int lane = threadIdx.x & 63, wave = attend_uniform(threadIdx.x >> 6), half = lane >> 5;
  const int n = attend_uniform(attend_len(k, s, h)), sink = attend_uniform(attend_sink(k, s, h));
  const int pmin = n - a.T + row0 / a.g, pmax = n - a.T + (min(row0 + AT_ROWS, set_rows) - 1) / a.g;
  const AttendSpan span = attend_span(k, n, sink, pmin, pmax);
  const int tiles = (span.count + AT_KEYS - 1) / AT_KEYS, per = (tiles + k.nsplit - 1) / k.nsplit;
  const int first = split * per, behind = min(tiles, first + per);
  const size_t head = (size_t)s * k.sample_rows + (size_t)h * k.stride;
  if (threadIdx.x < 2) sm.marked[threadIdx.x] = 0;
  bool look = false;                                   // whether some row of the head, if ROWS, has no numbers
  if constexpr (ROWS) for (int b = threadIdx.x; b * kCodeFlagRows < n; b += AT_THREADS) look |= args.bad[(size_t)set * args.flags + b] != 0;
  look = __syncthreads_or(look);
  const uint16_t *rows_k = args.rows_k + (size_t)set * k.stride * D, *rows_v = args.rows_v + (size_t)set * k.stride * D;

  // Q in the order of the values in LDS
  const int r = row0 + wave * 32 + (lane & 31);
  const AttendRow w = attend_row(a, k, s, min(r, set_rows - 1));
  const uint16_t* qrow = (const uint16_t*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt;
  const int pos = n - a.T + w.t;
  CodeFrag q[KK], qsum;
  float scale2;
  {
    TilePiece raw[KK];
    float top = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      raw[kk] = *(const TilePiece*)(qrow + 16 * kk + 8 * half);
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(raw[kk][i] << 16)), fabsf(__uint_as_float(raw[kk][i] & 0xffff0000u))));
    }
    top = fmaxf(top, __shfl_xor(top, 32));
    const float up = query_power(top, scale2);
    scale2 *= a.scale2 * kTileUnit;
    float sum = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = BITS == 4 ? (e >> 1) + 4 * (e & 1) : e;
        const uint32_t bits = raw[kk][c >> 1];
        const float x = __uint_as_float((c & 1) ? bits & 0xffff0000u : bits << 16) * up;
        q[kk].v[e] = (_Float16)x;
        sum += x;
      }
    // three parts of the sum, and as often the middle code, against a row's zero and scale: elements 0 .. 5 of 16
    sum = (sum + __shfl_xor(sum, 32)) * (1.f / kTileUnit);
    _Float16 part[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) { part[i] = (_Float16)sum; sum -= (float)part[i]; }
#pragma unroll
    for (int e = 0; e < 8; ++e) qsum.v[e] = half || e >= 6 ? (_Float16)0.f : e < 3 ? part[e] : part[e - 3] * (_Float16)code_middle(BITS);
  }

  // lane's places
  int at_k[KK], at_v[DB];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) at_k[kk] = place_k<D>(lane & 31, 2 * kk + half);
  const int vrow = 4 * half + ((lane & 15) >> 2);
#pragma unroll
  for (int db = 0; db < DB; ++db) at_v[db] = vrow * 2 * D + ((db ^ swap_v<D>(vrow)) << 6) + ((lane & 16) << 1) + ((lane & 3) << 3);

  // A thread's quarter row of a tile, as codes.
  const int row = threadIdx.x >> 2, part = threadIdx.x & 3;
  struct Codes { uint32_t k[WORDS], v[WORDS]; uint16_t ks, kz, vs, vz; };
  const auto load = [&](Codes& c, const int i) {
    const int v = min(AT_KEYS * i + row, span.count - 1);
    const size_t at = head + attend_key(span, v);
    const uint8_t *kp = args.k.codes + at * BYTES + part * (BYTES / 4), *vp = args.v.codes + at * BYTES + part * (BYTES / 4);
    if constexpr (WORDS == 2) {
      const uint2 x = *(const uint2*)kp, y = *(const uint2*)vp;
      c.k[0] = x.x; c.k[1] = x.y; c.v[0] = y.x; c.v[1] = y.y;
    } else {
#pragma unroll
      for (int j = 0; j < WORDS / 4; ++j) {
        const uint4 x = ((const uint4*)kp)[j], y = ((const uint4*)vp)[j];
        c.k[4 * j] = x.x; c.k[4 * j + 1] = x.y; c.k[4 * j + 2] = x.z; c.k[4 * j + 3] = x.w;
        c.v[4 * j] = y.x; c.v[4 * j + 1] = y.y; c.v[4 * j + 2] = y.z; c.v[4 * j + 3] = y.w;
      }
    }
    c.ks = args.k.scale[at]; c.kz = args.k.zero[at]; c.vs = args.v.scale[at]; c.vz = args.v.zero[at];
  };
  const auto put_numbers = [&](const int buf, const int at, const uint2 x) { sm.scale[buf][at] = __uint_as_float(x.x); sm.both[buf][at] = x.y; };
  // Tile i, to buffer buf.
  const auto store = [&](const Codes& c, const int buf, const int i) {
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const _Float16 scale = half_of(which ? c.vs : c.ks), zero = half_of(which ? c.vz : c.kz);
      CodeFrag f[PIECES];
      if (which) {
        const float reach = code_reach<BITS>(scale, zero);
        const bool past = !(reach < 65504.f), none = !(reach < INFINITY);
        if (none) sm.marked[buf] = i + 1;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) code_values<BITS>(f[p], c.v + p * (BITS / 4), scale, zero);
        if (__any(past) && past)
#pragma unroll
          for (int p = 0; p < PIECES; ++p) code_clamp(f[p], none);
      } else {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) code_numbers<BITS>(f[p], c.k + p * (BITS / 4), code_middle(BITS));
        if (part == 0) put_numbers(buf, row, key_numbers(c.ks, c.kz));
      }
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int piece = part * PIECES + p;
        char* at = sm.rows + (which ? 2 + buf : buf) * TILE;
        at += which ? row * 2 * D + (((piece >> 2) ^ swap_v<D>(row)) << 6) + ((piece & 3) << 4) : place_k<D>(row, piece);
        *(uint4*)at = make_uint4(f[p].w[0], f[p].w[1], f[p].w[2], f[p].w[3]);
      }
    }
  };

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
  float m = -INFINITY, l = 0.f;

  // One tile.  CUT: with the masks.
  const auto take = [&](const auto tag, const int buf, const int i) {
    constexpr bool CUT = decltype(tag)::value;
    const char *tk = sm.rows + buf * TILE, *tv = sm.rows + (2 + buf) * TILE;
    const int base = AT_KEYS * i;
    f32x16 x[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      CodeFrag kf[KK];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const TilePiece y = *(const TilePiece*)(tk + b * 32 * 2 * D + at_k[kk]);
#pragma unroll
        for (int e = 0; e < 4; ++e) kf[kk].w[e] = y[e];
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) x[b][e] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[kk].v, q[kk].v, x[b], 0, 0, 0);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 scale = *(const float4*)&sm.scale[buf][32 * b + 8 * g + 4 * half];
        x[b][4 * g] *= scale.x; x[b][4 * g + 1] *= scale.y; x[b][4 * g + 2] *= scale.z; x[b][4 * g + 3] *= scale.w;
      }
      const uint32_t both = half ? 0u : sm.both[buf][32 * b + (lane & 31)];
      CodeFrag rest;
      rest.w[0] = __builtin_amdgcn_perm(both, both, 0x01000100u); rest.w[1] = both; rest.w[2] = __builtin_amdgcn_perm(both, both, 0x03020302u); rest.w[3] = 0u;
      x[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(rest.v, qsum.v, x[b], 0, 0, 0);
    }
    const AttendView view = attend_view(k, span, sink, pos, base + 4 * half);
    if (CUT) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[b][e] = 32 * b + 8 * (e >> 2) + (e & 3) <= view.hi ? x[b][e] : -INFINITY;
      if (k.causal && k.window > 0 && base <= pmax - k.window - span.skip)
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
    const float mx = tile_max(tile_max(top[0], top[1]), tile_max(top[2], top[3])) * scale2;
    if (__any(mx > m + kAttendSlack)) {
      const float next = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32)));
      const float down = next > -INFINITY ? attend_exp2(m - next) : 1.f;
      m = next;
      l *= down;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] *= down;
    }
    const float ref = m > -INFINITY ? m - kTileTop : 0.f;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      x[0][e] = attend_exp2(fmaf(x[0][e], scale2, -ref));
      x[1][e] = attend_exp2(fmaf(x[1][e], scale2, -ref));
      s0 += x[0][e]; s1 += x[1][e];
    }
    l += s0 + s1;
    if (ROWS ? look : sm.marked[buf] == i + 1) {
      // some row of V has no numbers
#pragma unroll 1
      for (int e = 0; e < min(AT_KEYS, span.count - base); ++e) {
        const size_t at = head + attend_key(span, base + e);
        if (!(code_reach<BITS>(half_of(args.v.scale[at]), half_of(args.v.zero[at])) < INFINITY) && (!CUT || attend_sees(view, e - 4 * half)))
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int c = 0; c < 16; ++c) o[db][c] = NAN;
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      CodeFrag p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p.v[e] = (_Float16)x[t >> 1][8 * (t & 1) + e];
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        union { s16x4 h[2]; f16x8 v; } v;
        v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tv + at_v[db] + t * 16 * 2 * D));
        v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tv + at_v[db] + (t * 16 + 8) * 2 * D));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v.v, p.v, o[db], 0, 0, 0);
      }
    }
  };

  // Every row of the workgroup sees all of the tiles from whole0 to whole1; the others are taken with their masks.
  int whole0 = 0, whole1 = span.count / AT_KEYS;
  if (k.causal) {
    whole1 = min(whole1, max(0, pmin - span.skip + 1) / AT_KEYS);
    if (k.window > 0) whole0 = max(0, pmax - k.window - span.skip + AT_KEYS) / AT_KEYS;
  }
  Codes codes;
  int i = first, buf = 0;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)sm.rows;
  const uint2* numbers = args.numbers + (size_t)set * k.stride;
  uint2 pair;                                          // of K's row `lane` of the next tile
  const auto load_number = [&](const int tile) { if (wave == 0) pair = numbers[attend_key(span, min(AT_KEYS * tile + lane, span.count - 1))]; };
  const auto fill = [&](const int to, const int tile) {
    tile_fill<D, false>(lds + to * TILE, rows_k, span, tile * AT_KEYS, wave, lane);
    tile_fill<D, true>(lds + (2 + to) * TILE, rows_v, span, tile * AT_KEYS, wave, lane);
  };
  if (first < behind) {
    if constexpr (ROWS) {
      load_number(first);
      fill(0, first);
      if (wave == 0) put_numbers(0, lane, pair);
      if (first + 1 < behind) load_number(first + 1);
    } else {
      load(codes, first);
      store(codes, 0, first);
      if (first + 1 < behind) load(codes, first + 1);
    }
  }
  // Tile i is there, nobody reads the other buffer any more: tile i + 1 goes there, the codes of tile i + 2 on their way.
  const auto begin = [&]() {
    if constexpr (ROWS) {
      wait_loads<0>();
      __syncthreads();
      if (i + 1 < behind) {
        if (wave == 0) put_numbers(buf ^ 1, lane, pair);
        fill(buf ^ 1, i + 1);
      }
      if (i + 2 < behind) load_number(i + 2);
    } else {
      __syncthreads();
      if (i + 1 < behind) store(codes, buf ^ 1, i + 1);
      if (i + 2 < behind) load(codes, i + 2);
    }
  };
  while (i < behind) {
    const int whole = min(behind, i >= whole0 ? whole1 : i);
    for (; i < whole; ++i, buf ^= 1) { begin(); take(TileCut<false>(), buf, i); }
    const int cut = min(behind, i < whole0 ? whole0 : behind);
    for (; i < cut; ++i, buf ^= 1) { begin(); take(TileCut<true>(), buf, i); }
  }

  l += __shfl_xor(l, 32);
  // four channels 8 g + 4 half .. of a group of eight, as they are numbered
  const auto four = [&](const int db, const int g, float (&y)[4]) {
    const float x[4] = {o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
    if constexpr (BITS == 4) {
      // lanes below 32 hold channels 0 4 1 5, those above 2 6 3 7
      const float u = __shfl_xor(half ? x[0] : x[1], 32), v = __shfl_xor(half ? x[2] : x[3], 32);
      y[0] = half ? u : x[0]; y[1] = half ? v : x[2]; y[2] = half ? x[1] : u; y[3] = half ? x[3] : v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = x[e];
    }
  };
  if (r >= set_rows) return;                           // (both lanes of a row)
  const bool any = l != 0.f;                           // some key is visible (or some visible logit no number)
  const float inv = any ? 1.f / l : 0.f;
  const float lse2 = any ? m - kTileTop + attend_log2(l) : -INFINITY;
  const size_t number = attend_row_number(a, h, w);
  if (a.ranges > 1) {
    const size_t at = (size_t)(k.split0 + split) * a.rows + number;
    if (half == 0) a.part_lse[at] = lse2;
    if (!any) return;                                  // (nobody reads the others)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float y[4];
        four(db, c, y);
        *(float4*)(a.part_O + at * D + 32 * db + 8 * c + 4 * half) = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
      }
  } else {
    if (half == 0 && a.lse) a.lse[number] = lse2 * 0.69314718055994531f;
    uint16_t* out = (uint16_t*)a.O + (size_t)w.s * a.os + (size_t)(h * a.g + w.gi) * a.oh + (size_t)w.t * a.ot;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float y[4];
        four(db, c, y);
        union { __bf16 b[4]; uint2 u; } z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z.b[e] = (__bf16)(any ? y[e] * inv : 0.f);
        *(uint2*)(out + 32 * db + 8 * c + 4 * half) = z.u;
      }
  }
}

template <int D, int BITS>
static void tile_launch(const AttendCodesArgs& c, hipStream_t st) {
  const dim3 grid(c.a.keys[0].blocks), threads(AT_THREADS);
  if (c.rows_k) {
    hipLaunchKernelGGL((k_codes_rows<D, BITS>), dim3(c.a.S * c.a.H * c.flags), dim3(CR_THREADS), 0, st, c);
    hipLaunchKernelGGL((k_attend_codes_tile<D, BITS, true>), grid, threads, 0, st, c);
  } else hipLaunchKernelGGL((k_attend_codes_tile<D, BITS, false>), grid, threads, 0, st, c);
}

obf_status_t launch_attend_codes_tile(const AttendCodesArgs& c, int d, int bits, hipStream_t st) {
  ProfScope prof(ST_ATTEND, st);
  if (d == 128) { if (bits == 4) tile_launch<128, 4>(c, st); else tile_launch<128, 8>(c, st); }
  else { if (bits == 4) tile_launch<64, 4>(c, st); else tile_launch<64, 8>(c, st); }
  return check_launch("attend codes");
}

}  // namespace obf
