// Attention over a cache held in codes of 4 or 8 bits, few query rows per KV head (and any number of fp32 rows).
//
//   x_rj = (s_j q_r . c_j + z_j sum_c q_rc) / sqrt(d),  O_r = sum_j w_rj (s_j c_j + z_j),  w_rj = exp(x_rj - lse_r) over the visible rows j
//
// with c_j the codes of a row, s_j and z_j its scale and zero: the products are of whole numbers, the two numbers of a row come in where there is one value per row and
// query.  One pass over the codes: a wave takes tiles of 32 rows, holds the sum l of its query rows and O' = sum_j 2^(x_rj - m) (s_j c_j + z_j); waves and then
// ranges of a head are joined as in attend_few.hip, with the same lanes: K C^T leaves four rows of one query in a lane, the operand that V's product takes.
//
// A code n of 4 or 8 bits in the low bits of a half-precision number is n 2^-24, exactly (the matrix instructions take such numbers as they are): a mask
// is all that an operand needs, two codes at a time; codes four bits higher are 16 n 2^-24, which Q's elements, or O's at the end, take back.  So an operand of
// eight codes costs five instructions, and their order in it is Q's to follow.
// Q enters as half-precision numbers under a power of two per row, so that its largest lies in [2^14, 2^15): bf16 exactly but for elements 2^-39 of the largest, fp32
// as two parts of 11 bits.  The weights times s_j enter V's product as half-precision numbers of 11 bits (fp32: two parts): relative to a reference that follows the
// largest of 2^x_rj |s_j|, so that the largest product lies in [2^7, 2^15] whatever the scales are.  l, sum_j w z_j and O' are single precision.
#include "attend_codes.hpp"
#include "attend_few.hpp"
#include "codes.hpp"

namespace obf {

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
union CodeFrag { uint32_t w[4]; f16x8 v; };

constexpr float kCodeUnit = 16777216.f;       // 2^24: a code's number is code / kCodeUnit
constexpr float kCodeTop = 32768.f;           // largest weight times scale

template <int LANE> __device__ __forceinline__ float row_lane(const float x) {     // the value of lane LANE of the row of 16
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x150 + LANE, 0xF, 0xF, false));
}

// Operands of a tile of 32 rows.
template <int D, int BITS> struct CodeTile {
  static constexpr int KV = D / 32;                 // matrix instructions per block of 16 rows
  static constexpr int DB = D / 16;                 // blocks of 16 channels in O
  static constexpr int BYTES = D * BITS / 8;        // of a row
  static constexpr int KW = BYTES / 16;             // words of a K row per lane: a quarter of the row
  static constexpr int VB = BYTES / 16;             // bytes of a V row per lane: a sixteenth
  static constexpr int VW = VB < 4 ? 1 : VB / 4;
  struct Keys { uint32_t w[2][KW]; };
  struct Vals { uint32_t w[8][VW]; };

  // channel (of the lane's quarter row) and factor of element e of piece c
  static constexpr int channel(const int c, const int e) {
    return BITS == 4 ? 8 * c + (e >> 1) + 4 * (e & 1) : 8 * c + 4 * (e >> 2) + ((e >> 1) & 1) + 2 * (e & 1);
  }
  static constexpr float factor(const int e) { return BITS == 4 && ((e >> 1) & 1) ? 0.0625f : 1.f; }

  static __device__ __forceinline__ void load_key(uint32_t (&w)[KW], const uint8_t* p) {
    if constexpr (KW == 2) { const uint2 v = *(const uint2*)p; w[0] = v.x; w[1] = v.y; }
    else {
#pragma unroll
      for (int i = 0; i < KW / 4; ++i) {
        const uint4 v = ((const uint4*)p)[i];
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
    }
  }
  static __device__ __forceinline__ void load_val(uint32_t (&w)[VW], const uint8_t* p) {
    if constexpr (VB == 2) w[0] = *(const uint16_t*)p;
    else if constexpr (VB == 4) w[0] = *(const uint32_t*)p;
    else { const uint2 v = *(const uint2*)p; w[0] = v.x; w[1] = v.y; }
  }
  static __device__ __forceinline__ void key_piece(CodeFrag& f, const uint32_t (&w)[KW], const int c) {
    if constexpr (BITS == 4) {
      const uint32_t x = w[c], y = x >> 8;
      f.w[0] = x & 0x000f000fu; f.w[1] = x & 0x00f000f0u; f.w[2] = y & 0x000f000fu; f.w[3] = y & 0x00f000f0u;
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) { f.w[2 * i] = w[2 * c + i] & 0x00ff00ffu; f.w[2 * i + 1] = (w[2 * c + i] >> 8) & 0x00ff00ffu; }
    }
  }
  // channel block db of the eight rows, in pairs: rows 2 i and 2 i + 1
  static __device__ __forceinline__ void val_piece(CodeFrag& f, const Vals& v, const int db) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BITS == 4) {
        const uint32_t both = __builtin_amdgcn_perm(v.w[2 * i + 1][0], v.w[2 * i][0], db < 4 ? 0x05040100u : 0x07060302u);
        f.w[i] = ((db & 2) ? both >> 8 : both) & ((db & 1) ? 0x00f000f0u : 0x000f000fu);
      } else {
        f.w[i] = __builtin_amdgcn_perm(v.w[2 * i + 1][db >> 2], v.w[2 * i][db >> 2], 0x0c040c00u + (uint32_t)(db & 3) * 0x00010001u);
      }
    }
  }
  static constexpr float val_unit(const int db) { return BITS == 4 && (db & 1) ? kCodeUnit / 16.f : kCodeUnit; }
};

// Parts of a row of Q in the order of the K operands; the power of two, taken out, and the sum under it.
template <typename ET, int D, int BITS, int PARTS>
__device__ __forceinline__ void load_query(CodeFrag (&q)[PARTS][D / 32], float& unit, float& sum, const ET* row, const int quad) {
  typedef CodeTile<D, BITS> Tile;
  float x[D / 4];
  static_assert(D / 4 % QT_COLS == 0, "a quarter row in pieces of 16");
#pragma unroll
  for (int i = 0; i < D / 4 / QT_COLS; ++i) {
    float y[QT_COLS];
    load16(row + quad * (D / 4) + QT_COLS * i, y);
#pragma unroll
    for (int e = 0; e < QT_COLS; ++e) x[QT_COLS * i + e] = y[e];
  }
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) top = fmaxf(top, fabsf(x[i]));
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  // top in [2^(e - 1), 2^e), e from its bits (numbers below the normal ones as those next to them; an infinity: the largest ones' e)
  const int e = min(max((int)(__float_as_uint(top) >> 23) - 126, -125), 128);
  const float up = __uint_as_float((uint32_t)(min(127, 15 - e) + 127) << 23);      // 2^(15 - e), at most 2^127
  unit = __uint_as_float((uint32_t)(127 - min(127, 15 - e)) << 23 | (min(127, 15 - e) == 127 ? 0x00400000u : 0u));
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) { x[i] *= up; sum += x[i]; }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float y = x[Tile::channel(c, i)] * Tile::factor(i);
#pragma unroll
      for (int p = 0; p < PARTS; ++p) { q[p][c].v[i] = (_Float16)y; y -= (float)q[p][c].v[i]; }
    }
}

template <typename ET, int D, int BITS, int NB, int NW>
__global__ __launch_bounds__(NW * 64, 2) void k_attend_codes_few(const AttendCodesArgs args) {
  typedef CodeTile<D, BITS> Tile;
  constexpr int DB = Tile::DB, KV = Tile::KV, ROWS = 16 * NB, PARTS = sizeof(ET) == 4 ? 2 : 1, BYTES = Tile::BYTES;
  __shared__ __attribute__((aligned(16))) FewShared<D, NB, NW> sm;
  const AttendArgs& a = args.a;
  const AttendKeys& k = a.keys[0];
  const int split = blockIdx.x % k.nsplit, rest = blockIdx.x / k.nsplit;
  const int row_tile = rest % k.row_tiles, set = rest / k.row_tiles;
  const int h = set % a.H, s = set / a.H;
  const int set_rows = a.T * a.g, row0 = row_tile * ROWS;
  const int lane = threadIdx.x & 63, wave = attend_uniform(threadIdx.x >> 6), quad = lane >> 4, col = lane & 15;
  const int n = attend_uniform(attend_len(k, s, h)), sink = attend_uniform(attend_sink(k, s, h));
  const int pmin = n - a.T + row0 / a.g, pmax = n - a.T + (min(row0 + ROWS, set_rows) - 1) / a.g;
  const AttendSpan span = attend_span(k, n, sink, pmin, pmax);
  const int tiles = (span.count + 31) / 32, per = max(NW, (tiles + k.nsplit - 1) / k.nsplit);
  const int first = split * per, behind = min(tiles, first + per);
  const size_t head = (size_t)s * k.sample_rows + (size_t)h * k.stride;
  const uint8_t *kc = args.k.codes + head * BYTES, *vc = args.v.codes + head * BYTES;
  // lanes 0 .. 7 of a row of 16 hold the numbers of K's rows that the row's scores are of (4 quad + 0 .. 3 and 16 more), lanes 8 .. 15 those of V's
  const bool of_v = col & 8;
  const int num_row = 16 * ((col >> 2) & 1) + 4 * quad + (col & 3);
  const uint16_t *scales = (of_v ? args.v.scale : args.k.scale) + head, *zeros = (of_v ? args.v.zero : args.k.zero) + head;
  const float scale_unit = of_v ? 1.f : a.scale2 * kCodeUnit, zero_unit = of_v ? 1.f : a.scale2;

  CodeFrag q[NB][PARTS][KV];
  float qunit[NB], qsum[NB];
  int pos[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const AttendRow w = attend_row(a, k, s, min(row0 + 16 * nb + col, set_rows - 1));
    load_query<ET, D, BITS, PARTS>(q[nb], qunit[nb], qsum[nb], (const ET*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt, quad);
    pos[nb] = n - a.T + w.t;
  }
  f32x4 o[NB][DB];
  float m[NB], l[NB], zsum[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = -INFINITY; l[nb] = 0.f; zsum[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int i = first + wave; i < behind; i += NW) {
    const int base = 32 * i;
    typename Tile::Keys kf;
    typename Tile::Vals vf;
    uint16_t num_s, num_z;
    // rows of the tile, relative to its first entry's: the place of an entry in the span, the last one's behind it
    const int start = attend_key(span, base), jump = base < span.split ? span.split - base : 32, last = span.count - 1 - base;
    const uint8_t *kt = kc + (size_t)start * BYTES, *vt = vc + (size_t)start * BYTES;
    const uint16_t *st = scales + start, *zt = zeros + start;
    const auto load = [&](const auto place) {
#pragma unroll
      for (int b = 0; b < 2; ++b) Tile::load_key(kf.w[b], kt + ((uint32_t)place(16 * b + col) * BYTES + quad * (BYTES / 4)));
      num_s = st[(uint32_t)place(num_row)];
      num_z = zt[(uint32_t)place(num_row)];
#pragma unroll
      for (int e = 0; e < 8; ++e) Tile::load_val(vf.w[e], vt + ((uint32_t)place(16 * (e >> 2) + 4 * quad + (e & 3)) * BYTES + col * (BYTES / 16)));
    };
    if (jump >= 32 && last >= 31) load([](const int r) { return r; });
    else load([&](const int r) { const int x = min(r, last); return x + (x >= jump ? span.skip : 0); });
    const bool cut = attend_cut(k, span, sink, pmin, pmax, base, 32);

    const float num_scale = __half2float(__ushort_as_half(num_s)) * scale_unit, num_zero = __half2float(__ushort_as_half(num_z)) * zero_unit;
    const float sk[8] = {row_lane<0>(num_scale), row_lane<1>(num_scale), row_lane<2>(num_scale), row_lane<3>(num_scale),
                         row_lane<4>(num_scale), row_lane<5>(num_scale), row_lane<6>(num_scale), row_lane<7>(num_scale)};
    const float zk[8] = {row_lane<0>(num_zero), row_lane<1>(num_zero), row_lane<2>(num_zero), row_lane<3>(num_zero),
                         row_lane<4>(num_zero), row_lane<5>(num_zero), row_lane<6>(num_zero), row_lane<7>(num_zero)};
    const float sv[8] = {row_lane<8>(num_scale), row_lane<9>(num_scale), row_lane<10>(num_scale), row_lane<11>(num_scale),
                         row_lane<12>(num_scale), row_lane<13>(num_scale), row_lane<14>(num_scale), row_lane<15>(num_scale)};
    const float zv[8] = {row_lane<8>(num_zero), row_lane<9>(num_zero), row_lane<10>(num_zero), row_lane<11>(num_zero),
                         row_lane<12>(num_zero), row_lane<13>(num_zero), row_lane<14>(num_zero), row_lane<15>(num_zero)};

    f32x4 x[NB][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) x[nb][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KV; ++c) {
        CodeFrag f;
        Tile::key_piece(f, kf.w[b], c);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int p = 0; p < PARTS; ++p) x[nb][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.v, q[nb][p][c].v, x[nb][b], 0, 0, 0);
      }
    }
    CodeFrag hi[NB], lo[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const AttendView view = attend_view(k, span, sink, pos[nb], base + 4 * quad);
      float y[8], p[8], ps[8];
      bool sees[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = fmaf(x[nb][e >> 2][e & 3], sk[e], zk[e] * qsum[nb]);
        sees[e] = !cut || attend_sees(view, 16 * (e >> 2) + (e & 3));
        y[e] = sees[e] ? y[e] : -INFINITY;
      }
      // 2^(x - m) and its product with the scale, which what is hidden has none of, whatever its numbers are
      const auto weigh = [&]() {
        const float ref = m[nb] > -INFINITY ? m[nb] : 0.f;
        float most = 0.f, most_scaled = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = attend_exp2(fmaf(y[e], qunit[nb], -ref));
          ps[e] = sees[e] ? p[e] * sv[e] : 0.f;
          most = fmaxf(most, p[e]);
          most_scaled = fmaxf(most_scaled, fabsf(ps[e]));
        }
        return fmaxf(most_scaled, most * (1.f / kCodeUnit));        // (a scale of 0 counts as the smallest one)
      };
      const float most = weigh();
      if (__any(!(most <= kCodeTop) || m[nb] == -INFINITY)) {
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float scale = fminf(fmaxf(fabsf(sv[e]), 1.f / kCodeUnit), 65504.f);
          top = fmaxf(top, sees[e] ? fmaf(y[e], qunit[nb], attend_log2(scale)) : -INFINITY);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float next = top > m[nb] + 14.f ? top - 7.f : m[nb];
        const float f = m[nb] > -INFINITY ? attend_exp2(m[nb] - next) : 1.f;
        m[nb] = next;
        l[nb] *= f; zsum[nb] *= f;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[nb][db] *= f;
        weigh();
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        l[nb] += p[e];
        zsum[nb] = sees[e] ? fmaf(p[e], zv[e], zsum[nb]) : zsum[nb];
        hi[nb].v[e] = (_Float16)ps[e];
        if (PARTS == 2) lo[nb].v[e] = (_Float16)(ps[e] - (float)hi[nb].v[e]);
      }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      CodeFrag f;
      Tile::val_piece(f, vf, db);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.v, hi[nb].v, o[nb][db], 0, 0, 0);
        if (PARTS == 2) o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.v, lo[nb].v, o[nb][db], 0, 0, 0);
      }
    }
  }

  // the waves' parts
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    l[nb] += __shfl_xor(l[nb], 16);
    l[nb] += __shfl_xor(l[nb], 32);
    zsum[nb] += __shfl_xor(zsum[nb], 16);
    zsum[nb] += __shfl_xor(zsum[nb], 32);
    const int r = 16 * nb + col;
    if (quad == 0) { sm.m[wave][r] = m[nb]; sm.l[wave][r] = l[nb]; }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) sm.o[wave][r][DB * (4 * quad + c) + db] = fmaf(o[nb][db][c], Tile::val_unit(db), zsum[nb]);
  }
  __syncthreads();
  few_join<ET, D, NB, NW>(a, k, s, h, row0, split, sm);
}

// rows: of a workgroup's tile, 16, or 32 (bf16)
template <typename ET, int D, int BITS>
static void few_launch(const AttendCodesArgs& c, const int rows, hipStream_t st) {
  const dim3 grid(c.a.keys[0].blocks), threads(256);
  if constexpr (sizeof(ET) == 2) {
    if (rows == 32) { hipLaunchKernelGGL((k_attend_codes_few<ET, D, BITS, 2, 4>), grid, threads, 0, st, c); return; }
  }
  hipLaunchKernelGGL((k_attend_codes_few<ET, D, BITS, 1, 4>), grid, threads, 0, st, c);
}

obf_status_t launch_attend_codes_few(const AttendCodesArgs& c, int rows, int d, int dtype, int bits, hipStream_t st) {
  ProfScope prof(ST_ATTEND, st);
  if (dtype == OBF_BF16) {
    if (d == 128) { if (bits == 4) few_launch<uint16_t, 128, 4>(c, rows, st); else few_launch<uint16_t, 128, 8>(c, rows, st); }
    else { if (bits == 4) few_launch<uint16_t, 64, 4>(c, rows, st); else few_launch<uint16_t, 64, 8>(c, rows, st); }
  } else {
    if (d == 128) { if (bits == 4) few_launch<float, 128, 4>(c, rows, st); else few_launch<float, 128, 8>(c, rows, st); }
    else { if (bits == 4) few_launch<float, 64, 4>(c, rows, st); else few_launch<float, 64, 8>(c, rows, st); }
  }
  return check_launch("attend codes");
}

}  // namespace obf
