// Attention over a cache held in codes of 4 or 8 bits, few query rows per KV head; and any number of them over short caches, and of fp32 rows.
//
//   x_rj = (s_j q_r . c_j + z_j sum_c q_rc) / sqrt(d),  O_r = sum_j w_rj (s_j c_j + z_j),  w_rj = exp(x_rj - lse_r) over the visible rows j
//
// with c_j the codes of a row, s_j and z_j its scale and zero: the products are of whole numbers, the two numbers of a row come in where there is one value per row and
// query.  One pass over the codes: a wave takes tiles of 32 rows, holds the sum l of its query rows and O' = sum_j 2^(x_rj - m) (s_j c_j + z_j); waves and then
// ranges of a head are joined as in attend_few.hip, with the same lanes: K C^T leaves four rows of one query in a lane, the operand that V's product takes.
//
// bf16: a code n in the low bits of a half-precision number is n 2^-24, exactly, four bits higher 16 n 2^-24, and the matrix instructions take such numbers: a shift and
// a mask make two codes of an operand, whose order is Q's to follow.  But they line their products up by the exponents as written, the smallest normal one for all of
// these, and drop what lies 2^-24 below: of sums of codes below 16 in the lowest bits 2^-20 is lost, in the bits above, or of 8-bit codes, 2^-25 (measured).  K's
// codes therefore stand four bits up, seven instructions for eight codes; V's, behind whose sums the result is rounded to 2^-8, as they come, five for eight.
// fp32: codes less the one in the middle of the range, beside the value of that one in the place of the zero, so that the two sums are small where the values lie
// about 0 (3 x 2 heads, 333 queries: 4e-6 of the result's norm off 64 bits with the codes as they are, 2e-7 so, where the same sums in fp32 are 4e-7 off).
// Q enters as half-precision numbers under a power of two per row, so that its largest lies in [2^14, 2^15): bf16 exactly but for elements 2^-39 of the largest, fp32
// as two parts, rounded, which three numbers in four are exactly and the others within 2^-23.  The weights times s_j enter V's product as half-precision numbers of 11 bits, behind
// which the result is rounded to 8 (fp32: two parts): relative to a reference that follows the largest of 2^x_rj |s_j|, so that the largest product lies in [2^7, 2^15] whatever
// the scales are.  l, sum_j w z_j and O' are single precision.  A part more was measured: bf16 weights of 22 bits take 16 x 8 heads of 16000 rows from 52.7 to 54.3 us, 32 heads'
// 40 queries over 2 x 8 of 4000 from 24.4 to 26.2, and leave the result as far off, 1.6e-3 of its norm; fp32 of 33 bits 324 to 374 (2000 queries of 32 heads over 8 of 4000 rows),
// 104 to 111 (one query, 16 x 8 of 16000, 8 bits), and the result 1.1e-7 off where it is 1.2e-7 (heads of two rows), 2.8e-7 where it is 3.1e-7 (512 rows).
//
// Bound by the codes' bytes where the caches are long: 16 x 8 heads of 8192 to 32768 rows of 128, 4 bits, one query of 4 heads, 69 to 72 us and 5 for the join (5.0 to 5.2 TB/s, the
// vector pipe busy for 0.52 of the time, the matrix pipe for 0.12); 32 x 8 heads of 1000 to 4096, 8 bits, 34 us (5.1 TB/s).  With a window of 1024, 48 x 8 heads, 17 to 18 us: all
// 384 workgroups run at once, one on some compute units and two on the others, whose waves take four or five of a head's 33 or 34 tiles; 8 heads of 100 to 340 rows 7 us, one chain
// of loads; fp32, 3 x 2 heads of 333 to 512, 333 queries of 2 heads, d 64, 8 to 9 us, 8 heads of 4000 rows of 128, 2000 queries of 32 heads, which read the codes for every 16 query
// rows, 385 to 392 (0.25 PFLOP/s).  No gain: loads a tile ahead, two query tiles a workgroup, the queries' loads behind the first tile's.
#include "attend_codes.hpp"
#include "attend_few.hpp"
#include "codes.hpp"

namespace obf {

constexpr float kCodeUnit = 16777216.f;       // 2^24: a code's number is code / kCodeUnit
constexpr float kCodeTop = 32768.f;           // largest weight times scale

template <int LANE> __device__ __forceinline__ float row_lane(const float x) {     // the value of lane LANE of the row of 16
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), 0x150 + LANE, 0xF, 0xF, true));
}
// The largest magnitude of eight, numbers or not (one instruction for two; fmaxf would first make its operands quiet).
__device__ __forceinline__ float most_of(const float (&x)[8]) {
  float m;
  asm("v_max3_f32 %0, |%1|, |%2|, |%3|" : "=v"(m) : "v"(x[0]), "v"(x[1]), "v"(x[2]));
  asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(m) : "v"(m), "v"(x[3]), "v"(x[4]));
  asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(m) : "v"(m), "v"(x[5]), "v"(x[6]));
  asm("v_max_f32 %0, %1, |%2|" : "=v"(m) : "v"(m), "v"(x[7]));
  return m;
}

// Operands of a tile of 32 rows.
template <int D, int BITS, bool MIDDLE> struct CodeTile {
  static constexpr int KV = D / 32;                 // matrix instructions per block of 16 rows
  static constexpr int DB = D / 16;                 // blocks of 16 channels in O
  static constexpr int BYTES = D * BITS / 8;        // of a row
  static constexpr int KW = BYTES / 16;             // words of a K row per lane: a quarter of the row
  static constexpr int VB = BYTES / 16;             // bytes of a V row per lane: a sixteenth
  static constexpr int VW = VB < 4 ? 1 : VB / 4;
  struct Keys { uint32_t w[2][KW]; };
  struct Vals { uint32_t w[8][VW]; };

  // channel (of the lane's quarter row) of element e of piece c; what a code of 1 is in it
  static constexpr int channel(const int c, const int e) {
    return BITS == 4 ? 8 * c + (e >> 1) + 4 * (e & 1) : 8 * c + 4 * (e >> 2) + ((e >> 1) & 1) + 2 * (e & 1);
  }
  static constexpr float KEY_UNIT = MIDDLE ? 1.f : BITS == 4 ? kCodeUnit / 16.f : kCodeUnit;
  // MIDDLE: the two codes of a word as numbers, less the middle one
  static __device__ __forceinline__ void settle(CodeFrag& f, const int i) {
    if constexpr (MIDDLE) {
      const _Float16 less = (_Float16)(-1024.f - code_middle(BITS));
      f.w[i] |= 0x64006400u;
      f.h[i] += f16x2{less, less};
    }
  }

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
      const uint32_t x = w[c];
      if constexpr (MIDDLE) { f.w[0] = x & 0x000f000fu; f.w[1] = (x >> 4) & 0x000f000fu; f.w[2] = (x >> 8) & 0x000f000fu; f.w[3] = (x >> 12) & 0x000f000fu; }
      else { f.w[0] = (x << 4) & 0x00f000f0u; f.w[1] = x & 0x00f000f0u; f.w[2] = (x >> 4) & 0x00f000f0u; f.w[3] = (x >> 8) & 0x00f000f0u; }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) { f.w[2 * i] = w[2 * c + i] & 0x00ff00ffu; f.w[2 * i + 1] = (w[2 * c + i] >> 8) & 0x00ff00ffu; }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) settle(f, i);
  }
  // channel block db of the eight rows, in pairs: rows 2 i and 2 i + 1
  static __device__ __forceinline__ void val_piece(CodeFrag& f, const Vals& v, const int db) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BITS == 4) {
        const uint32_t both = __builtin_amdgcn_perm(v.w[2 * i + 1][0], v.w[2 * i][0], db < 4 ? 0x05040100u : 0x07060302u);
        if (MIDDLE) f.w[i] = (both >> 4 * (db & 3)) & 0x000f000fu;
        else f.w[i] = ((db & 2) ? both >> 8 : both) & ((db & 1) ? 0x00f000f0u : 0x000f000fu);
      } else {
        f.w[i] = __builtin_amdgcn_perm(v.w[2 * i + 1][db >> 2], v.w[2 * i][db >> 2], 0x0c040c00u + (uint32_t)(db & 3) * 0x00010001u);
      }
      settle(f, i);
    }
  }
  static constexpr float val_unit(const int db) { return MIDDLE ? 1.f : BITS == 4 && (db & 1) ? kCodeUnit / 16.f : kCodeUnit; }
};

// Parts of a row of Q in the order of the K operands; the power of two, taken out, and the row's sum under it.
template <typename ET, int D, int BITS, int PARTS>
__device__ __forceinline__ void load_query(CodeFrag (&q)[PARTS][D / 32], float& unit, float& sum, const ET* row, const int quad) {
  typedef CodeTile<D, BITS, PARTS == 2> Tile;
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
  const float up = query_power(top, unit);
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) { x[i] *= up; sum += x[i]; }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float y = x[Tile::channel(c, i)];
#pragma unroll
      for (int p = 0; p < PARTS; ++p) { q[p][c].v[i] = (_Float16)y; y -= (float)q[p][c].v[i]; }
    }
}

template <typename ET, int D, int BITS, int NW, int PER_SIMD>
__global__ __launch_bounds__(NW * 64, PER_SIMD) void k_attend_codes_few(const AttendCodesArgs args) {
  constexpr int PARTS = sizeof(ET) == 4 ? 2 : 1;
  typedef CodeTile<D, BITS, PARTS == 2> Tile;
  constexpr int DB = Tile::DB, KV = Tile::KV, ROWS = kCodesFewRows, BYTES = Tile::BYTES;
  __shared__ __attribute__((aligned(16))) FewShared<D, 1, NW> sm;
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
  const uint16_t *scales = (of_v ? args.v.scale : args.k.scale) + head + num_row, *zeros = (of_v ? args.v.zero : args.k.zero) + head + num_row;
  const float scale_unit = of_v ? 1.f : a.scale2 * Tile::KEY_UNIT, zero_unit = of_v ? 1.f : a.scale2;

  CodeFrag q[PARTS][KV];
  float qunit, qsum;
  const AttendRow w = attend_row(a, k, s, min(row0 + col, set_rows - 1));
  load_query<ET, D, BITS, PARTS>(q, qunit, qsum, (const ET*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt, quad);
  const int pos = n - a.T + w.t;
  f32x4 o[DB];
  float m = -INFINITY, l = 0.f, zsum = 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};

  // What a tile's loads bring.
  struct Loads { typename Tile::Keys k; typename Tile::Vals v; uint16_t scale, zero; };
  // a lane's places in a tile; the others are constants further
  const uint32_t at_k = col * BYTES + quad * (BYTES / 4), at_v = 4 * quad * BYTES + col * (BYTES / 16);
  const auto load = [&](Loads& f, const int i) {
    const int base = 32 * i, start = attend_uniform(attend_key(span, base));
    const int jump = attend_uniform(base < span.split ? span.split - base : 32), last = attend_uniform(span.count - 1 - base);
    // (a tile's address in scalar registers: the compiler would keep a sum of lane and head for every load)
    const uint8_t *kt = (const uint8_t*)attend_uniform((const void*)(kc + (size_t)start * BYTES)), *vt = (const uint8_t*)attend_uniform((const void*)(vc + (size_t)start * BYTES));
    if (jump >= 32 && last >= 31) {
      const uint8_t *kl = kt + at_k, *vl = vt + at_v;
#pragma unroll
      for (int b = 0; b < 2; ++b) Tile::load_key(f.k.w[b], kl + b * 16 * BYTES);
      f.scale = scales[start];
      f.zero = zeros[start];
#pragma unroll
      for (int e = 0; e < 8; ++e) Tile::load_val(f.v.w[e], vl + (16 * (e >> 2) + (e & 3)) * BYTES);
    } else {
      // rows relative to the tile's first entry; entries behind the span's last one repeat it
      const auto row = [&](const int r) { const int x = min(r, last); return (uint32_t)(x + (x >= jump ? span.skip : 0)); };
      int at = lane;
      asm volatile("" : "+v"(at));                     // (nothing of this is kept in registers for the other tiles)
      const int quad = at >> 4, col = at & 15;
#pragma unroll
      for (int b = 0; b < 2; ++b) Tile::load_key(f.k.w[b], kt + (row(16 * b + col) * BYTES + quad * (BYTES / 4)));
      const int number = 16 * ((col >> 2) & 1) + 4 * quad + (col & 3), further = start + (int)row(number) - number;
      f.scale = scales[further];
      f.zero = zeros[further];
#pragma unroll
      for (int e = 0; e < 8; ++e) Tile::load_val(f.v.w[e], vt + (row(16 * (e >> 2) + 4 * quad + (e & 3)) * BYTES + col * (BYTES / 16)));
      asm volatile("");                                // (or the loads of both branches become one, from an address in registers for each)
    }
  };
  for (int i = first + wave; i < behind; i += NW) {
    Loads f;
    load(f, i);
    const int base = 32 * i;
    const bool cut = attend_cut(k, span, sink, pmin, pmax, base, 32);
    const float given = __half2float(__ushort_as_half(f.scale)), base_value = __half2float(__ushort_as_half(f.zero));
    // (an infinite number is none: by itself it would hide a key from the queries whose sums have one sign)
    const float none = 0.f * (given + base_value);
    const float scale = given * scale_unit, zero = fmaf(PARTS == 2 ? fmaf(given, code_middle(BITS), base_value) : base_value, zero_unit, none);
    const bool flat = __any(of_v && scale == 0.f);
    f32x4 x[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      x[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KV; ++c) {
        CodeFrag kf;
        Tile::key_piece(kf, f.k.w[b], c);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) x[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf.v, q[p][c].v, x[b], 0, 0, 0);
      }
    }
    CodeFrag hi, lo;
    const float sk[8] = {row_lane<0>(scale), row_lane<1>(scale), row_lane<2>(scale), row_lane<3>(scale), row_lane<4>(scale), row_lane<5>(scale), row_lane<6>(scale), row_lane<7>(scale)};
    const float zk[8] = {row_lane<0>(zero), row_lane<1>(zero), row_lane<2>(zero), row_lane<3>(zero), row_lane<4>(zero), row_lane<5>(zero), row_lane<6>(zero), row_lane<7>(zero)};
    float y[8], p[8], ps[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fmaf(sk[e], x[e >> 2][e & 3], zk[e] * qsum);
    float sv[8] = {row_lane<8>(scale), row_lane<9>(scale), row_lane<10>(scale), row_lane<11>(scale), row_lane<12>(scale), row_lane<13>(scale), row_lane<14>(scale), row_lane<15>(scale)};
    float zv[8] = {row_lane<8>(zero), row_lane<9>(zero), row_lane<10>(zero), row_lane<11>(zero), row_lane<12>(zero), row_lane<13>(zero), row_lane<14>(zero), row_lane<15>(zero)};
    if (cut) {
      // what is hidden has no weight, no scale and no zero, whatever its numbers are
      const AttendView view = attend_view(k, span, sink, pos, base + 4 * quad);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool sees = attend_sees(view, 16 * (e >> 2) + (e & 3));
        y[e] = sees ? y[e] : -INFINITY; sv[e] = sees ? sv[e] : 0.f; zv[e] = sees ? zv[e] : 0.f;
        asm volatile("" : "+v"(y[e]), "+v"(sv[e]), "+v"(zv[e]));            // (a branch, not selects in every tile: few have masks)
      }
    }
    // 2^(x - m) and its product with the scale
    const auto weigh = [&]() {
      const float ref = m > -INFINITY ? m : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = attend_exp2(fmaf(y[e], qunit, -ref));
        ps[e] = sv[e] * p[e];
      }
    };
    weigh();
    float most = most_of(ps);
    if (flat) most = fmaxf(most, most_of(p) * (1.f / kCodeUnit));        // (a scale of 0 counts as the smallest one)
    if (__any(!(most <= kCodeTop) || m == -INFINITY)) {
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaf(y[e], qunit, attend_log2(fminf(fmaxf(fabsf(sv[e]), 1.f / kCodeUnit), 65504.f))));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = top > m + 14.f ? top - 7.f : m;
      const float down = m > -INFINITY ? attend_exp2(m - next) : 1.f;
      m = next;
      l *= down; zsum *= down;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= down;
      weigh();
    }
    // (a tile's terms first: a lane adds up long ranges)
    float sum = p[0], zero_sum = zv[0] * p[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) { sum += p[e]; zero_sum = fmaf(zv[e], p[e], zero_sum); }
    l += sum;
    zsum += zero_sum;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi.v[e] = (_Float16)ps[e];
      if (PARTS == 2) lo.v[e] = (_Float16)(ps[e] - (float)hi.v[e]);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      CodeFrag vf;
      Tile::val_piece(vf, f.v, db);
      o[db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf.v, hi.v, o[db], 0, 0, 0);
      if (PARTS == 2) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf.v, lo.v, o[db], 0, 0, 0);
    }
  }

  // the waves' parts
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  zsum += __shfl_xor(zsum, 16);
  zsum += __shfl_xor(zsum, 32);
  if (quad == 0) { sm.m[wave][col] = m; sm.l[wave][col] = l; }
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int c = 0; c < 4; ++c) sm.o[wave][col][DB * (4 * quad + c) + db] = fmaf(o[db][c], Tile::val_unit(db), zsum);
  __syncthreads();
  few_join<ET, D, 1, NW>(a, k, s, h, row0, split, sm);
}

// waves: of a workgroup, 4 or 8
template <typename ET, int D, int BITS>
static void few_launch(const AttendCodesArgs& c, const int waves, hipStream_t st) {
  constexpr int PER_SIMD = few_codes_per_cu(D, sizeof(ET) == 4, BITS) == 2 ? 4 : 3;      // waves of a SIMD, by their registers
  const dim3 grid(c.a.keys[0].blocks), threads(64 * waves);
  if (waves == 8) hipLaunchKernelGGL((k_attend_codes_few<ET, D, BITS, 8, PER_SIMD>), grid, threads, 0, st, c);
  else hipLaunchKernelGGL((k_attend_codes_few<ET, D, BITS, 4, PER_SIMD>), grid, threads, 0, st, c);
}

obf_status_t launch_attend_codes_few(const AttendCodesArgs& c, int waves, int d, int dtype, int bits, hipStream_t st) {
  ProfScope prof(ST_ATTEND, st);
  if (dtype == OBF_BF16) {
    if (d == 128) { if (bits == 4) few_launch<uint16_t, 128, 4>(c, waves, st); else few_launch<uint16_t, 128, 8>(c, waves, st); }
    else { if (bits == 4) few_launch<uint16_t, 64, 4>(c, waves, st); else few_launch<uint16_t, 64, 8>(c, waves, st); }
  } else {
    if (d == 128) { if (bits == 4) few_launch<float, 128, 4>(c, waves, st); else few_launch<float, 128, 8>(c, waves, st); }
    else { if (bits == 4) few_launch<float, 64, 4>(c, waves, st); else few_launch<float, 64, 8>(c, waves, st); }
  }
  return check_launch("attend codes");
}

}  // namespace obf
