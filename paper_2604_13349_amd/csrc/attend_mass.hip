// Accumulated attention weight: mass_j += sum over the query rows of exp(x_rj - lse_r), from the rows' final normalisers.
//
// A wave holds the operands of 32 keys and goes over the query rows that see any of them, 16 at a time; a lane sums the weights of its four times
// two keys over one row in sixteen, and the sixteen are added at the end.  Every cache row belongs to one wave, so that no sum depends on an order of
// arrival.
#include "attend_few.hpp"
#include "attend_tile.hpp"
#include "lds_load.hpp"

namespace obf {

constexpr int AM_WAVES = 4;

template <typename ET, int D>
__global__ __launch_bounds__(AM_WAVES * 64) void k_attend_mass(const AttendArgs a, const float* __restrict__ lse, float* __restrict__ mass) {
  typedef FewTile<ET, D> Tile;
  const AttendKeys& k = a.keys[0];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quad = lane >> 4;
  const int set = blockIdx.x / k.row_tiles, h = set % a.H, s = set / a.H;
  const int base = ((int)(blockIdx.x % k.row_tiles) * AM_WAVES + wave) * 32;
  const int n = attend_len(k, s, h), sink = attend_sink(k, s, h);
  if (base >= n) return;                                             // (no barrier follows)
  // the queries that see a key of the tile
  const int p0 = n - a.T;
  int t0 = 0, t1 = a.T;
  if (k.causal) {
    t0 = max(0, base - p0);
    if (k.window > 0 && base >= sink) t1 = (int)min((long)a.T, (long)base + 31 + k.window - p0);
  }
  if (t0 >= t1) return;
  const size_t first_row = (size_t)s * k.sample_rows + (size_t)h * k.stride;
  typename Tile::Keys kf;
  const AttendSpan all = {n, 0, 0};
  Tile::load_keys(kf, (const ET*)k.K + first_row * D, all, base, lane);
  float sum[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  const int behind = t1 * a.g;
  for (int r0 = t0 * a.g; r0 < behind; r0 += 16) {
    const int r = r0 + (lane & 15);
    const AttendRow w = attend_row(a, attend_step(a, r0), s, min(lane & 15, behind - 1 - r0));
    typename Tile::Query q;
    Tile::load_query(q, (const ET*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt, lane);
    const float row_lse = lse[attend_row_number(a, h, w)];
    const float ref = row_lse > -INFINITY ? row_lse * 1.44269504088896341f : row_lse;
    const bool counts = r < behind && !(row_lse == -INFINITY);       // (a row that sees nothing has weights of 0)
    f32x4 x[2];
    Tile::scores(x, kf, q);
    AttendView view = attend_view(k, all, sink, p0 + w.t, base + 4 * quad);
    if (!counts) view.hi = -1;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float v = attend_exp2(fmaf(x[b][c], a.scale2, -ref));
        sum[b][c] += attend_sees(view, 16 * b + c) ? v : 0.f;
      }
  }
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float v = sum[b][c];
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) v += __shfl_xor(v, off);
      const int j = base + 16 * b + 4 * quad + c;
      if ((lane & 15) == 0 && j < n) mass[first_row + j] += v;
    }
}

// The same for many query rows, bf16: a wave holds the operands of 64 keys (two of 32), a workgroup of 256; the query rows that see any of them pass through LDS,
// 64 at a time, loaded straight to it while the present ones' weights are taken (operands read from memory row by row cost a cache line per lane and load).
// The rows are cut into ranges of ms.per steps, so that a head's early keys, which many queries see, take no longer than its late ones; the ranges' sums are
// added in their order by k_attend_mass_add.
// Two samples of 40 heads and 2048 queries: 100 us; vector work takes 0.38 of the cycles, the products 0.19, a quarter of that beside it.  Of 6.4 vector
// instructions per exponential three are the weights' (a multiply-add, the exponential, an addition): the rows' addresses take some 80 a step of about 300, the
// fixed part of a range some 500, and the masked blocks bring scalars back that have no register.  Loads three steps ahead, both keys' products before their
// weights: no faster.
constexpr int MT_WAVES = 4, MT_THREADS = MT_WAVES * 64, MT_KEYS = MT_WAVES * 64, MT_ROWS = 64;

// query rows r0 .. r1 - 1 that see a key of the 256 from base on
struct MassRows { int r0, r1; };
__device__ __forceinline__ MassRows mass_rows(const AttendArgs& a, const AttendKeys& k, const int n, const int sink, const int base) {
  int t0 = 0, t1 = a.T;
  if (k.causal) {
    t0 = max(0, base - (n - a.T));
    if (k.window > 0 && base >= sink) t1 = (int)min((long)a.T, (long)base + MT_KEYS - 1 + k.window - (n - a.T));
  }
  return {t0 * a.g, max(t0, t1) * a.g};
}

template <int D>
__global__ __launch_bounds__(MT_THREADS, 2) void k_attend_mass_tile(const AttendArgs a, const AttendMass ms, const float* __restrict__ lse) {
  constexpr int KK = D / 16, PIECES = D / 8, LOADS = MT_ROWS * PIECES / MT_THREADS, BYTES = MT_ROWS * D * 2;
  __shared__ __attribute__((aligned(1024))) char sm[2 * BYTES];
  const AttendKeys& k = a.keys[0];
  const int lane = threadIdx.x & 63, wave = attend_uniform(threadIdx.x >> 6), half = lane >> 5;
  // the sets go round the dies; where they do not fill the round the ranges, of which a late tile has fewer, are shifted from tile to tile
  int within;
  const int set = attend_set(blockIdx.x, a.S * a.H, ms.tiles * ms.nsplit, within);
  const int tile = within / ms.nsplit, split = (within + tile) % ms.nsplit, h = set % a.H, s = set / a.H;
  const int n = attend_uniform(attend_len(k, s, h)), sink = attend_uniform(attend_sink(k, s, h));
  const int base0 = tile * MT_KEYS, base = base0 + wave * 64, p0 = n - a.T;
  if (base0 >= n) return;
  const MassRows rows = mass_rows(a, k, n, sink, base0);
  const int first = rows.r0 + split * ms.per * MT_ROWS, behind = (int)min((long)rows.r1, (long)first + (long)ms.per * MT_ROWS);
  if (first >= behind) return;
  const size_t row_base = (size_t)s * k.sample_rows + (size_t)h * k.stride;
  const AttendSpan all = {n, 0, 0};
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)sm;
  const uint16_t* Q = (const uint16_t*)a.Q + (size_t)s * a.qs + (size_t)h * a.g * a.qh;
  const float* head_lse = lse + ((size_t)s * a.H + h) * a.g * a.T;
  // A thread's rows of a step: LOADS whose pieces it loads, and two whose normaliser and query its lane needs.  From step to step they move by 64 rows, that is
  // by `dt` queries and `dg` query heads, with a carry: additions, where the row's number would have to be divided and multiplied anew.
  const int dt = MT_ROWS / a.g, dg = MT_ROWS % a.g;
  const long move = dt * a.qt + dg * a.qh, carry = a.qt - a.g * a.qh;
  const int move_lse = dt + dg * a.T, carry_lse = 1 - a.g * a.T;
  const AttendStep start = attend_step(a, first);
  const uint16_t* piece[LOADS];
  int piece_gi[LOADS], row_gi[2], row_t[2], row_lse[2];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = i * (MT_THREADS / PIECES) + (int)threadIdx.x / PIECES, place = threadIdx.x % PIECES;
    const AttendRow w = attend_row(a, start, s, row);
    piece_gi[i] = w.gi;
    piece[i] = Q + (long)w.gi * a.qh + (long)w.t * a.qt + 8 * (place ^ (D == 128 ? row & 15 : (row >> 1) & 7));
  }
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) {
    const AttendRow w = attend_row(a, start, s, 32 * qb + (lane & 31));
    row_gi[qb] = w.gi; row_t[qb] = w.t; row_lse[qb] = w.gi * a.T + w.t;
  }
  const uint16_t* const any = Q + (long)start.gi * a.qh + (long)start.t * a.qt;          // a row of the range, in the place of those behind it
  // The step's rows from r0 on to LDS, and of the lane's two the normaliser and the query; then on to the next step's.
  struct Rows { float lse[2]; int t[2]; };
  const auto fill = [&](Rows& x, const int buf, const int r0) {
    const void* from[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = i * (MT_THREADS / PIECES) + (int)threadIdx.x / PIECES;
      from[i] = r0 + row < behind ? piece[i] : any;
      piece_gi[i] += dg;
      piece[i] += move;
      if (piece_gi[i] >= a.g) { piece_gi[i] -= a.g; piece[i] += carry; }
    }
    load_to_lds(lds + buf * BYTES + wave * 1024, from);
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      const bool there = r0 + 32 * qb + (lane & 31) < behind;
      x.lse[qb] = head_lse[there ? row_lse[qb] : 0];
      x.t[qb] = row_t[qb];
      row_gi[qb] += dg; row_t[qb] += dt; row_lse[qb] += move_lse;
      if (row_gi[qb] >= a.g) { row_gi[qb] -= a.g; row_t[qb] += 1; row_lse[qb] += carry_lse; }
    }
  };
  Rows now, next = {};
  fill(next, 0, first);
  // queries of the step's first and last row
  int q0 = start.t, g0 = start.gi;
  const int q_last = (behind - 1) / a.g;
  TileFrag kf[2][KK];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      kf[b][kk].u = *(const TilePiece*)((const uint16_t*)k.K + (row_base + min(base + 32 * b + (lane & 31), n - 1)) * D + 16 * kk + 8 * half);
  float sum[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) sum[e] = 0.f;

  for (int r0 = first, buf = 0; r0 < behind; r0 += MT_ROWS, buf ^= 1) {
    now = next;
    wait_loads<0>();
    __syncthreads();                                   // the rows are there, and nobody reads the other ones any more
    if (r0 + MT_ROWS < behind) fill(next, buf ^ 1, r0 + MT_ROWS);
    const int qmin = p0 + q0, qmax = p0 + min(q_last, q0 + (int)(((uint32_t)(g0 + MT_ROWS - 1) * a.g_inv) >> 23));
    g0 += dg; q0 += dt;
    if (g0 >= a.g) { g0 -= a.g; q0 += 1; }
    // none of the rows sees a key of the wave
    if (base >= n || (k.causal && (base > qmax || (k.window > 0 && base + 63 <= qmin - k.window && base >= sink)))) continue;
    // (a row whose lse says that it does not count is masked too: its query may hold anything)
    const bool cut = r0 + MT_ROWS > behind || attend_cut(k, all, sink, qmin, qmax, base, 64) || __any(fminf(now.lse[0], now.lse[1]) == -INFINITY);
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      TileFrag q[KK];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) q[kk].u = *(const TilePiece*)(sm + buf * BYTES + place_k<D>(32 * qb + (lane & 31), 2 * kk + half));
      // (a row that sees nothing has weights of 0, and so has one behind the range)
      const bool counts = r0 + 32 * qb + (lane & 31) < behind && !(now.lse[qb] == -INFINITY);
      const float ref = counts ? now.lse[qb] * 1.44269504088896341f : INFINITY;
      AttendView view = attend_view(k, all, sink, p0 + now.t[qb], base + 4 * half);
      if (!counts) view.hi = -1;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        f32x16 x;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[b][kk].v, q[kk].v, x, 0, 0, 0);
        if (cut) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float v = attend_exp2(fmaf(x[e], a.scale2, -ref));
            sum[16 * b + e] += attend_sees(view, 32 * b + 8 * (e >> 2) + (e & 3)) ? v : 0.f;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) sum[16 * b + e] += attend_exp2(fmaf(x[e], a.scale2, -ref));
        }
      }
    }
  }
  // Sums over the 32 lanes of a half, half of the values passed on at each step: lane i ends with value i.
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const bool upper = lane & off;
#pragma unroll
    for (int e = 0; e < off; ++e) {
      const float mine = upper ? sum[e + off] : sum[e], other = upper ? sum[e] : sum[e + off];
      sum[e] = mine + __shfl_xor(other, off);
    }
  }
  const int e = lane & 31, j = base + 32 * (e >> 4) + 8 * ((e & 15) >> 2) + 4 * half + (e & 3);
  if (j < n) {
    if (ms.nsplit > 1) ms.part[((size_t)split * a.S * a.H + set) * k.stride + j] = sum[0];
    else ms.mass[row_base + j] += sum[0];
  }
}

__global__ __launch_bounds__(256) void k_attend_mass_add(const AttendArgs a, const AttendMass ms) {
  const AttendKeys& k = a.keys[0];
  const int set = blockIdx.y, h = set % a.H, s = set / a.H, j = blockIdx.x * 256 + threadIdx.x, n = attend_len(k, s, h);
  if (j >= n) return;
  const MassRows rows = mass_rows(a, k, n, attend_sink(k, s, h), j & -MT_KEYS);
  const int ranges = ((rows.r1 - rows.r0 + MT_ROWS - 1) / MT_ROWS + ms.per - 1) / ms.per;      // (the others have not written)
  float v = 0.f;
#pragma unroll 4
  for (int i = 0; i < ranges; ++i) v += ms.part[((size_t)i * a.S * a.H + set) * k.stride + j];
  if (ranges > 0) ms.mass[(size_t)s * k.sample_rows + (size_t)h * k.stride + j] += v;
}

// Steps of a range: three rounds of workgroups, two per compute unit, where half of a causal call's steps are not taken; not less than 8, beside whose 2400
// vector instructions a wave's fixed 500 (operands of the keys, addresses, the sums over lanes at the end) still count.  (2 x 8 heads, 2048 queries of 5 heads, us of the
// whole call: one round 263, two 245, three 240, four with 4 steps at least 243.)
AttendMass plan_attend_mass(const AttendArgs& a, int dtype) {
  const AttendKeys& k = a.keys[a.n_keys - 1];
  AttendMass ms = {nullptr, nullptr, 1, 0, 0};
  const long rows = (long)a.T * a.g;
  if (dtype != OBF_BF16 || rows <= kAttendFewRows) return ms;
  ms.tiles = (k.stride + MT_KEYS - 1) / MT_KEYS;
  const long steps = (rows + MT_ROWS - 1) / MT_ROWS, groups = (long)ms.tiles * a.S * a.H;
  long per = groups * steps / (k.causal ? 2 : 1) / (3 * 2 * kNumCU);
  per = per < 8 ? 8 : per;
  per = per > steps ? steps : per;
  ms.per = (int)per;
  ms.nsplit = (int)((steps + per - 1) / per);
  return ms;
}

obf_status_t launch_attend_mass(const AttendArgs& args, int d, int dtype, const float* lse, const AttendMass& ms, hipStream_t st) {
  ProfScope prof(ST_ATTEND_MASS, st);
  AttendArgs a = args;
  AttendKeys& k = a.keys[0];
  if (ms.tiles > 0) {
    const dim3 grid((unsigned)((long)ms.tiles * a.S * a.H * ms.nsplit));
    if (d == 128) hipLaunchKernelGGL(k_attend_mass_tile<128>, grid, dim3(MT_THREADS), 0, st, a, ms, lse);
    else hipLaunchKernelGGL(k_attend_mass_tile<64>, grid, dim3(MT_THREADS), 0, st, a, ms, lse);
    if (ms.nsplit > 1) hipLaunchKernelGGL(k_attend_mass_add, dim3((k.stride + 255) / 256, a.S * a.H), dim3(256), 0, st, a, ms);
    return check_launch("attend mass");
  }
  k.row_tiles = (k.stride + AM_WAVES * 32 - 1) / (AM_WAVES * 32);
  const dim3 grid((unsigned)((long)k.row_tiles * a.S * a.H));
  if (dtype == OBF_BF16) {
    if (d == 128) hipLaunchKernelGGL((k_attend_mass<uint16_t, 128>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, ms.mass);
    else hipLaunchKernelGGL((k_attend_mass<uint16_t, 64>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, ms.mass);
  } else {
    if (d == 128) hipLaunchKernelGGL((k_attend_mass<float, 128>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, ms.mass);
    else hipLaunchKernelGGL((k_attend_mass<float, 64>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, ms.mass);
  }
  return check_launch("attend mass");
}

}  // namespace obf
