// Accumulated attention weight: mass_j += sum over the query rows of exp(x_rj - lse_r), from the rows' final normalisers.
//
// A wave holds the operands of 32 keys and goes over the query rows that see any of them, 16 at a time; a lane sums the weights of its four times
// two keys over one row in sixteen, and the sixteen are added at the end.  Every cache row belongs to one wave, so that no sum depends on an order of
// arrival.
#include "attend_few.hpp"

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
  Tile::load_keys(kf, (const ET*)k.K + first_row * D, base, n - 1, lane);
  float sum[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  const int behind = t1 * a.g;
  for (int r0 = t0 * a.g; r0 < behind; r0 += 16) {
    const int r = r0 + (lane & 15);
    const AttendRow w = attend_row(a, k, s, min(r, behind - 1));
    typename Tile::Query q;
    Tile::load_query(q, (const ET*)a.Q + (size_t)w.s * a.qs + (size_t)(h * a.g + w.gi) * a.qh + (size_t)w.t * a.qt, lane);
    const float row_lse = lse[attend_row_number(a, h, w)];
    const float ref = row_lse > -INFINITY ? row_lse * 1.44269504088896341f : row_lse;
    const bool counts = r < behind && !(row_lse == -INFINITY);       // (a row that sees nothing has weights of 0)
    f32x4 x[2];
    Tile::scores(x, kf, q);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = base + 16 * b + 4 * quad + c;
        const bool sees = counts && attend_sees(k.causal, k.window, sink, p0 + w.t, j);
        sum[b][c] += sees ? attend_exp2(fmaf(x[b][c], a.scale2, -ref)) : 0.f;
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

obf_status_t launch_attend_mass(const AttendArgs& args, int d, int dtype, const float* lse, float* mass, hipStream_t st) {
  ProfScope prof(ST_ATTEND_MASS, st);
  AttendArgs a = args;
  AttendKeys& k = a.keys[0];
  k.row_tiles = (k.stride + AM_WAVES * 32 - 1) / (AM_WAVES * 32);
  const dim3 grid((unsigned)((long)k.row_tiles * a.S * a.H));
  if (dtype == OBF_BF16) {
    if (d == 128) hipLaunchKernelGGL((k_attend_mass<uint16_t, 128>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, mass);
    else hipLaunchKernelGGL((k_attend_mass<uint16_t, 64>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, mass);
  } else {
    if (d == 128) hipLaunchKernelGGL((k_attend_mass<float, 128>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, mass);
    else hipLaunchKernelGGL((k_attend_mass<float, 64>), grid, dim3(AM_WAVES * 64), 0, st, a, lse, mass);
  }
  return check_launch("attend mass");
}

}  // namespace obf
