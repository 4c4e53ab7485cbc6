// Accumulated attention weight: mass_j += sum over the query rows of exp(x_rj - lse_r), from the rows' final normalisers.
//
// A wave holds the operands of 32 keys and goes over the query rows that see any of them, 16 at a time; a lane sums the weights of its four times
// two keys over one row in sixteen, and the sixteen are added at the end.  Every cache row belongs to one wave, so that no sum depends on an order of
// arrival.
#include "attend_few.hpp"
#include "attend_tile.hpp"

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

// The same for many query rows, bf16: a wave holds the operands of 64 keys, a workgroup of 256; the query rows pass through LDS, 64 at a time, their normalisers
// with them.  The rows are cut into ranges where the keys alone do not fill the chip; the ranges' sums are added in their order by k_attend_mass_add.
constexpr int MT_KEYS = 256, MT_ROWS = 64, MT_THREADS = 256;

template <int D>
__global__ __launch_bounds__(MT_THREADS, 2) void k_attend_mass_tile(const AttendArgs a, const AttendMass ms, const float* __restrict__ lse) {
  constexpr int KK = D / 16, PIECES = D / 8, LOADS = MT_ROWS * PIECES / MT_THREADS;
  __shared__ __attribute__((aligned(16))) char sm_q[2][MT_ROWS * 2 * D];
  __shared__ float sm_ref[2][MT_ROWS];
  __shared__ AttendView sm_view[2][MT_ROWS];
  const AttendKeys& k = a.keys[0];
  const int lane = threadIdx.x & 63, wave = attend_uniform(threadIdx.x >> 6), half = lane >> 5;
  const int split = blockIdx.x % ms.nsplit, tile = blockIdx.x / ms.nsplit % ms.tiles, set = blockIdx.x / ms.nsplit / ms.tiles, h = set % a.H, s = set / a.H;
  const int n = attend_uniform(attend_len(k, s, h)), sink = attend_uniform(attend_sink(k, s, h));
  const int base0 = tile * MT_KEYS, base = base0 + wave * 64, p0 = n - a.T;
  if (base0 >= n) return;
  // the queries that see a key of the workgroup
  int t0 = 0, t1 = a.T;
  if (k.causal) {
    t0 = max(0, base0 - p0);
    if (k.window > 0 && base0 >= sink) t1 = max(t0, (int)min((long)a.T, (long)base0 + MT_KEYS - 1 + k.window - p0));
  }
  const int steps = (int)(((long)max(0, t1 - t0) * a.g + MT_ROWS - 1) / MT_ROWS), per = (steps + ms.nsplit - 1) / ms.nsplit;
  const int first = t0 * a.g + split * per * MT_ROWS, behind = (int)min((long)t1 * a.g, (long)first + (long)per * MT_ROWS);
  const size_t row_base = (size_t)s * k.sample_rows + (size_t)h * k.stride;
  const AttendSpan all = {n, 0, 0};
  TileFrag kf[2][KK];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      kf[b][kk].u = *(const TilePiece*)((const uint16_t*)k.K + (row_base + min(base + 32 * b + (lane & 31), n - 1)) * D + 16 * kk + 8 * half);
  float sum[2][16];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[b][e] = 0.f;

  // 64 rows from r0 on, to registers and from there to LDS; a thread fetches LOADS pieces, and the first 64 threads a row's normaliser and view
  TilePiece next[LOADS];
  float next_ref = 0.f;
  AttendView next_view = {-1, -1, 0};
  const uint16_t* Q = (const uint16_t*)a.Q + (size_t)s * a.qs + (size_t)h * a.g * a.qh + 8 * (threadIdx.x % PIECES);
  const auto fetch = [&](const int r0) {
    const AttendStep at = attend_step(a, r0);
    const int most = behind - 1 - r0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const AttendRow w = attend_row(a, at, s, min((int)(i * (MT_THREADS / PIECES) + threadIdx.x / PIECES), most));
      next[i] = *(const TilePiece*)(Q + (size_t)w.gi * a.qh + (size_t)w.t * a.qt);
    }
    const int i = (int)(threadIdx.x % MT_ROWS);
    const AttendRow w = attend_row(a, at, s, min(i, most));
    const float v = lse[attend_row_number(a, h, w)];
    next_view = attend_view(k, all, sink, p0 + w.t);
    // (a row that sees nothing has weights of 0, and so has one behind the range)
    const bool counts = i <= most && !(v == -INFINITY);
    next_ref = counts ? v * 1.44269504088896341f : INFINITY;
    if (!counts) next_view.hi = -1;
  };
  const auto put = [&](const int buf) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      *(TilePiece*)(sm_q[buf] + place_k<D>(i * (MT_THREADS / PIECES) + threadIdx.x / PIECES, threadIdx.x % PIECES)) = next[i];
    if (threadIdx.x < MT_ROWS) { sm_ref[buf][threadIdx.x] = next_ref; sm_view[buf][threadIdx.x] = next_view; }
  };
  if (first < behind) { fetch(first); put(0); }
  __syncthreads();
  int buf = 0;
  for (int r0 = first; r0 < behind; r0 += MT_ROWS, buf ^= 1) {
    const bool more = r0 + MT_ROWS < behind;
    if (more) fetch(r0 + MT_ROWS);
    // some row of the step does not see some key of the wave; none sees any
    const int wmin = p0 + r0 / a.g, wmax = p0 + (min(r0 + MT_ROWS, behind) - 1) / a.g;
    const bool cut = r0 + MT_ROWS > behind || attend_cut(k, all, sink, wmin, wmax, base, 64);
    const bool none = base >= n || (k.causal && (base > wmax || (k.window > 0 && base + 63 <= wmin - k.window && base >= sink)));
    if (!none) {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) {
        const int row = 32 * qb + (lane & 31);
        TileFrag q[KK];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) q[kk].u = *(const TilePiece*)(sm_q[buf] + place_k<D>(row, 2 * kk + half));
        const float ref = sm_ref[buf][row];
        const AttendView view = attend_from(sm_view[buf][row], base + 4 * half);
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
              sum[b][e] += attend_sees(view, 32 * b + 8 * (e >> 2) + (e & 3)) ? v : 0.f;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[b][e] += attend_exp2(fmaf(x[e], a.scale2, -ref));
          }
        }
      }
    }
    if (more) put(buf ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = sum[b][e];
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) v += __shfl_xor(v, off);
      const int j = base + 32 * b + 8 * (e >> 2) + 4 * half + (e & 3);
      if ((lane & 31) == 0 && j < n) {
        if (ms.nsplit > 1) ms.part[((size_t)split * a.S * a.H + set) * k.stride + j] = v;
        else ms.mass[row_base + j] += v;
      }
    }
}

__global__ __launch_bounds__(256) void k_attend_mass_add(const AttendArgs a, const AttendMass ms) {
  const AttendKeys& k = a.keys[0];
  const int set = blockIdx.y, h = set % a.H, s = set / a.H, j = blockIdx.x * 256 + threadIdx.x;
  if (j >= attend_len(k, s, h)) return;
  float v = 0.f;
  for (int i = 0; i < ms.nsplit; ++i) v += ms.part[((size_t)i * a.S * a.H + set) * k.stride + j];
  ms.mass[(size_t)s * k.sample_rows + (size_t)h * k.stride + j] += v;
}

// Ranges of query rows of the kernel of many rows: four workgroups per compute unit and more, not less than 256 rows each.
int attend_mass_ranges(const AttendArgs& a, int dtype) {
  const AttendKeys& k = a.keys[a.n_keys - 1];
  const long rows = (long)a.T * a.g, blocks = (long)((k.stride + MT_KEYS - 1) / MT_KEYS) * a.S * a.H;
  if (dtype != OBF_BF16 || rows <= kAttendFewRows) return 1;
  const long want = (4 * kNumCU + blocks - 1) / blocks, most = (rows + 255) / 256;
  return (int)(want < most ? want : most);
}

obf_status_t launch_attend_mass(const AttendArgs& args, int d, int dtype, const float* lse, const AttendMass& mass, hipStream_t st) {
  ProfScope prof(ST_ATTEND_MASS, st);
  AttendArgs a = args;
  AttendKeys& k = a.keys[0];
  AttendMass ms = mass;
  if (dtype == OBF_BF16 && (long)a.T * a.g > kAttendFewRows) {
    ms.tiles = (k.stride + MT_KEYS - 1) / MT_KEYS;
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
