// Attention of few query rows per KV head (generation: the group's query heads, a handful of queries), and of any number for fp32 caches.
//
//   O_r = sum_j exp(x_rj - lse_r) V_j,  x_rj = q_r . k_j / sqrt(d) over the visible keys j,  lse_r = log sum_j exp(x_rj)
//
// One pass over K and V: every wave takes tiles of 32 keys, holds the running maximum m and sum l of its query rows and
// O' = sum_j 2^(x_rj - m) V_j; the waves of a workgroup, and then the ranges of keys of a head, are joined by their maxima.
// A tile's products are K Q^T (keys by rows, so that a lane holds four keys of one query row) and V^T P^T: the first one's result has the
// lane layout of the second one's operand, and V, read row by row in full lines, becomes the other operand by byte permutes inside the lane.
// Nothing passes through LDS before the end.  m follows the maximum only where that outgrows it by 2^8 (the sums have room for that), so that
// most tiles need no exchange between lanes.
// bf16: P is split into two bf16 parts, each with its own product, so that it keeps 16 bits; the matrix pipe has the room where the caches' bytes bound
// the kernel.  fp32: all products by v_mfma_f32_16x16x4_f32.
#include "attend_few.hpp"

namespace obf {

template <typename ET, int D, int NB, int NW>
__global__ __launch_bounds__(NW * 64, 2) void k_attend_few(const AttendArgs a) {
  typedef FewTile<ET, D> Tile;
  constexpr int DB = Tile::DB, ROWS = 16 * NB;
  __shared__ __attribute__((aligned(16))) float sm_o[NW][ROWS][D];
  __shared__ float sm_m[NW][ROWS], sm_l[NW][ROWS];
  // which set of keys, tile of rows and range of keys
  int block = blockIdx.x;
  const bool second = block >= a.keys[0].blocks;
  AttendKeys k = a.keys[0];
  if (second) { k = a.keys[1]; block -= a.keys[0].blocks; }
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
  float* logits = a.logits && !second ? a.logits + ((size_t)set * a.logit_tiles * set_rows + (lane & 15)) * 32 + 4 * quad : nullptr;
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
    if (quad == 0) { sm_m[wave][r] = m[nb]; sm_l[wave][r] = l[nb]; }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) sm_o[wave][r][Tile::channel(quad, db, c)] = o[nb][db][c];
  }
  __syncthreads();
  constexpr int PIECES = D / 4;
  for (int e = threadIdx.x; e < ROWS * PIECES; e += NW * 64) {
    const int r = e / PIECES, c = (e % PIECES) * 4;
    if (row0 + r >= set_rows) break;
    float top = sm_m[0][r];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, sm_m[w][r]);
    const float ref = top > -INFINITY ? top : 0.f;
    float sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = attend_exp2(sm_m[w][r] - ref);
      sum = fmaf(f, sm_l[w][r], sum);
      const float4 x = *(const float4*)&sm_o[w][r][c];
      v[0] = fmaf(f, x.x, v[0]); v[1] = fmaf(f, x.y, v[1]); v[2] = fmaf(f, x.z, v[2]); v[3] = fmaf(f, x.w, v[3]);
    }
    const float inv = top > -INFINITY ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = top > -INFINITY ? v[i] * inv : 0.f;
    const float lse2 = top > -INFINITY ? top + attend_log2(sum) : -INFINITY;
    const AttendRow w = attend_row(a, k, ks, row0 + r);
    const size_t number = attend_row_number(a, h, w);
    if (joined) {
      const size_t at = (size_t)(k.split0 + split) * a.rows + number;
      if (c == 0) a.part_lse[at] = lse2;
      if (top > -INFINITY) *(float4*)(a.part_O + at * D + c) = make_float4(v[0], v[1], v[2], v[3]);   // (nobody reads the others)
    } else {
      if (c == 0 && a.lse) a.lse[number] = lse2 * 0.69314718055994531f;
      store4((ET*)a.O + (size_t)w.s * a.os + (size_t)(h * a.g + w.gi) * a.oh + (size_t)w.t * a.ot + c, v);
    }
  }
}

// Joins the ranges of a query row, O = sum_i 2^(lse_i - lse) O_i, and turns the logits of the own keys into weights, mass_j += sum_r 2^(x_rj - lse_r).
// GROUPS lanes share a row's ranges and a lane has four channels, so that the loads of many ranges are in flight; bound by the partial results' bytes, or
// by its launch.  Workgroups behind those of the rows take 32 tiles of keys of a set each, for which they join the normalisers of its few rows themselves.
constexpr int JN_THREADS = 256, JN_TILES = 32;

template <typename ET, int D, int GROUPS>
__global__ __launch_bounds__(JN_THREADS) void k_attend_join(const AttendArgs a, const int row_blocks) {
  constexpr int PIECES = D / 4, PER_ROW = PIECES * GROUPS, PER_BLOCK = JN_THREADS / PER_ROW;
  __shared__ float sm_sum[PER_BLOCK][GROUPS][PIECES];
  __shared__ __attribute__((aligned(16))) float sm_o[PER_BLOCK][GROUPS][D];
  __shared__ float sm_ref[32];
  if ((int)blockIdx.x >= row_blocks) {
    const AttendKeys& k = a.keys[0];
    constexpr int OWN = 32 * JN_TILES / JN_THREADS, RUN = 8;       // keys of a thread, rows whose logits it has in flight
    const int chunks = (a.logit_tiles + JN_TILES - 1) / JN_TILES, block = blockIdx.x - row_blocks, set = block / chunks, h = set % a.H, s = set / a.H;
    const int n = attend_len(k, s, h), first = block % chunks * JN_TILES, set_rows = a.T * a.g;
    const AttendSpan span = attend_span(k, n, attend_sink(k, s, h), n - a.T, n - 1);
    if (32 * first >= span.count) return;
    const float* logits[OWN];
    float* mass[OWN];
    bool valid[OWN];
    float x[OWN][RUN], sum[OWN];
#pragma unroll
    for (int e = 0; e < OWN; ++e) {
      const int i = first + (int)threadIdx.x / 32 + e * (JN_THREADS / 32);
      const int v = 32 * i + (int)threadIdx.x % 32, j = attend_key(span, v);
      valid[e] = v < span.count;
      logits[e] = a.logits + ((size_t)set * a.logit_tiles + i) * set_rows * 32 + threadIdx.x % 32;
      mass[e] = a.mass + (size_t)s * k.sample_rows + (size_t)h * k.stride + j;
      sum[e] = valid[e] ? *mass[e] : 0.f;
#pragma unroll
      for (int r = 0; r < RUN; ++r) x[e][r] = valid[e] && r < set_rows ? logits[e][32 * r] : -INFINITY;
    }
    if ((int)threadIdx.x < set_rows) {
      const size_t row = attend_row_number(a, h, attend_row(a, k, s, threadIdx.x));
      float ref;
      if (a.ranges > 1) {
        float top = -INFINITY, sum = 0.f;
        for (int i = 0; i < a.ranges; ++i) top = fmaxf(top, a.part_lse[(size_t)i * a.rows + row]);
        for (int i = 0; i < a.ranges; ++i) { const float x = a.part_lse[(size_t)i * a.rows + row]; if (x > -INFINITY) sum += attend_exp2(x - top); }
        ref = top > -INFINITY ? top + attend_log2(sum) : -INFINITY;
      } else {
        ref = a.lse[row] * 1.44269504088896341f;
      }
      sm_ref[threadIdx.x] = ref;
    }
    __syncthreads();
    for (int r0 = 0;; r0 += RUN) {
      float w[OWN] = {};
#pragma unroll
      for (int r = 0; r < RUN; ++r) {
        const float ref = sm_ref[min(r0 + r, 31)];
#pragma unroll
        for (int e = 0; e < OWN; ++e) w[e] += x[e][r] == -INFINITY ? 0.f : attend_exp2(x[e][r] - ref);
      }
#pragma unroll
      for (int e = 0; e < OWN; ++e) sum[e] += w[e];
      if (r0 + RUN >= set_rows) break;
#pragma unroll
      for (int e = 0; e < OWN; ++e)
#pragma unroll
        for (int r = 0; r < RUN; ++r) x[e][r] = valid[e] && r0 + RUN + r < set_rows ? logits[e][32 * (r0 + RUN + r)] : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < OWN; ++e) if (valid[e]) *mass[e] = sum[e];
    return;
  }
  const int in_block = threadIdx.x / PER_ROW, group = threadIdx.x / PIECES % GROUPS, piece = threadIdx.x % PIECES, c = piece * 4;
  const size_t row = (size_t)blockIdx.x * PER_BLOCK + in_block;
  const bool valid = row < (size_t)a.rows;
  float top = -INFINITY, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (valid) {
    const float* lse = a.part_lse + row;
#pragma unroll 8
    for (int i = 0; i < a.ranges; ++i) top = fmaxf(top, lse[(size_t)i * a.rows]);
    const float ref = top > -INFINITY ? top : 0.f;
#pragma unroll 4
    for (int i = group; i < a.ranges; i += GROUPS) {
      const float part = lse[(size_t)i * a.rows];
      // (a range without visible keys has no O)
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (part != -INFINITY) x = *(const float4*)(a.part_O + ((size_t)i * a.rows + row) * D + c);
      const float f = attend_exp2(part - ref);
      sum += f;
      v[0] = fmaf(f, x.x, v[0]); v[1] = fmaf(f, x.y, v[1]); v[2] = fmaf(f, x.z, v[2]); v[3] = fmaf(f, x.w, v[3]);
    }
  }
  if (GROUPS > 1) {
    sm_sum[in_block][group][piece] = sum;
    *(float4*)&sm_o[in_block][group][c] = make_float4(v[0], v[1], v[2], v[3]);
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) {
      const float4 x = *(const float4*)&sm_o[in_block][i][c];
      sum += sm_sum[in_block][i][piece];
      v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    }
  }
  if (!valid) return;
  const bool any = top != -INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = any ? v[i] / sum : 0.f;
  const int t = (int)(row % a.T), hq = (int)(row / a.T % ((size_t)a.H * a.g)), s = (int)(row / a.T / ((size_t)a.H * a.g));
  if (c == 0 && a.lse) a.lse[row] = any ? (top + attend_log2(sum)) * 0.69314718055994531f : -INFINITY;
  store4((ET*)a.O + (size_t)s * a.os + (size_t)hq * a.oh + (size_t)t * a.ot + c, v);
}

#ifndef FEW_NW
#define FEW_NW 4
#endif
template <typename ET, int D>
static void few_launch(const AttendArgs& a, int rows, hipStream_t st) {
  const int blocks = a.keys[0].blocks + (a.n_keys > 1 ? a.keys[1].blocks : 0);
  if (rows == 16) hipLaunchKernelGGL((k_attend_few<ET, D, 1, FEW_NW>), dim3(blocks), dim3(FEW_NW * 64), 0, st, a);
  else hipLaunchKernelGGL((k_attend_few<ET, D, 2, 2>), dim3(blocks), dim3(128), 0, st, a);
}

// rows: of a workgroup's tile, 16 or 32
obf_status_t launch_attend_few(const AttendArgs& a, int rows, int d, int dtype, hipStream_t st) {
  ProfScope prof(ST_ATTEND, st);
  if (dtype == OBF_BF16) { if (d == 128) few_launch<uint16_t, 128>(a, rows, st); else few_launch<uint16_t, 64>(a, rows, st); }
  else { if (d == 128) few_launch<float, 128>(a, rows, st); else few_launch<float, 64>(a, rows, st); }
  return check_launch("attend");
}

template <typename ET, int D>
static void join_launch(const AttendArgs& a, hipStream_t st) {
  const int mass_blocks = a.logits ? (a.logit_tiles + JN_TILES - 1) / JN_TILES * a.S * a.H : 0;
  if (a.ranges > 8) {
    const int per = JN_THREADS / D, rows = (int)((a.rows + per - 1) / per);
    hipLaunchKernelGGL((k_attend_join<ET, D, 4>), dim3(rows + mass_blocks), dim3(JN_THREADS), 0, st, a, rows);
  } else {
    const int per = JN_THREADS * 4 / D, rows = a.ranges > 1 ? (int)((a.rows + per - 1) / per) : 0;
    hipLaunchKernelGGL((k_attend_join<ET, D, 1>), dim3(rows + mass_blocks), dim3(JN_THREADS), 0, st, a, rows);
  }
}

obf_status_t launch_attend_join(const AttendArgs& a, int d, int dtype, hipStream_t st) {
  ProfScope prof(ST_ATTEND_JOIN, st);
  if (dtype == OBF_BF16) { if (d == 128) join_launch<uint16_t, 128>(a, st); else join_launch<uint16_t, 64>(a, st); }
  else { if (d == 128) join_launch<float, 128>(a, st); else join_launch<float, 64>(a, st); }
  return check_launch("attend join");
}

}  // namespace obf
