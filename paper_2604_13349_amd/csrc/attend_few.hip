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
//
// Four waves of 16 rows each a workgroup.  Long caches are bound by their bytes: 16 x 8 heads of 8192 to 32768 rows 246 us, 5.4 TB/s read (a large copy moves
// 4.9), 48 x 8 heads of 1044 visible rows 37 us, 5.4; short ones by the launch and one chain of loads: 8 heads of 100 to 340 rows 8 us.  Eight waves a
// workgroup: 5 to 20 % slower but for few long heads (8 of 32000 rows 35 us for 38).  Loads one tile ahead: the same times.  With the logits kept (32 x 8 heads
// of 1000 to 4096 rows) 75 us for 60 without, where a second pass over the keys takes 58.  fp32, 3 x 2 heads, 333 queries of 2: 12 us, the chain of
// products of a wave (32 rows a workgroup: 21 us).  32 rows a workgroup of head_dim 128 do not fit the registers whole: 96 bytes a lane lie in scratch memory.
#include "attend_few.hpp"

namespace obf {

template <typename ET, int D, int NB, int NW>
__global__ __launch_bounds__(NW * 64, 2) void k_attend_few(const AttendArgs a) {
  __shared__ __attribute__((aligned(16))) FewShared<D, NB, NW> sm;
  int block = blockIdx.x;
  AttendKeys k = a.keys[0];
  const bool second = block >= k.blocks;
  if (second) { block -= k.blocks; k = a.keys[1]; }
  attend_few<ET, D, NB, NW>(a, k, block, !second, sm);
}

// Joins the ranges of a query row, O = sum_i 2^(lse_i - lse) O_i, and turns the logits of the own keys into weights, mass_j += sum_r 2^(x_rj - lse_r).
// GROUPS lanes share a row's ranges and a lane has four channels, so that the loads of many ranges are in flight; bound by the partial results' bytes, or
// by its launch (2048 rows of 17 ranges 6.6 us, 512 of four 5.6).  Workgroups behind those of the rows take 32 tiles of keys of a set each, for which they join the normalisers of its few rows themselves.
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
        // (as in the join of O: a part that is no number makes the normaliser none, and with it the weights of all that the row sees)
        const float base = top > -INFINITY ? top : 0.f;
        for (int i = 0; i < a.ranges; ++i) { const float x = a.part_lse[(size_t)i * a.rows + row]; if (x != -INFINITY) sum += attend_exp2(x - base); }
        ref = sum != 0.f ? base + attend_log2(sum) : -INFINITY;
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
  const bool any = sum != 0.f;                         // (also where it is no number)
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = any ? v[i] / sum : 0.f;
  const int t = (int)(row % a.T), hq = (int)(row / a.T % ((size_t)a.H * a.g)), s = (int)(row / a.T / ((size_t)a.H * a.g));
  if (c == 0 && a.lse) a.lse[row] = any ? (top + attend_log2(sum)) * 0.69314718055994531f : -INFINITY;
  store4((ET*)a.O + (size_t)s * a.os + (size_t)hq * a.oh + (size_t)t * a.ot + c, v);
}

// rows: of a workgroup's tile, 16, or 32 (bf16)
obf_status_t launch_attend_few(const AttendArgs& a, int rows, int d, int dtype, hipStream_t st) {
  ProfScope prof(ST_ATTEND, st);
  const dim3 grid(a.keys[0].blocks + (a.n_keys > 1 ? a.keys[1].blocks : 0)), threads(256);
  if (dtype == OBF_F32) {
    if (d == 128) hipLaunchKernelGGL((k_attend_few<float, 128, 1, 4>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((k_attend_few<float, 64, 1, 4>), grid, threads, 0, st, a);
  } else if (rows == 16) {
    if (d == 128) hipLaunchKernelGGL((k_attend_few<uint16_t, 128, 1, 4>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((k_attend_few<uint16_t, 64, 1, 4>), grid, threads, 0, st, a);
  } else {
    if (d == 128) hipLaunchKernelGGL((k_attend_few<uint16_t, 128, 2, 4>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((k_attend_few<uint16_t, 64, 2, 4>), grid, threads, 0, st, a);
  }
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
