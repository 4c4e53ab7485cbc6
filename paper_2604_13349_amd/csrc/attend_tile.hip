// Attention of many query rows per KV head, bf16: prompts, and the rows of all samples against a shared message.
//
//   O_r = sum_j exp(x_rj - lse_r) V_j,  x_rj = q_r . k_j / sqrt(d) over the visible keys j,  lse_r = log sum_j exp(x_rj)
//
// A workgroup has 128 query rows (queries by the query heads of the group, so that the heads share the keys), a wave 32 of them.  K and V pass through
// LDS in tiles of 64 keys, two of them there: the loads of the next one, straight to LDS, run beside the products of the present one.  A wave takes
// K Q^T (keys by rows: a lane holds half the keys of one query row, so that the running maximum and sum need no exchange between lanes), the terms
// 2^(x - m), and V^T P^T, whose operand P^T is the first product's result as it lies in its lanes; V's operand is read from LDS transposed
// (ds_read_b64_tr_b16).  m follows the row's maximum only where that outgrows it by 2^8.
// Pieces of 16 bytes (K) and 64 bytes (V) of a row lie in LDS permuted by the row's number, so that the operand reads use all banks.
// P is rounded to bf16, 2^-8 of a weight at most: at this many rows the matrix pipe bounds the kernel, and the result is rounded as coarsely (8192 queries: 1.7e-3
// of the result's norm off 64 bits, where its own rounding makes 1.5e-3).  As two parts, as few rows have them: 957 us for 702, 250 for 189 (head_dim 64,
// window), 340 for 265 (8 x 500 queries behind a message).  A sample's few rows against a message have two parts too (64 samples behind 8192 rows: 41.7 us for 40.1).
//
// Two workgroups share a compute unit, so that one's products run beside the other's exponentials.  32 query heads of 8192 queries over 9421 rows: 710 us,
// 1.01 PFLOP/s (the library's largest product reaches 1.22), the matrix pipe busy half the time at a clock that its power holds at 1.7 to 1.95 GHz.  Two
// samples of 40 heads and 2048 queries 125 us, 0.77, the matrix pipe busy 0.34 of the cycles: 7.5 vector instructions beside the products per exponential, where
// the long prompt has 6.1 (starts and ends of the workgroups, rescaling, masked tiles), and a last round of workgroups that is not full.  head_dim 64, 16384
// queries, window of 1024: 190 us, 0.70 PFLOP/s, the vector work (a multiply-add, an exponential, an addition and a half of a maximum and a rounding per weight)
// takes 0.69 of the cycles, it or the products 0.84.  A raised wave priority during the products, operands of V read ahead of the exponentials: within 1 %.  The check for
// values that are not finite in every tile with masks, before it came to be made only where a result is none: 1 to 3 % more.
#include "attend_few.hpp"
#include "attend_tile.hpp"

namespace obf {

template <int D>
__global__ __launch_bounds__(AT_THREADS, 2) void k_attend_tile(const AttendArgs a) {
  __shared__ __attribute__((aligned(1024))) char sm[attend_tile_bytes<D>()];
  AttendKeys k = a.keys[0];
  if (a.fused) k = a.keys[1];
  attend_tile<D, 1>(a, k, blockIdx.x, sm);
}

// A message's rows against all samples' queries, and the samples' own rows against theirs, in one launch: products beside loads.  The weights of both enter V's
// product as two parts, so that what a sample gets does not hang on the number of samples beside it.
template <int D>
__global__ __launch_bounds__(AT_THREADS, 2) void k_attend_tile_few(const AttendArgs a) {
  constexpr int BYTES = attend_tile_bytes<D>() > (int)sizeof(FewShared<D, 1, 4>) ? attend_tile_bytes<D>() : (int)sizeof(FewShared<D, 1, 4>);
  __shared__ __attribute__((aligned(1024))) char sm[BYTES];
  const int block = blockIdx.x, tiles = a.keys[0].blocks;
  if (block < tiles) attend_tile<D, 2>(a, a.keys[0], block, sm);
  else attend_few<uint16_t, D, 1, 4>(a, a.keys[1], block - tiles, false, *(FewShared<D, 1, 4>*)sm);
}

obf_status_t launch_attend_tile(const AttendArgs& a, int d, hipStream_t st) {
  ProfScope prof(ST_ATTEND, st);
  const int blocks = a.keys[a.fused ? 1 : 0].blocks;
  if (d == 128) hipLaunchKernelGGL(k_attend_tile<128>, dim3(blocks), dim3(AT_THREADS), 0, st, a);
  else hipLaunchKernelGGL(k_attend_tile<64>, dim3(blocks), dim3(AT_THREADS), 0, st, a);
  return check_launch("attend");
}

obf_status_t launch_attend_tile_few(const AttendArgs& a, int d, hipStream_t st) {
  ProfScope prof(ST_ATTEND, st);
  const int blocks = a.keys[0].blocks + a.keys[1].blocks;
  if (d == 128) hipLaunchKernelGGL(k_attend_tile_few<128>, dim3(blocks), dim3(AT_THREADS), 0, st, a);
  else hipLaunchKernelGGL(k_attend_tile_few<64>, dim3(blocks), dim3(AT_THREADS), 0, st, a);
  return check_launch("attend");
}

}  // namespace obf
