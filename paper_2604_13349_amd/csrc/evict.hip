// Eviction by accumulated attention weight: per head the first rows, the newest rows and the rows of the largest mass are kept, in their order.
//
// First launch, a workgroup per head: the mass of the last row that is kept, by a histogram of an order-preserving integer image of the masses
// (2048 bins over the range that can still hold it) and again inside its bin until it is one key wide or its keys fit a list, whose entries then count the
// larger ones among themselves; then the list of kept rows by prefix counts.  All decisions are integer compares: exact, ties to the lowest index.  Heads of
// up to 32768 rows keep their keys in registers (288 heads of 8192 rows: 19 us, latency).  Second launch: the kept rows of K and V in 16-byte pieces, their masses and positions
// (1229 of 8192 rows in 288 heads: 77 us, 4.9 TB/s, a copy's rate).
#include "attend.hpp"

namespace obf {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t EvictRow;     // 16 bytes of a row

constexpr int EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64, EV_BINS = 2048;

// larger float <=> larger key
__device__ __forceinline__ uint32_t mass_key(const float f) {
  const uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int EV_LIST = 256;
constexpr long kEvictOwnRows = 128 << 10;      // bytes of a head's kept rows up to which its own workgroup copies them

// Rows r0, r0 + step, ... of a head, UNROLL at a time, by the threads of a row's 16-byte pieces c; n: rows kept, at least one.
template <int UNROLL>
__device__ __forceinline__ void evict_rows(const EvictArgs& a, const int head, const int n, const int r0, const int step, const int c) {
  const EvictRow *K = (const EvictRow*)a.K, *V = (const EvictRow*)a.V;
  EvictRow *K_out = (EvictRow*)a.K_out, *V_out = (EvictRow*)a.V_out;
  const int32_t* idx = a.idx + (size_t)head * a.out_stride;
  // (rows behind the end load the last one's again: no condition holds up a load)
  size_t from[UNROLL];
  EvictRow kv[UNROLL], vv[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) from[u] = (size_t)head * a.in_stride + idx[min(r0 + u * step, n - 1)];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) { kv[u] = K[from[u] * a.row_vec + c]; vv[u] = V[from[u] * a.row_vec + c]; }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u)
    if (r0 + u * step < n) {
      const size_t row = (size_t)head * a.out_stride + r0 + u * step;
      K_out[row * a.row_vec + c] = kv[u];
      V_out[row * a.row_vec + c] = vv[u];
    }
}

// What goes with row r.
__device__ __forceinline__ void evict_beside(const EvictArgs& a, const int head, const int r) {
  const size_t row = (size_t)head * a.out_stride + r, at = (size_t)head * a.in_stride + a.idx[row];
  a.mass_out[row] = a.mass[at];
  if (a.pos) a.pos_out[row] = a.pos[at];
}

// The list of a head's kept rows; returns their number, or -1.  PER keys per thread in registers, thread t those of rows t, t + 1024, ...; 0: read again for
// every pass.
template <int PER>
__device__ __forceinline__ int evict_list(const EvictArgs& a) {
  constexpr int REGS = PER > 0 ? PER : 1;
  __shared__ int hist[EV_BINS];
  __shared__ uint32_t wlo[EV_WAVES], whi[EV_WAVES], list[EV_LIST], s_key;
  __shared__ int wsum[EV_WAVES], s_bin, s_above, s_inside, s_listed;
  __shared__ int before_gt[REGS * EV_WAVES], before_eq[REGS * EV_WAVES], s_gt[EV_WAVES], s_eq[EV_WAVES];
  const int head = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* out = a.idx + (size_t)head * a.out_stride;
  const int n = a.len ? a.len[head] : a.len_all;
  const int first = min(max(0, a.sink_len ? a.sink_len[head] : a.sink), max(n, 0));
  const int kept = first + min(a.budget, n - first);
  if (n < 0 || n > a.in_stride || kept > a.out_stride) {            // no length, or no room: flagged, nothing of the head is written
    for (int i = tid; i < a.out_stride; i += EV_THREADS) out[i] = -1;
    if (tid == 0) a.len_out[head] = -1;
    return -1;
  }
  if (tid == 0) a.len_out[head] = kept;
  for (int i = kept + tid; i < a.out_stride; i += EV_THREADS) out[i] = -1;
  if (kept == n) {
    for (int i = tid; i < n; i += EV_THREADS) out[i] = i;
    return kept;
  }
  const int last = n - a.recent, want = a.budget - a.recent;        // of the rows first .. last - 1 the `want` of largest mass are kept
  for (int i = tid; i < first; i += EV_THREADS) out[i] = i;
  for (int i = tid; i < a.recent; i += EV_THREADS) out[first + want + i] = last + i;
  if (want == 0) return kept;
  const float* mass = a.mass + (size_t)head * a.in_stride;
  uint32_t key[REGS];
  if (PER > 0) {
#pragma unroll
    for (int c = 0; c < REGS; ++c) { const int i = first + c * EV_THREADS + tid; key[c] = i < last ? mass_key(mass[i]) : 0u; }
  }
  // f(key, place) for the rows of this thread
  const auto each = [&](const auto f) {
    if (PER > 0) {
#pragma unroll
      for (int c = 0; c < REGS; ++c) if (first + c * EV_THREADS + tid < last) f(key[c]);
    } else {
      for (int i = first + tid; i < last; i += EV_THREADS) f(mass_key(mass[i]));
    }
  };
  uint32_t lo = 0xffffffffu, hi = 0u;
  each([&](const uint32_t k) { lo = min(lo, k); hi = max(hi, k); });
  for (int off = 32; off > 0; off >>= 1) { lo = min(lo, (uint32_t)__shfl_xor((int)lo, off)); hi = max(hi, (uint32_t)__shfl_xor((int)hi, off)); }
  if (lane == 0) { wlo[wave] = lo; whi[wave] = hi; }
  if (tid == 0) s_listed = 0;
  hist[tid] = 0; hist[tid + EV_THREADS] = 0;
  __syncthreads();
  lo = 0xffffffffu; hi = 0u;
#pragma unroll
  for (int w = 0; w < EV_WAVES; ++w) { lo = min(lo, wlo[w]); hi = max(hi, whi[w]); }
  int need = want;                                                  // rank wanted among the keys of [lo, hi]
  while (lo < hi) {                                                 // uniform; the histogram is clear
    const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);      // (hi - lo) >> shift < EV_BINS
    each([&](const uint32_t k) {
      const uint32_t o = k - lo;                                    // keys below the range wrap to above it
      if (o <= hi - lo) atomicAdd(&hist[o >> shift], 1);
    });
    __syncthreads();
    // from the top: this thread's bins are top and top - 1
    const int top = EV_BINS - 1 - 2 * tid;
    const int c0 = hist[top], c1 = hist[top - 1];
    int inc = c0 + c1;
    for (int off = 1; off < 64; off <<= 1) { const int x = __shfl_up(inc, off); if (lane >= off) inc += x; }
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    int before = inc - c0 - c1;
#pragma unroll
    for (int w = 0; w < EV_WAVES; ++w) before += w < wave ? wsum[w] : 0;
    if (before < need && need <= before + c0) { s_bin = top; s_above = before; s_inside = c0; }
    else if (before + c0 < need && need <= before + c0 + c1) { s_bin = top - 1; s_above = before + c0; s_inside = c1; }
    hist[top] = 0; hist[top - 1] = 0;
    __syncthreads();
    need -= s_above;
    const uint64_t bin_top = (uint64_t)lo + (((uint64_t)s_bin + 1u) << shift) - 1u;
    if (bin_top < (uint64_t)hi) hi = (uint32_t)bin_top;
    lo += (uint32_t)s_bin << shift;
    if (lo < hi && s_inside <= EV_LIST) {
      each([&](const uint32_t k) { if (k - lo <= hi - lo) list[atomicAdd(&s_listed, 1)] = k; });
      __syncthreads();
      if (tid < s_inside) {
        const uint32_t k = list[tid];
        int gt = 0, ge = 0;
        for (int j = 0; j < s_inside; ++j) { gt += list[j] > k; ge += list[j] >= k; }
        if (gt < need && need <= ge) { s_key = k; s_above = gt; }   // the same from every copy of the key
      }
      __syncthreads();
      lo = hi = s_key;
      need -= s_above;
      break;
    }
    __syncthreads();                                                // s_bin and wsum are written again
  }
  // keys above lo are kept; of those equal to it the first `need`
  const uint64_t under = (1ull << lane) - 1ull;
  if (PER > 0) {
#pragma unroll
    for (int c = 0; c < REGS; ++c) {
      const bool valid = first + c * EV_THREADS + tid < last;
      const uint64_t gt = __ballot(valid && key[c] > lo), eq = __ballot(valid && key[c] == lo);
      if (lane == 0) { before_gt[c * EV_WAVES + wave] = __popcll(gt); before_eq[c * EV_WAVES + wave] = __popcll(eq); }
    }
    __syncthreads();
    // exclusive sums over (chunk, wave), the rows' order
    const int mine_gt = tid < REGS * EV_WAVES ? before_gt[tid] : 0, mine_eq = tid < REGS * EV_WAVES ? before_eq[tid] : 0;
    int g = mine_gt, e = mine_eq;
    for (int off = 1; off < 64; off <<= 1) { const int x = __shfl_up(g, off), y = __shfl_up(e, off); if (lane >= off) { g += x; e += y; } }
    if (lane == 63) { s_gt[wave] = g; s_eq[wave] = e; }
    __syncthreads();
    if (tid < REGS * EV_WAVES) {
      g -= mine_gt; e -= mine_eq;
      for (int w = 0; w < wave; ++w) { g += s_gt[w]; e += s_eq[w]; }
      before_gt[tid] = g; before_eq[tid] = e;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < REGS; ++c) {
      const int i = first + c * EV_THREADS + tid;
      const bool gt = i < last && key[c] > lo, eq = i < last && key[c] == lo;
      const uint64_t bg = __ballot(gt), be = __ballot(eq);
      const int eq_before = before_eq[c * EV_WAVES + wave] + __popcll(be & under);
      if (gt || (eq && eq_before < need)) out[first + before_gt[c * EV_WAVES + wave] + __popcll(bg & under) + min(eq_before, need)] = i;
    }
  } else {
    int at = first, equal = 0;                                      // rows kept, and rows equal to lo, before this chunk
    for (int c = first; c < last; c += EV_THREADS) {
      const int i = c + tid;
      const uint32_t k = i < last ? mass_key(mass[i]) : 0u;
      const bool gt = i < last && k > lo, eq = i < last && k == lo;
      const uint64_t bg = __ballot(gt), be = __ballot(eq);
      if (lane == 0) { s_gt[wave] = __popcll(bg); s_eq[wave] = __popcll(be); }
      __syncthreads();
      int g = __popcll(bg & under), e = equal + __popcll(be & under), tg = 0, te = 0;
#pragma unroll
      for (int w = 0; w < EV_WAVES; ++w) { if (w < wave) { g += s_gt[w]; e += s_eq[w]; } tg += s_gt[w]; te += s_eq[w]; }
      // kept rows before this one: the larger ones, and of the equal ones as many as were still needed
      const int eq_before = min(e, need) - min(equal, need);
      if (gt || (eq && e < need)) out[at + g + eq_before] = i;
      at += tg + min(equal + te, need) - min(equal, need);
      equal += te;
      __syncthreads();
    }
  }
  return kept;
}

// with_rows: the workgroup copies its head's rows too.
template <int PER>
__global__ __launch_bounds__(EV_THREADS) void k_evict_select(const EvictArgs a, const int with_rows) {
  const int n = evict_list<PER>(a);
  if (!with_rows || n <= 0) return;
  __syncthreads();                                                  // (the list, written by the whole workgroup)
  const int step = EV_THREADS / a.row_vec, c = threadIdx.x % a.row_vec;
  for (int r = (int)threadIdx.x / a.row_vec; r < n; r += 2 * step) evict_rows<2>(a, blockIdx.x, n, r, step, c);
  for (int r = threadIdx.x; r < n; r += EV_THREADS) evict_beside(a, blockIdx.x, r);
}

constexpr int EG_THREADS = 256, EG_UNROLL = 4;

__global__ __launch_bounds__(EG_THREADS) void k_evict_rows(const EvictArgs a) {
  const int head = blockIdx.y, per = EG_THREADS / a.row_vec;
  const int block0 = (int)blockIdx.x * per * EG_UNROLL;
  const int n = a.len_out[head];                                    // -1 for a head that was flagged
  if (block0 >= n) return;
  evict_rows<EG_UNROLL>(a, head, n, block0 + (int)threadIdx.x / a.row_vec, per, threadIdx.x % a.row_vec);
  // a lane per row for what goes with it
  const int r = block0 + (int)threadIdx.x;
  if ((int)threadIdx.x < per * EG_UNROLL && r < n) evict_beside(a, head, r);
}

obf_status_t launch_evict(const EvictArgs& a, hipStream_t st) {
  ProfScope prof(ST_EVICT, st);
  // A head's own workgroup copies its rows where they are few: one launch for two (us, two and one, heads x rows kept of 512 bytes: 2 x 64 8.9 - 7.3,
  // 64 x 205 12.8 - 11.5, 288 x 120 22.7 - 21.0, 1000 x 100 41 - 37; 8 x 400 12.0 - 13.0, 288 x 1229 93 - 110).  First rows counted per head may be any number
  // of them that fits, unless `sink` says about how many (8 x 8064 rows: 28 - 109).
  const long most = a.sink_len && a.sink == 0 ? (long)a.out_stride : (long)a.budget + a.sink, bytes = (a.out_stride < most ? a.out_stride : most) * a.row_vec * 32;
  const int with_rows = bytes <= kEvictOwnRows;
  const dim3 grid(a.heads), threads(EV_THREADS);
  if (a.in_stride <= EV_THREADS) hipLaunchKernelGGL(k_evict_select<1>, grid, threads, 0, st, a, with_rows);
  else if (a.in_stride <= 8 * EV_THREADS) hipLaunchKernelGGL(k_evict_select<8>, grid, threads, 0, st, a, with_rows);
  else if (a.in_stride <= 32 * EV_THREADS) hipLaunchKernelGGL(k_evict_select<32>, grid, threads, 0, st, a, with_rows);
  else hipLaunchKernelGGL(k_evict_select<0>, grid, threads, 0, st, a, with_rows);
  if (!with_rows) {
    const int per = EG_THREADS / a.row_vec * EG_UNROLL;
    hipLaunchKernelGGL(k_evict_rows, dim3((a.out_stride + per - 1) / per, a.heads), dim3(EG_THREADS), 0, st, a);
  }
  return check_launch("evict");
}

}  // namespace obf
