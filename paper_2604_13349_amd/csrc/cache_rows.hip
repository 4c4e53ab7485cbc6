// Rows into a cache held in codes, and back: k_cache_write, k_cache_read.
//
// The arithmetic is that of the row code (codes.hpp); what these kernels add is the addressing: rows at the strides of a projection's output,
// a number of them per head, behind what the head holds, and back by row numbers.  16 columns a lane, keys and values in one launch.
//
// Bound by memory: 4 x 8 heads of 8192 rows as a projection leaves them, 4 bits, in 38 us and back in 29 (4.5 and 5.8 TB/s), the kept rows of 36 x 8 heads (800 to
// 1229), 8 bits, in 50 and back in 41 (4.5 and 5.5), 1229 of 8192 rows by their numbers in 52 (5.5 with the whole lines that rows of 64 bytes are part of); fp32 rows, 4 x 8 heads of
// 8192 to 4 bits, in 78 and back in 71 (3.9 and 4.3).
// One row a lane: 42, 35, 52, 56 and 63; four rows: 40, 32, 52, 44 and 52.  Stores that bypass the caches double the time of the way back.
#include "attend_codes.hpp"
#include "codes.hpp"

namespace obf {

// Head and rows of a lane: of PASSES rows, PER apart, the first.  CHUNKED, many rows per head: a workgroup takes PER * PASSES rows of one head, so that lengths and counts are
// scalars and a lane has the loads of all its rows in flight; otherwise rows of all heads one after another, one a lane.
struct CacheRow { int s, h, t; };
template <bool CHUNKED, int PER, int PASSES> __device__ __forceinline__ CacheRow cache_row(const CacheRowsArgs& a) {
  const uint32_t heads = a.H, sets = (uint32_t)a.S * heads, in = threadIdx.x / (QT_THREADS / PER);
  uint32_t set, t;
  if (CHUNKED) {
    const uint32_t chunk = blockIdx.x / sets;
    set = blockIdx.x - chunk * sets;
    t = chunk * (PER * PASSES) + in;
  } else {
    const uint32_t at = blockIdx.x * PER + in;
    set = at / (uint32_t)a.n_rows;
    t = set < sets ? at - set * a.n_rows : a.n_rows;
    set = min(set, sets - 1);
  }
  const uint32_t s = set / heads;
  return {(int)s, (int)(set - s * heads), (int)t};
}
// Rows that the head holds; none where that is no length.
__device__ __forceinline__ int cache_len(const CacheRowsArgs& a, const CacheRow r) {
  const int n = a.len ? a.len[(size_t)r.s * a.len_stride + r.h] : a.len_all;
  return n < 0 || n > a.token_stride ? 0 : n;
}

template <typename T, int D, int BITS, bool CHUNKED, int PASSES>
__global__ __launch_bounds__(QT_THREADS) void k_cache_write(const CacheRowsArgs a) {
  constexpr int LPR = D / QT_COLS, BYTES = D * BITS / 8, PER = QT_THREADS / LPR;
  const int part = threadIdx.x % LPR, which = blockIdx.y;
  const CacheRow r = cache_row<CHUNKED, PER, PASSES>(a);
  const int m = a.count ? a.count[(size_t)r.s * a.len_stride + r.h] : a.n_rows;
  if (m < 0 || m > a.n_rows || r.t >= m) return;                // all lanes of a row together, here and below
  const int before = cache_len(a, r) - m;
  const T* from = (const T*)a.x[which] + r.s * a.stride[which][0] + r.h * a.stride[which][1] + part * QT_COLS;
  const size_t head = (size_t)r.s * a.sample_rows + (size_t)r.h * a.token_stride;
  const CodeRows& c = a.rows[which];
  float x[PASSES][QT_COLS];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) load16(from + min(r.t + p * PER, m - 1) * a.stride[which][2], x[p]);
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int t = r.t + p * PER, j = before + t;
    uint32_t w[QT_COLS * BITS / 32];
    uint16_t scale, zero;
    encode16<LPR, BITS>(x[p], w, scale, zero);
    if (t >= m || j < 0) continue;
    const size_t row = head + j;
    store_codes16<BITS>((uint8_t*)c.codes + row * BYTES + part * (BYTES / LPR), w);
    if (part == 0) { ((uint16_t*)c.scale)[row] = scale; ((uint16_t*)c.zero)[row] = zero; }
  }
}

template <typename T, int D, int BITS, bool CHUNKED, int PASSES>
__global__ __launch_bounds__(QT_THREADS) void k_cache_read(const CacheRowsArgs a) {
  constexpr int LPR = D / QT_COLS, BYTES = D * BITS / 8, PER = QT_THREADS / LPR;
  const int part = threadIdx.x % LPR, which = blockIdx.y;
  const CacheRow r = cache_row<CHUNKED, PER, PASSES>(a);
  if (r.t >= a.n_rows) return;
  const int n = cache_len(a, r);
  if (n == 0) return;
  const int32_t* list = a.count ? a.count + ((size_t)r.s * a.H + r.h) * a.n_rows : nullptr;
  const size_t head = (size_t)r.s * a.sample_rows + (size_t)r.h * a.token_stride;
  const CodeRows& c = a.rows[which];
  T* to = (T*)a.x[which] + r.s * a.stride[which][0] + r.h * a.stride[which][1];
  int j[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int t = r.t + p * PER;
    j[p] = t >= a.n_rows ? -1 : list ? list[t] : t;
  }
  uint32_t w[PASSES][QT_COLS * BITS / 32];
  uint16_t scale[PASSES], zero[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const size_t row = head + min(max(j[p], 0), n - 1);
    load_codes_part<D, BITS>(c.codes + row * BYTES, part, w[p]);
    scale[p] = c.scale[row]; zero[p] = c.zero[row];
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (j[p] < 0 || j[p] >= n) continue;
    float x[QT_COLS];
    decode16<BITS>(w[p], scale[p], zero[p], x);
    store_part<D>(to + (r.t + p * PER) * a.stride[which][2], part, x);
  }
}

template <typename T, int D, int BITS>
static void cache_rows(const CacheRowsArgs& a, const bool write, hipStream_t st) {
  constexpr uint32_t PER = QT_THREADS * QT_COLS / D, PASSES = 2;
  const uint32_t sets = (uint32_t)a.S * a.H, rows = a.n_rows;
  const bool chunked = rows >= PER * PASSES;                    // (a head's last chunk may be nearly empty)
  const dim3 grid(chunked ? sets * ((rows + PER * PASSES - 1) / (PER * PASSES)) : (sets * rows + PER - 1) / PER, 2), threads(QT_THREADS);
  if (write) {
    if (chunked) hipLaunchKernelGGL((k_cache_write<T, D, BITS, true, PASSES>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((k_cache_write<T, D, BITS, false, 1>), grid, threads, 0, st, a);
  } else {
    if (chunked) hipLaunchKernelGGL((k_cache_read<T, D, BITS, true, PASSES>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((k_cache_read<T, D, BITS, false, 1>), grid, threads, 0, st, a);
  }
}

template <typename T>
static void cache_rows(const CacheRowsArgs& a, const int d, const int bits, const bool write, hipStream_t st) {
  if (d == 128) { if (bits == 8) cache_rows<T, 128, 8>(a, write, st); else cache_rows<T, 128, 4>(a, write, st); }
  else { if (bits == 8) cache_rows<T, 64, 8>(a, write, st); else cache_rows<T, 64, 4>(a, write, st); }
}

obf_status_t launch_cache_write(const CacheRowsArgs& a, int d, int dtype, int bits, hipStream_t st) {
  ProfScope prof(ST_CACHE_WRITE, st);
  if (dtype == OBF_BF16) cache_rows<uint16_t>(a, d, bits, true, st); else cache_rows<float>(a, d, bits, true, st);
  return check_launch("cache write");
}

obf_status_t launch_cache_read(const CacheRowsArgs& a, int d, int dtype, int bits, hipStream_t st) {
  ProfScope prof(ST_CACHE_READ, st);
  if (dtype == OBF_BF16) cache_rows<uint16_t>(a, d, bits, false, st); else cache_rows<float>(a, d, bits, false, st);
  return check_launch("cache read");
}

}  // namespace obf
