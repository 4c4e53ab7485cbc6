// Rows into a cache held in codes, and back: k_cache_write, k_cache_read.
//
// The arithmetic is that of the row code (codes.hpp); what these kernels add is the addressing: rows at the strides of a projection's output,
// a number of them per head, behind what the head holds, and back by row numbers.  16 columns a lane, keys and values in one launch.
#include "attend_codes.hpp"
#include "codes.hpp"

namespace obf {

// Row `at` of the launch's rows: sample, head and number.
struct CacheRow { int s, h, t; };
__device__ __forceinline__ CacheRow cache_row(const CacheRowsArgs& a, const uint32_t at) {
  const uint32_t set = at / (uint32_t)a.n_rows, s = set / (uint32_t)a.H;
  return {(int)s, (int)(set - s * a.H), (int)(at - set * a.n_rows)};
}
// Rows that the head holds; none where that is no length.
__device__ __forceinline__ int cache_len(const CacheRowsArgs& a, const CacheRow r) {
  const int n = a.len ? a.len[(size_t)r.s * a.len_stride + r.h] : a.len_all;
  return n < 0 || n > a.token_stride ? 0 : n;
}

template <typename T, int D, int BITS>
__global__ __launch_bounds__(QT_THREADS) void k_cache_write(const CacheRowsArgs a) {
  constexpr int LPR = D / QT_COLS, BYTES = D * BITS / 8;
  const uint32_t at = blockIdx.x * (QT_THREADS / LPR) + threadIdx.x / LPR;
  const int part = threadIdx.x % LPR, which = blockIdx.y;
  if (at >= (uint32_t)a.S * a.H * a.n_rows) return;             // all lanes of a row together, here and below
  const CacheRow r = cache_row(a, at);
  const int m = a.count ? a.count[(size_t)r.s * a.len_stride + r.h] : a.n_rows;
  if (m > a.n_rows || r.t >= m) return;
  const int j = cache_len(a, r) - m + r.t;
  if (j < 0) return;
  float x[QT_COLS];
  load16((const T*)a.x[which] + r.s * a.stride[which][0] + r.h * a.stride[which][1] + r.t * a.stride[which][2] + part * QT_COLS, x);
  uint32_t w[QT_COLS * BITS / 32];
  uint16_t scale, zero;
  encode16<LPR, BITS>(x, w, scale, zero);
  const size_t row = (size_t)r.s * a.sample_rows + (size_t)r.h * a.token_stride + j;
  const CodeRows& c = a.rows[which];
  store_codes16<BITS>((uint8_t*)c.codes + row * BYTES + part * (BYTES / LPR), w);
  if (part == 0) { ((uint16_t*)c.scale)[row] = scale; ((uint16_t*)c.zero)[row] = zero; }
}

template <typename T, int D, int BITS>
__global__ __launch_bounds__(QT_THREADS) void k_cache_read(const CacheRowsArgs a) {
  constexpr int LPR = D / QT_COLS, BYTES = D * BITS / 8;
  const uint32_t at = blockIdx.x * (QT_THREADS / LPR) + threadIdx.x / LPR;
  const int part = threadIdx.x % LPR, which = blockIdx.y;
  if (at >= (uint32_t)a.S * a.H * a.n_rows) return;
  const CacheRow r = cache_row(a, at);
  const int j = a.count ? a.count[at] : r.t;
  if (j < 0 || j >= cache_len(a, r)) return;
  const size_t row = (size_t)r.s * a.sample_rows + (size_t)r.h * a.token_stride + j;
  const CodeRows& c = a.rows[which];
  uint32_t w[QT_COLS * BITS / 32];
  load_codes16<BITS>(c.codes + row * BYTES + part * (BYTES / LPR), w);
  float x[QT_COLS];
  decode16<BITS>(w, c.scale[row], c.zero[row], x);
  store16((T*)a.x[which] + r.s * a.stride[which][0] + r.h * a.stride[which][1] + r.t * a.stride[which][2] + part * QT_COLS, x);
}

template <typename T, int D, int BITS>
static void cache_rows(const CacheRowsArgs& a, const bool write, hipStream_t st) {
  constexpr uint32_t rows = QT_THREADS * QT_COLS / D;
  const dim3 grid(((uint32_t)a.S * a.H * a.n_rows + rows - 1) / rows, 2), threads(QT_THREADS);
  if (write) hipLaunchKernelGGL((k_cache_write<T, D, BITS>), grid, threads, 0, st, a);
  else hipLaunchKernelGGL((k_cache_read<T, D, BITS>), grid, threads, 0, st, a);
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
