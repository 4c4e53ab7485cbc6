// A cache held in codes: what the kernels of cache_rows.hip, attend_codes.hip and the host side share.
#pragma once
#include "attend.hpp"

namespace obf {

// The codes of a cache's rows and the two half-precision numbers of each.
struct CodeRows { const uint8_t* codes; const uint16_t* scale; const uint16_t* zero; };

// Rows into, or out of, a cache: element (s, h, t) of x[0] (keys) and x[1] (values) at strides of elements.
struct CacheRowsArgs {
  void* x[2];
  long stride[2][3];
  CodeRows rows[2];
  const int32_t* len;        // nullable: len_all
  const int32_t* count;      // write: nullable, new rows per head; read: nullable, row numbers
  int len_all, len_stride, S, H, n_rows, token_stride;
  long sample_rows;
};
obf_status_t launch_cache_write(const CacheRowsArgs& a, int d, int dtype, int bits, hipStream_t st);
obf_status_t launch_cache_read(const CacheRowsArgs& a, int d, int dtype, int bits, hipStream_t st);

struct AttendCodesArgs {
  AttendArgs a;
  CodeRows k, v;
  // nullable: K's codes and V's values as half-precision numbers [set][stride][d], K's two numbers per row [set][stride], and for every kCodeFlagRows rows of
  // a set whether one of V's has no numbers, [set][flags]
  uint16_t *rows_k, *rows_v;
  uint2* numbers;
  uint8_t* bad;
  int flags;
};
constexpr int kCodeFlagRows = 64;
// Workgroups of eight waves of the kernel of few rows that a compute unit holds.
constexpr int few_codes_per_cu(const int d, const bool f32, const int bits) { return d == 64 || (bits == 4 && !f32) ? 2 : 1; }
constexpr int kCodesFewRows = 16;        // its query rows per workgroup
constexpr int kCodesManyRows = 64;       // query rows per KV head up to which all bf16 calls take it
obf_status_t launch_attend_codes_few(const AttendCodesArgs& c, int waves, int d, int dtype, int bits, hipStream_t st);
obf_status_t launch_attend_codes_tile(const AttendCodesArgs& c, int d, int bits, hipStream_t st);          // bf16, tiles of kAttendTileRows; with c.rows_k: over those rows, which it writes

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
union CodeFrag { uint32_t w[4]; f16x8 v; f16x2 h[4]; };

// The code in the middle of the range.
constexpr float code_middle(const int bits) { return (float)(1 << (bits - 1)); }

// The power of two that a query row whose largest element is `top` gets as half-precision numbers, so that it lies in [2^14, 2^15), and the one that takes it back.
__device__ __forceinline__ float query_power(const float top, float& unit) {
  // top in [2^(e - 1), 2^e), e from its bits (numbers below the normal ones as those next to them; an infinity as the largest ones); 2^127 at most
  const int e = min(max((int)(__float_as_uint(top) >> 23) - 126, -125), 128), up = min(127, 15 - e);
  unit = __uint_as_float((uint32_t)(127 - up) << 23 | (up == 127 ? 0x00400000u : 0u));
  return __uint_as_float((uint32_t)(up + 127) << 23);
}

}  // namespace obf
