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

struct AttendCodesArgs { AttendArgs a; CodeRows k, v; };
obf_status_t launch_attend_codes_few(const AttendCodesArgs& c, int tile_rows, int d, int dtype, int bits, hipStream_t st);

}  // namespace obf
