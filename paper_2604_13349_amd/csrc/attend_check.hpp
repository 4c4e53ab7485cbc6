// Host side that the calls on caches share: what a descriptor says, argument checks.
#pragma once
#include "attend.hpp"

namespace obf {

constexpr int kAttendMaxStride = 1 << 24;     // rows between heads
constexpr int kAttendMaxQueries = 1 << 20;
constexpr int kAttendMaxGroup = 128;

// Whether rows of `row` elements meet, at strides[i] between the counts[i] of each of three dimensions: from the smallest stride up, each has to pass what lies
// below it.
bool rows_meet(const int64_t (&strides)[3], const int64_t (&counts)[3], int64_t row);
obf_status_t check_attend(const obf_attend_t* c);
obf_status_t check_aligned(const char* name, const void* p);
obf_status_t check_attend_ws(size_t need, const void* ws, size_t ws_bytes);

// Queries, and the samples' own rows, without the launch.
AttendArgs attend_args(const obf_attend_t* c);
AttendKeys attend_own(const obf_attend_t* c);

// Memory that a call certainly reads or writes: all of a tensor without gaps, the first run of one with gaps (whose gaps may hold another).
struct Region { const char* name; const void* p; size_t bytes; };
obf_status_t check_apart(const Region* outs, int n_outs, const Region* ins, int n_ins);
// Elements of a tensor of rows of d elements, S by heads by T of them at the strides s, h, t.
size_t region_rows(long S, long heads, long T, long d, long s, long h, long t);
// Rows of a cache, entries of its lengths.
size_t region_cache(const AttendArgs& a, const AttendKeys& k);
size_t region_lens(const AttendArgs& a, const AttendKeys& k);

}  // namespace obf
