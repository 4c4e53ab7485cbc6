// Attention over a relayed cache: what the kernels of attend_few.hip, attend_tile.hip, attend_mass.hip and the host side share.
#pragma once
#include "common.hpp"

namespace obf {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

// A set of keys and the query rows that read it: the samples' own rows (one set per sample and KV head), or the rows of a message that all samples share.
struct AttendKeys {
  const void* K;
  const void* V;
  const int32_t* len;        // nullable: len_all rows in every head
  const int32_t* sink_len;   // nullable: `sink` first rows in every head
  int len_all, len_stride;   // len_stride: entries of len and sink_len between samples
  int stride;                // rows between heads; a length above it is no length
  long sample_rows;          // rows between samples
  int sink, window, causal;
  int samples;               // sets of keys per KV head: S, or 1 for a message
  int row_samples;           // samples whose query rows read one set: 1, or S for a message
  // the launch: a workgroup per (set, tile of query rows, range of keys)
  int nsplit, split0;        // ranges, and the first one's place among the partial results
  int row_tiles, blocks;
};

struct AttendArgs {
  const void* Q;
  void* O;
  float* lse;                // nullable
  long qs, qh, qt, os, oh, ot;   // elements between samples, query heads, queries
  int S, H, g, T;
  uint32_t g_inv;            // ceil(2^23 / g)
  float scale2;              // log2(e) / sqrt(d)
  long rows;                 // S * H * g * T query rows; a row's number is its place in lse, [S][H * g][T]
  float* part_O;             // [ranges][rows][d] and [ranges][rows] (powers of two); used unless there is one range
  float* part_lse;
  int ranges;
  float* logits;             // nullable: [set][tile of 32 keys][query row of the set][32], in powers of two, -inf where hidden (one tile of rows only)
  float* mass;               // with logits: the weights go there
  int logit_tiles;           // tiles of a set, the most that its span can have
  AttendKeys keys[2];
  int n_keys;
  int fused;                 // a workgroup goes over both sets (the message first): keys[1] describes the launch
};

constexpr float kAttendSlack = 8.f;      // powers of two by which a row's terms may pass its reference

__device__ __forceinline__ float attend_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float attend_log2(float x) { return __builtin_amdgcn_logf(x); }

// The same in every lane of the wave, in a scalar register.
__device__ __forceinline__ int attend_uniform(const int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const void* attend_uniform(const void* p) {
  const uint64_t u = (uint64_t)p;
  return (const void*)((uint64_t)(uint32_t)attend_uniform((int)(uint32_t)u) | (uint64_t)(uint32_t)attend_uniform((int)(uint32_t)(u >> 32)) << 32);
}

// The set of keys of a workgroup, and its place `within` the set's workgroups: eight sets at a time go round the eight dies, so that a set's workgroups share a
// second-level cache; the next eight one die further, since the heads of one number may all be longer than the others.
__device__ __forceinline__ int attend_set(const int block, const int sets, const int per_set, int& within) {
  const int round = sets & 7 ? sets & -sets : 8, group = block / (round * per_set);
  within = block / round % per_set;
  return group * round + (block + group) % round;
}

// Rows of a head: a length that lies outside its storage (the -1 of a message that did not fit among them) counts as none.
__device__ __forceinline__ int attend_len(const AttendKeys& k, const int sample, const int h) {
  const int n = k.len ? k.len[(size_t)sample * k.len_stride + h] : k.len_all;
  return n < 0 || n > k.stride ? 0 : n;
}
__device__ __forceinline__ int attend_sink(const AttendKeys& k, const int sample, const int h) {
  return max(0, k.sink_len ? k.sink_len[(size_t)sample * k.len_stride + h] : k.sink);
}

// The keys that the query rows at positions pmin .. pmax of a head see, as one list of `count`: entry v is key v below `split` (the first rows, where the window
// begins behind them) and key v + skip from there on.
struct AttendSpan { int count, split, skip; };
__device__ __forceinline__ AttendSpan attend_span(const AttendKeys& k, const int n, const int sink, const int pmin, const int pmax) {
  AttendSpan s = {max(0, k.causal ? min(n, pmax + 1) : n), 0, 0};
  if (k.window > 0) {
    const int lo = pmin - k.window + 1, first = min(sink, s.count);
    if (lo > first) { s.split = first; s.skip = lo - first; s.count = max(first, s.count - s.skip); }
  }
  return s;
}
__device__ __forceinline__ int attend_key(const AttendSpan s, const int v) { return v < s.split ? v : v + s.skip; }

// The entries of a span that the query at position p sees: v <= hi and (v > lo or v < first); numbers relative to `from`, so that a tile's entries are
// constants.  (Where the span skips rows, every query sees those in front.)
struct AttendView { int hi, lo, first; };
__device__ __forceinline__ AttendView attend_view(const AttendKeys& k, const AttendSpan s, const int sink, const int p, const int from = 0) {
  return {(k.causal ? min(p - s.skip, s.count - 1) : s.count - 1) - from, (k.causal && k.window > 0 ? p - k.window - s.skip : -1) - from,
          (s.skip > 0 ? s.split : sink) - from};
}
__device__ __forceinline__ bool attend_sees(const AttendView v, const int j) { return (j <= v.hi) & ((j > v.lo) | (j < v.first)); }
// Whether some query at pmin .. pmax does not see some of the entries v .. v + width - 1.
__device__ __forceinline__ bool attend_cut(const AttendKeys& k, const AttendSpan s, const int sink, const int pmin, const int pmax, const int v, const int width) {
  const int last = v + width - 1;
  return last >= s.count || (k.causal && (last > pmin - s.skip || (k.window > 0 && v <= pmax - k.window - s.skip && last >= (s.skip > 0 ? s.split : sink))));
}

// Query row r of the rows that read a set of keys: query head, query and sample, and the row's number.
struct AttendRow { int s, gi, t; };
__device__ __forceinline__ AttendRow attend_row(const AttendArgs& a, const AttendKeys& k, const int set_sample, const int r) {
  AttendRow w;
  w.t = r / a.g;
  w.gi = r - w.t * a.g;
  w.s = set_sample;
  if (k.row_samples > 1) { w.s = w.t / a.T; w.t -= w.s * a.T; }
  return w;
}
// Row first + i (i < 128) of a sample's own rows, from the query and query head of row `first`: small numbers, so that a product with a reciprocal divides.
struct AttendStep { int t, gi; };
__device__ __forceinline__ AttendStep attend_step(const AttendArgs& a, const int first) { return {first / a.g, first % a.g}; }
__device__ __forceinline__ AttendRow attend_row(const AttendArgs& a, const AttendStep first, const int s, const int i) {
  const uint32_t n = (uint32_t)(first.gi + i), q = (n * a.g_inv) >> 23;        // exact for n < 512 and g <= 128
  return {s, (int)(n - q * a.g), first.t + (int)q};
}
__device__ __forceinline__ size_t attend_row_number(const AttendArgs& a, const int h, const AttendRow& w) {
  return ((size_t)w.s * a.H * a.g + (size_t)h * a.g + w.gi) * a.T + w.t;
}

constexpr int kAttendFewRows = 32;    // query rows per set of keys up to which the waves read the keys straight into registers
constexpr int kAttendTileRows = 128;
obf_status_t launch_attend_few(const AttendArgs& a, int tile_rows, int d, int dtype, hipStream_t st);
obf_status_t launch_attend_tile(const AttendArgs& a, int d, hipStream_t st);              // keys[0] alone, or (fused) both sets
obf_status_t launch_attend_tile_few(const AttendArgs& a, int d, hipStream_t st);          // keys[0] by tiles of many rows, keys[1] by tiles of 16
obf_status_t launch_attend_join(const AttendArgs& a, int d, int dtype, hipStream_t st);   // joins the ranges; adds the logits' weights to the mass

// Accumulated weights of the own rows.  tiles > 0: by the kernel of many rows, per steps of query rows in each of nsplit ranges, whose sums (unless there is one
// range) go to part, [range][set][stride].
struct AttendMass { float* mass; float* part; int nsplit, tiles, per; };
AttendMass plan_attend_mass(const AttendArgs& a, int dtype);
obf_status_t launch_attend_mass(const AttendArgs& a, int d, int dtype, const float* lse, const AttendMass& mass, hipStream_t st);

struct EvictArgs {
  const void* K; const void* V; const float* mass; const int32_t* pos;
  const int32_t* len; const int32_t* sink_len;
  int heads, len_all, in_stride, budget, recent, sink, out_stride, row_vec;
  void* K_out; void* V_out; float* mass_out; int32_t* pos_out; int32_t* idx; int32_t* len_out;
};
obf_status_t launch_evict(const EvictArgs& a, hipStream_t st);

}  // namespace obf
