// Entry points of the operators that read and thin out a relayed cache: argument checks, workspace, launches.
#include "attend.hpp"

namespace obf {

constexpr int kAttendMaxStride = 1 << 24;     // rows between heads
constexpr int kAttendMaxQueries = 1 << 20;
constexpr int kAttendMaxGroup = 128;

static bool attend_overlap(const void* a, size_t an, const void* b, size_t bn) {
  return a && b && (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}

// Whether rows of `row` elements meet, at strides[i] between the counts[i] of each of three dimensions: from the smallest stride up, each has to pass what lies
// below it.
static bool rows_meet(const int64_t (&strides)[3], const int64_t (&counts)[3], const int64_t row) {
  __int128 span = row;                                 // (before the limits of the numbers are checked)
  bool done[3] = {counts[0] == 1, counts[1] == 1, counts[2] == 1};
  for (;;) {
    int next = -1;
    for (int i = 0; i < 3; ++i) if (!done[i] && (next < 0 || strides[i] < strides[next])) next = i;
    if (next < 0) return false;
    if (strides[next] < span) return true;
    done[next] = true;
    span += (__int128)(counts[next] - 1) * strides[next];
  }
}

static obf_status_t check_attend(const obf_attend_t* c) {
  if (!c) { set_error("attend: descriptor is NULL"); return OBF_ERR_INVALID_ARG; }
  if (c->n_samples < 1 || c->n_kv_heads < 1 || c->group < 1 || c->n_queries < 1 || c->token_stride < 1) {
    set_error("attend: n_samples, n_kv_heads, group, n_queries, token_stride must all be >= 1");
    return OBF_ERR_INVALID_ARG;
  }
  if (c->dtype != OBF_F32 && c->dtype != OBF_BF16) { set_error("attend: unknown dtype %d", c->dtype); return OBF_ERR_INVALID_ARG; }
  if (c->window < 0 || c->sink < 0) { set_error("attend: window and sink must not be negative"); return OBF_ERR_INVALID_ARG; }
  if (c->window > 0 && !c->causal) { set_error("attend: a window needs causal queries"); return OBF_ERR_INVALID_ARG; }
  if (c->kv_len_all < 0 || c->kv_len_all > c->token_stride) { set_error("attend: kv_len_all outside [0, token_stride]"); return OBF_ERR_INVALID_ARG; }
  if (c->len_stride < 0 || (c->len_stride > 0 && c->len_stride < c->n_kv_heads)) { set_error("attend: len_stride below n_kv_heads"); return OBF_ERR_INVALID_ARG; }
  if (c->sample_stride < 0 || (c->sample_stride > 0 && c->sample_stride < (int64_t)c->n_kv_heads * c->token_stride)) {
    set_error("attend: sample_stride below n_kv_heads * token_stride");
    return OBF_ERR_INVALID_ARG;
  }
  const int unit = c->dtype == OBF_BF16 ? 8 : 4;
  for (int i = 0; i < 3; ++i)
    if (c->q_stride[i] < 0 || c->q_stride[i] % unit || c->o_stride[i] < 0 || c->o_stride[i] % unit) {
      set_error("attend: strides of Q and O must be multiples of 16 bytes and not negative");
      return OBF_ERR_INVALID_ARG;
    }
  if ((c->o_stride[0] || c->o_stride[1] || c->o_stride[2]) && rows_meet(c->o_stride, {c->n_samples, (int64_t)c->n_kv_heads * c->group, c->n_queries}, c->head_dim)) {
    set_error("attend: rows of O must not overlap");
    return OBF_ERR_INVALID_ARG;
  }
  if (c->head_dim != 64 && c->head_dim != 128) { set_error("head_dim %d unsupported (64 or 128)", c->head_dim); return OBF_ERR_UNSUPPORTED; }
  if (c->token_stride > kAttendMaxStride) { set_error("attend: token_stride above the supported %d", kAttendMaxStride); return OBF_ERR_UNSUPPORTED; }
  if (c->n_queries > kAttendMaxQueries) { set_error("attend: n_queries above the supported %d", kAttendMaxQueries); return OBF_ERR_UNSUPPORTED; }
  if (c->group > kAttendMaxGroup) { set_error("attend: group above the supported %d", kAttendMaxGroup); return OBF_ERR_UNSUPPORTED; }
  if ((int64_t)c->n_samples * c->n_kv_heads > 65535) { set_error("attend: more than 65535 heads in one call"); return OBF_ERR_UNSUPPORTED; }
  if ((int64_t)c->n_samples * c->n_kv_heads * c->group * c->n_queries > ((int64_t)1 << 26)) {
    set_error("attend: more than 2^26 query rows in one call");
    return OBF_ERR_UNSUPPORTED;
  }
  if ((int64_t)c->n_samples * c->n_kv_heads * c->token_stride > ((int64_t)1 << 30)) {
    set_error("attend: more than 2^30 cache rows in one call");
    return OBF_ERR_UNSUPPORTED;
  }
  return OBF_OK;
}

static obf_status_t check_aligned(const char* name, const void* p) {
  if (!p) { set_error("%s is NULL", name); return OBF_ERR_INVALID_ARG; }
  if ((uintptr_t)p & 15) { set_error("%s must be 16-byte aligned", name); return OBF_ERR_INVALID_ARG; }
  return OBF_OK;
}

// The launch of one call: which kernel goes over which set of keys, tiles, ranges; and the workspace, in the order partial sums, partial normalisers, row
// normalisers, partial weights.
struct AttendPlan {
  AttendArgs a;
  int tile_rows[2];            // query rows of a workgroup's tile, by set of keys; kAttendTileRows: the kernel of many rows
  AttendMass ms;
  bool keep_logits;
  size_t part_O, part_lse, lse, mass, logits, total;
};

// sinks_per_head: sink_len is given (or may be, where a workspace is asked for: its size is the larger one then).
static AttendPlan plan_attend(const obf_attend_t* c, int prefix_stride, bool with_mass, bool sinks_per_head) {
  AttendPlan p;
  AttendArgs& a = p.a;
  a = AttendArgs();
  a.S = c->n_samples; a.H = c->n_kv_heads; a.g = c->group; a.T = c->n_queries;
  a.g_inv = ((1u << 23) + a.g - 1) / a.g;
  const long d = c->head_dim, hq = (long)a.H * a.g;
  const bool qd = c->q_stride[0] || c->q_stride[1] || c->q_stride[2], od = c->o_stride[0] || c->o_stride[1] || c->o_stride[2];
  a.qs = qd ? c->q_stride[0] : hq * a.T * d; a.qh = qd ? c->q_stride[1] : a.T * d; a.qt = qd ? c->q_stride[2] : d;
  a.os = od ? c->o_stride[0] : hq * a.T * d; a.oh = od ? c->o_stride[1] : a.T * d; a.ot = od ? c->o_stride[2] : d;
  a.scale2 = (float)(1.4426950408889634 / (d == 128 ? 11.313708498984761 : 8.0));
  a.rows = (long)a.S * hq * a.T;
  a.n_keys = 0;
  if (prefix_stride > 0) {
    AttendKeys& k = a.keys[a.n_keys++];
    k = AttendKeys();
    k.stride = prefix_stride; k.samples = 1; k.row_samples = a.S;
  }
  AttendKeys& k = a.keys[a.n_keys++];
  k = AttendKeys();
  k.len_all = c->kv_len_all; k.len_stride = c->len_stride ? c->len_stride : a.H;
  k.stride = c->token_stride; k.sample_rows = c->sample_stride ? c->sample_stride : (long)a.H * c->token_stride;
  k.sink = c->sink;
  k.window = c->window < c->token_stride ? c->window : 0;      // (positions lie below the stride: the others hide nothing)
  k.causal = c->causal != 0;
  k.samples = a.S; k.row_samples = 1;
  const long own_rows = (long)a.T * a.g;
  // A sample's queries fill tiles of many rows by themselves: one pass over the message and the own rows, no partial results of the message.
  a.fused = a.n_keys > 1 && c->dtype == OBF_BF16 && own_rows > kAttendFewRows;
  // Up to 32 rows the waves read the keys straight into registers for 16 rows at a time; for 17 to 32 rows at once where there are keys enough to fill the chip
  // (us, 16 and 32 rows: 4 x 8 heads of 1000 rows 13.7 - 18.7, 32 x 8 of 1000 41.8 - 41.9, 16 x 8 of 4000 46 - 29, 8 x 8 of 32000 309 - 226).  fp32 caches have
  // no other kernel, their 32 rows do not fit the registers (2 x 8 heads, 2048 queries of 4: 1009 - 1319).
  for (int i = 0; i < a.n_keys; ++i) {
    const long r = a.keys[i].row_samples * own_rows;
    const bool many = a.n_keys == 1 && r > 16 && (long)a.S * a.H * c->token_stride >= (1L << 17);
    p.tile_rows[i] = c->dtype != OBF_BF16 ? 16 : r > kAttendFewRows ? kAttendTileRows : many ? 32 : 16;
  }
  a.ranges = 0;
  for (int i = a.fused ? 1 : 0; i < a.n_keys; ++i) {
    AttendKeys& s = a.keys[i];
    s.row_tiles = (int)((s.row_samples * own_rows + p.tile_rows[i] - 1) / p.tile_rows[i]);
    // Rows that a tile sees, at most; first rows counted per head may be any number of them, unless `sink` says about how many (us, ranges for the window and
    // for all rows: 8 heads of 8200 rows, window of 64, 8000 first rows, one query 73 - 17.5, 64 queries 277 - 34; 1 to 40 first rows, one query 9.4 - 13.4).
    const bool few_seen = s.window > 0 && (s.sink > 0 || !sinks_per_head);
    const long blocks = (long)s.row_tiles * s.samples * a.H, seen = few_seen ? (long)s.window + s.sink + p.tile_rows[i] / a.g + 1 : s.stride;
    const long rows = (seen < s.stride ? seen : s.stride) + (a.fused ? a.keys[0].stride : 0);
    // Ranges where the sets do not fill the chip, two workgroups per compute unit (one where a message's tiles of many rows share it with the own rows' loads);
    // none for short caches, whose join would take longer (us, ranges and none: 128 sets of 590 rows 17.0 - 15.4, 256 of 1000 31 - 28, of 1500 43.3 - 39.7,
    // 252 workgroups of fp32 rows 20 - 13.5; 64 sets of 1000 15.8 - 18.6, 128 of 2000 32.4 - 34.7; 8 sets of 340 9.8 - 8.1, of 1000 11.8 - 12.6).
    const bool none = rows <= 512 || (blocks >= 128 && rows <= 8 * blocks && rows <= 2048);
    const long most_ranges = none ? 1 : (rows + 255) / 256, fill = s.row_samples > 1 && p.tile_rows[i] == kAttendTileRows ? kNumCU : 2 * kNumCU;
    const long want = (fill + blocks - 1) / blocks;
    s.nsplit = (int)(want < most_ranges ? want : most_ranges);
    s.split0 = a.ranges;
    a.ranges += s.nsplit;
    s.blocks = (int)(blocks * s.nsplit);
  }
  size_t at = 0;
  p.part_O = at;
  if (a.ranges > 1) at += (size_t)a.ranges * a.rows * d * sizeof(float);
  p.part_lse = at;
  if (a.ranges > 1) at += ((size_t)a.ranges * a.rows * sizeof(float) + 255) & ~(size_t)255;
  p.lse = at;
  if (with_mass) at += ((size_t)a.rows * sizeof(float) + 255) & ~(size_t)255;
  p.ms = plan_attend_mass(a, c->dtype);
  p.mass = at;
  if (with_mass && p.ms.nsplit > 1) at += ((size_t)p.ms.nsplit * a.S * a.H * c->token_stride * sizeof(float) + 255) & ~(size_t)255;
  // Few query rows: the logits are kept and weighted at the end, 4 bytes a row and key written and read beside the 2 d or 4 d of a key, where a second pass
  // would read the keys again.
  const bool keep = a.n_keys == 1 && own_rows <= p.tile_rows[0] && own_rows <= kAttendFewRows;
  p.logits = at;
  a.logit_tiles = (c->token_stride + 31) / 32;
  if (with_mass && keep) at += (size_t)a.rows * a.logit_tiles * 32 * sizeof(float);
  if (at == 0) at = 256;
  p.total = at;
  p.keep_logits = keep;
  return p;
}

static obf_status_t launch_plan(const AttendPlan& p, int d, int dtype, hipStream_t st) {
  if (p.tile_rows[0] != kAttendTileRows) return launch_attend_few(p.a, p.tile_rows[0], d, dtype, st);
  return p.a.n_keys == 1 || p.a.fused ? launch_attend_tile(p.a, d, st) : launch_attend_tile_few(p.a, d, st);
}

static obf_status_t check_attend_ws(const AttendPlan& p, const void* ws, size_t ws_bytes) {
  if (!ws) { set_error("workspace is NULL"); return OBF_ERR_INVALID_ARG; }
  if (((uintptr_t)ws & 255) != 0) { set_error("workspace must be 256-byte aligned"); return OBF_ERR_INVALID_ARG; }
  if (ws_bytes < p.total) { set_error("workspace too small: %zu bytes given, %zu needed", ws_bytes, p.total); return OBF_ERR_WORKSPACE_TOO_SMALL; }
  return OBF_OK;
}

// Memory that a call certainly reads or writes: all of a tensor without gaps, the first run of one with gaps (whose gaps may hold another).
struct Region { const char* name; const void* p; size_t bytes; };

static obf_status_t check_apart(const Region* outs, const int n_outs, const Region* ins, const int n_ins) {
  for (int i = 0; i < n_outs; ++i) {
    const auto meets = [&](const Region& r) {
      if (!attend_overlap(outs[i].p, outs[i].bytes, r.p, r.bytes)) return false;
      set_error("%s must not overlap %s", outs[i].name, r.name);
      return true;
    };
    for (int j = 0; j < n_ins; ++j) if (meets(ins[j])) return OBF_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j) if (meets(outs[j])) return OBF_ERR_INVALID_ARG;
  }
  return OBF_OK;
}

// Elements of a Q or O.
static size_t region_rows(const AttendArgs& a, const long d, const long s, const long h, const long t) {
  const long heads = (long)a.H * a.g, all = a.S * heads * a.T * d;
  if ((a.S - 1) * s + (heads - 1) * h + (a.T - 1) * t + d == all) return (size_t)all;
  if (a.T > 1 && t != d) return (size_t)d;
  if (heads > 1 && h != a.T * d) return (size_t)(a.T * d);
  return (size_t)(heads * a.T * d);
}
// Rows of a cache, entries of its lengths.
static size_t region_cache(const AttendArgs& a, const AttendKeys& k) {
  const size_t one = (size_t)a.H * k.stride;
  return k.samples > 1 && (size_t)k.sample_rows == one ? one * k.samples : one;
}
static size_t region_lens(const AttendArgs& a, const AttendKeys& k) { return (size_t)a.H * (k.samples > 1 && k.len_stride == a.H ? k.samples : 1); }

static obf_status_t check_attend_apart(const obf_attend_t* c, const AttendPlan& p, const float* lse, const bool lse_out, const float* mass, const void* ws) {
  const AttendArgs& a = p.a;
  const size_t es = c->dtype == OBF_BF16 ? 2 : 4, row = c->head_dim * es;
  const AttendKeys& own = a.keys[a.n_keys - 1];
  const AttendKeys& front = a.keys[0];
  const bool shared = a.n_keys > 1;
  const Region first = {"lse", lse, (size_t)a.rows * 4}, none = {"", nullptr, 0};
  const Region outs[] = {{"O", a.O, a.O ? region_rows(a, c->head_dim, a.os, a.oh, a.ot) * es : 0}, lse_out ? first : none,
                         {"mass", mass, region_cache(a, own) * 4}, {"the workspace", ws, p.total}};
  const Region ins[] = {{"Q", a.Q, region_rows(a, c->head_dim, a.qs, a.qh, a.qt) * es}, {"K", own.K, region_cache(a, own) * row},
                        {"V", own.V, region_cache(a, own) * row}, {"kv_len", own.len, region_lens(a, own) * 4},
                        {"sink_len", own.sink_len, region_lens(a, own) * 4}, lse_out ? none : first,
                        {"prefix_K", shared ? front.K : nullptr, region_cache(a, front) * row}, {"prefix_V", shared ? front.V : nullptr, region_cache(a, front) * row},
                        {"prefix_len", shared ? front.len : nullptr, region_lens(a, front) * 4}};
  return check_apart(outs, sizeof(outs) / sizeof(outs[0]), ins, sizeof(ins) / sizeof(ins[0]));
}

static obf_status_t run_attend(const obf_attend_t* c, const void* Q, const void* prefix_K, const void* prefix_V, const int32_t* prefix_len,
                               int32_t prefix_len_all, int32_t prefix_stride, const void* K, const void* V, const int32_t* kv_len,
                               const int32_t* sink_len, void* O, float* lse, float* mass, void* ws, size_t ws_bytes, hipStream_t st) {
  AttendPlan p = plan_attend(c, prefix_stride, mass != nullptr, sink_len != nullptr);
  OBF_TRY(check_attend_ws(p, ws, ws_bytes));
  AttendArgs& a = p.a;
  char* base = (char*)ws;
  a.Q = Q; a.O = O;
  a.part_O = (float*)(base + p.part_O);
  a.part_lse = (float*)(base + p.part_lse);
  AttendKeys& own = a.keys[a.n_keys - 1];
  own.K = K; own.V = V; own.len = kv_len; own.sink_len = sink_len;
  if (a.n_keys > 1) {
    AttendKeys& m = a.keys[0];
    m.K = prefix_K; m.V = prefix_V; m.len = prefix_len; m.len_all = prefix_len_all;
  }
  OBF_TRY(check_attend_apart(c, p, lse, true, mass, ws));
  if (mass && !lse) lse = (float*)(base + p.lse);
  a.lse = lse;
  if (mass && p.keep_logits) { a.logits = (float*)(base + p.logits); a.mass = mass; }
  OBF_TRY(launch_plan(p, c->head_dim, c->dtype, st));
  if (a.ranges > 1 || a.logits) OBF_TRY(launch_attend_join(a, c->head_dim, c->dtype, st));
  p.ms.mass = mass; p.ms.part = (float*)(base + p.mass);
  return mass && !a.logits ? launch_attend_mass(a, c->head_dim, c->dtype, lse, p.ms, st) : OBF_OK;
}

}  // namespace obf

using namespace obf;

extern "C" {

size_t obf_attend_workspace_bytes(const obf_attend_t* call, int32_t prefix_stride, int32_t with_mass) {
  if (check_attend(call) != OBF_OK) return 0;
  if (prefix_stride < 0 || prefix_stride > kAttendMaxStride) { set_error("attend: prefix_stride outside [0, %d]", kAttendMaxStride); return 0; }
  return plan_attend(call, prefix_stride, with_mass != 0, true).total;
}

obf_status_t obf_attend(const obf_attend_t* call, const void* Q, const void* K, const void* V, const int32_t* kv_len, const int32_t* sink_len,
                        void* O, float* lse, float* mass, void* ws, size_t ws_bytes, void* stream) {
  OBF_TRY(check_attend(call));
  OBF_TRY(check_aligned("Q", Q)); OBF_TRY(check_aligned("K", K)); OBF_TRY(check_aligned("V", V)); OBF_TRY(check_aligned("O", O));
  return run_attend(call, Q, nullptr, nullptr, nullptr, 0, 0, K, V, kv_len, sink_len, O, lse, mass, ws, ws_bytes, (hipStream_t)stream);
}

obf_status_t obf_attend_shared(const obf_attend_t* call, const void* Q, const void* prefix_K, const void* prefix_V, const int32_t* prefix_len,
                               int32_t prefix_len_all, int32_t prefix_stride, const void* K, const void* V, const int32_t* kv_len,
                               const int32_t* sink_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  OBF_TRY(check_attend(call));
  if (prefix_stride < 1 || prefix_len_all < 0 || prefix_len_all > prefix_stride) {
    set_error("attend: prefix_stride must be >= 1 and prefix_len_all lie in [0, prefix_stride]");
    return OBF_ERR_INVALID_ARG;
  }
  if (prefix_stride > kAttendMaxStride) { set_error("attend: prefix_stride above the supported %d", kAttendMaxStride); return OBF_ERR_UNSUPPORTED; }
  OBF_TRY(check_aligned("Q", Q)); OBF_TRY(check_aligned("prefix_K", prefix_K)); OBF_TRY(check_aligned("prefix_V", prefix_V));
  OBF_TRY(check_aligned("K", K)); OBF_TRY(check_aligned("V", V)); OBF_TRY(check_aligned("O", O));
  return run_attend(call, Q, prefix_K, prefix_V, prefix_len, prefix_len_all, prefix_stride, K, V, kv_len, sink_len, O, lse, nullptr, ws, ws_bytes,
                    (hipStream_t)stream);
}

obf_status_t obf_attend_mass(const obf_attend_t* call, const void* Q, const void* K, const float* lse, const int32_t* kv_len,
                             const int32_t* sink_len, float* mass, void* ws, size_t ws_bytes, void* stream) {
  OBF_TRY(check_attend(call));
  OBF_TRY(check_aligned("Q", Q)); OBF_TRY(check_aligned("K", K)); OBF_NONNULL(lse); OBF_NONNULL(mass);
  AttendPlan p = plan_attend(call, 0, true, sink_len != nullptr);
  OBF_TRY(check_attend_ws(p, ws, ws_bytes));
  p.a.Q = Q;
  p.a.keys[0].K = K; p.a.keys[0].len = kv_len; p.a.keys[0].sink_len = sink_len;
  OBF_TRY(check_attend_apart(call, p, lse, false, mass, ws));
  p.ms.mass = mass; p.ms.part = (float*)((char*)ws + p.mass);
  return launch_attend_mass(p.a, call->head_dim, call->dtype, lse, p.ms, (hipStream_t)stream);
}

obf_status_t obf_evict(int32_t n_heads, int32_t head_dim, int32_t dtype, const void* K, const void* V, const float* mass, const int32_t* pos,
                       const int32_t* kv_len, int32_t kv_len_all, int32_t in_stride, int32_t budget, int32_t recent, const int32_t* sink_len,
                       int32_t sink, void* K_out, void* V_out, float* mass_out, int32_t* pos_out, int32_t* idx, int32_t* len_out,
                       int32_t out_stride, void* stream) {
  if (n_heads < 1 || n_heads > 65535) { set_error("n_heads must lie in [1, 65535]"); return OBF_ERR_INVALID_ARG; }
  if (dtype != OBF_F32 && dtype != OBF_BF16) { set_error("unknown dtype %d", dtype); return OBF_ERR_INVALID_ARG; }
  if (head_dim != 64 && head_dim != 128) { set_error("head_dim %d unsupported (64 or 128)", head_dim); return OBF_ERR_UNSUPPORTED; }
  if (in_stride < 1 || out_stride < 1) { set_error("in_stride and out_stride must be >= 1"); return OBF_ERR_INVALID_ARG; }
  if (in_stride > kAttendMaxStride || out_stride > kAttendMaxStride) { set_error("in_stride or out_stride above the supported %d", kAttendMaxStride); return OBF_ERR_UNSUPPORTED; }
  if (kv_len_all < 0 || kv_len_all > in_stride) { set_error("kv_len_all outside [0, in_stride]"); return OBF_ERR_INVALID_ARG; }
  if (sink < 0 || recent < 0 || budget < 0) { set_error("budget, recent and sink must not be negative"); return OBF_ERR_INVALID_ARG; }
  if (recent > budget) { set_error("recent %d above budget %d", recent, budget); return OBF_ERR_INVALID_ARG; }
  const int64_t most = (int64_t)budget + (sink_len ? 0 : sink);
  if ((most < in_stride ? most : in_stride) > out_stride) { set_error("budget and sink exceed out_stride %d", out_stride); return OBF_ERR_INVALID_ARG; }
  OBF_TRY(check_aligned("K", K)); OBF_TRY(check_aligned("V", V)); OBF_TRY(check_aligned("K_out", K_out)); OBF_TRY(check_aligned("V_out", V_out));
  OBF_NONNULL(mass); OBF_NONNULL(mass_out); OBF_NONNULL(idx); OBF_NONNULL(len_out);
  if (!pos != !pos_out) { set_error("pos and pos_out come together"); return OBF_ERR_INVALID_ARG; }
  const size_t row = (size_t)head_dim * (dtype == OBF_BF16 ? 2 : 4);
  const size_t in = (size_t)n_heads * in_stride, out = (size_t)n_heads * out_stride;
  const size_t heads = (size_t)n_heads * 4;
  const Region outs[] = {{"K_out", K_out, out * row}, {"V_out", V_out, out * row}, {"mass_out", mass_out, out * 4}, {"pos_out", pos_out, out * 4}, {"idx", idx, out * 4},
                         {"len_out", len_out, heads}};
  const Region ins[] = {{"K", K, in * row}, {"V", V, in * row}, {"mass", mass, in * 4}, {"pos", pos, in * 4}, {"kv_len", kv_len, heads}, {"sink_len", sink_len, heads}};
  OBF_TRY(check_apart(outs, sizeof(outs) / sizeof(outs[0]), ins, sizeof(ins) / sizeof(ins[0])));
  EvictArgs a;
  a.K = K; a.V = V; a.mass = mass; a.pos = pos; a.len = kv_len; a.sink_len = sink_len;
  a.heads = n_heads; a.len_all = kv_len_all; a.in_stride = in_stride; a.budget = budget; a.recent = recent; a.sink = sink; a.out_stride = out_stride;
  a.row_vec = (int)(row / 16);
  a.K_out = K_out; a.V_out = V_out; a.mass_out = mass_out; a.pos_out = pos_out; a.idx = idx; a.len_out = len_out;
  return launch_evict(a, (hipStream_t)stream);
}

}  // extern "C"
