// Entry points of the operators of a cache held in codes: argument checks, workspace, launches.
#include "attend_check.hpp"
#include "attend_codes.hpp"

namespace obf {

static obf_status_t check_codes(const char* name, const obf_codes_t* c) {
  if (!c || !c->codes || !c->scale_f16 || !c->zero_f16) { set_error("%s: codes, scale and zero are needed", name); return OBF_ERR_INVALID_ARG; }
  if ((uintptr_t)c->codes & 15) { set_error("%s: codes must be 16-byte aligned", name); return OBF_ERR_INVALID_ARG; }
  if (((uintptr_t)c->scale_f16 | (uintptr_t)c->zero_f16) & 1) { set_error("%s: scale and zero must be 2-byte aligned", name); return OBF_ERR_INVALID_ARG; }
  return OBF_OK;
}

static obf_status_t check_bits(int32_t bits) {
  if (bits != 4 && bits != 8) { set_error("bits must be 4 or 8"); return OBF_ERR_INVALID_ARG; }
  return OBF_OK;
}

static obf_status_t check_rows(const obf_cache_rows_t* c) {
  if (!c) { set_error("cache rows: descriptor is NULL"); return OBF_ERR_INVALID_ARG; }
  if (c->n_samples < 1 || c->n_kv_heads < 1 || c->n_rows < 1 || c->token_stride < 1) {
    set_error("cache rows: n_samples, n_kv_heads, n_rows, token_stride must all be >= 1");
    return OBF_ERR_INVALID_ARG;
  }
  OBF_TRY(check_bits(c->bits));
  if (c->dtype != OBF_F32 && c->dtype != OBF_BF16) { set_error("cache rows: unknown dtype %d", c->dtype); return OBF_ERR_INVALID_ARG; }
  if (c->kv_len_all < 0 || c->kv_len_all > c->token_stride) { set_error("cache rows: kv_len_all outside [0, token_stride]"); return OBF_ERR_INVALID_ARG; }
  if (c->len_stride < 0 || (c->len_stride > 0 && c->len_stride < c->n_kv_heads)) { set_error("cache rows: len_stride below n_kv_heads"); return OBF_ERR_INVALID_ARG; }
  if (c->sample_stride < 0 || (c->sample_stride > 0 && c->sample_stride < (int64_t)c->n_kv_heads * c->token_stride)) {
    set_error("cache rows: sample_stride below n_kv_heads * token_stride");
    return OBF_ERR_INVALID_ARG;
  }
  const int unit = c->dtype == OBF_BF16 ? 8 : 4;
  for (int i = 0; i < 3; ++i)
    if (c->k_stride[i] < 0 || c->k_stride[i] % unit || c->v_stride[i] < 0 || c->v_stride[i] % unit) {
      set_error("cache rows: strides of K and V must be multiples of 16 bytes and not negative");
      return OBF_ERR_INVALID_ARG;
    }
  if (c->head_dim != 64 && c->head_dim != 128) { set_error("head_dim %d unsupported (64 or 128)", c->head_dim); return OBF_ERR_UNSUPPORTED; }
  if (c->token_stride > kAttendMaxStride || c->n_rows > kAttendMaxStride) {
    set_error("cache rows: token_stride or n_rows above the supported %d", kAttendMaxStride);
    return OBF_ERR_UNSUPPORTED;
  }
  if ((int64_t)c->n_samples * c->n_kv_heads > 65535) { set_error("cache rows: more than 65535 heads in one call"); return OBF_ERR_UNSUPPORTED; }
  if ((int64_t)c->n_samples * c->n_kv_heads * c->token_stride > ((int64_t)1 << 30) || (int64_t)c->n_samples * c->n_kv_heads * c->n_rows > ((int64_t)1 << 29)) {
    set_error("cache rows: more than 2^30 cache rows or 2^29 rows of K in one call");        // (the latter: a launch has less than 2^32 threads)
    return OBF_ERR_UNSUPPORTED;
  }
  return OBF_OK;
}

// Strides of a tensor of rows; all three 0: contiguous.
static void row_strides(const int64_t (&given)[3], const obf_cache_rows_t* c, long (&out)[3]) {
  const bool any = given[0] || given[1] || given[2];
  const long row = c->head_dim, head = row * c->n_rows;
  out[0] = any ? given[0] : head * c->n_kv_heads; out[1] = any ? given[1] : head; out[2] = any ? given[2] : row;
}

static CacheRowsArgs rows_args(const obf_cache_rows_t* c, const void* K, const void* V, const int32_t* kv_len, const int32_t* count, const obf_codes_t* kc,
                               const obf_codes_t* vc) {
  CacheRowsArgs a;
  a.x[0] = const_cast<void*>(K); a.x[1] = const_cast<void*>(V);
  row_strides(c->k_stride, c, a.stride[0]);
  row_strides(c->v_stride, c, a.stride[1]);
  a.rows[0] = {kc->codes, kc->scale_f16, kc->zero_f16};
  a.rows[1] = {vc->codes, vc->scale_f16, vc->zero_f16};
  a.len = kv_len; a.count = count;
  a.len_all = c->kv_len_all; a.len_stride = c->len_stride ? c->len_stride : c->n_kv_heads;
  a.S = c->n_samples; a.H = c->n_kv_heads; a.n_rows = c->n_rows; a.token_stride = c->token_stride;
  a.sample_rows = c->sample_stride ? c->sample_stride : (long)c->n_kv_heads * c->token_stride;
  return a;
}

// The six arrays of a cache, of `rows` rows that certainly belong to it.
static void code_regions(Region (&out)[6], const obf_codes_t* k, const obf_codes_t* v, const size_t rows, const size_t bytes) {
  out[0] = {"K's codes", k->codes, rows * bytes}; out[1] = {"K's scale", k->scale_f16, rows * 2}; out[2] = {"K's zero", k->zero_f16, rows * 2};
  out[3] = {"V's codes", v->codes, rows * bytes}; out[4] = {"V's scale", v->scale_f16, rows * 2}; out[5] = {"V's zero", v->zero_f16, rows * 2};
}

static obf_status_t check_rows_apart(const obf_cache_rows_t* c, const CacheRowsArgs& a, const obf_codes_t* kc, const obf_codes_t* vc, const bool write) {
  const size_t es = c->dtype == OBF_BF16 ? 2 : 4, one = (size_t)a.H * a.token_stride;
  const bool whole = a.S == 1 || (size_t)a.sample_rows == one, lens_whole = a.S == 1 || a.len_stride == a.H;
  Region codes[6];
  code_regions(codes, kc, vc, whole ? one * a.S : one, (size_t)c->head_dim * c->bits / 8);
  const auto rows = [&](const int i) { return region_rows(a.S, a.H, a.n_rows, c->head_dim, a.stride[i][0], a.stride[i][1], a.stride[i][2]) * es; };
  const size_t lens = (size_t)a.H * (lens_whole ? a.S : 1) * 4;
  const Region k = {"K", a.x[0], rows(0)}, v = {"V", a.x[1], rows(1)}, len = {"kv_len", a.len, lens},
               count = {write ? "n_new" : "idx", a.count, write ? lens : (size_t)a.S * a.H * a.n_rows * 4};
  if (write) {
    const Region ins[] = {k, v, len, count};
    return check_apart(codes, 6, ins, 4);
  }
  const Region outs[] = {k, v}, ins[] = {codes[0], codes[1], codes[2], codes[3], codes[4], codes[5], len, count};
  return check_apart(outs, 2, ins, 8);
}

struct AttendCodesPlan { AttendCodesArgs c; bool tile, rows; int waves; size_t part_O, part_lse, least, rows_k, rows_v, numbers, bad, total; };      // least: without the rows' numbers

// Ranges of a launch of the kernel of many rows: the least of an estimate, in us.  A workgroup takes its tiles of 64 rows and as long as two more to begin and end, alone on a
// compute unit `step` a tile, two in 1.5 times that, more one after another; a join 3 and the partial results' way to memory and back.  Of 190 shapes (8 to 128 heads of 700 to
// 12000 rows, of one length and ragged, 80 to 2000 query rows) it chooses launches that take 1.014 of the time of the best of up to 12 on average, 1.15 at worst
// (profiles/codes_launches.txt).  (As many ranges as give each compute unit two workgroups, none from one a unit on: 1.067 and 1.58; 8 x 8 heads of 4000 to 12000 rows of 64, 500
// query rows 236 - 161 us.)
static long tile_ranges(const long blocks, const long rows, const long out_rows, const int d) {
  const double step = d == 128 ? 1.42 : 1.06, join = 3.0, partial = out_rows * (double)d * 8 / 6e6;
  const long tiles = (rows + 63) / 64;
  long best = 1;
  double least = 0;
  for (long r = 1; r <= 64 && (r == 1 || rows >= 100 * r); r = r < 3 ? r + 1 : r % 3 ? r / 2 * 3 : r / 3 * 4) {        // 1 2 3 4 6 8 12 ...
    const double each = (double)(blocks * r) / kNumCU, load = each <= 1 ? 1.0 : each <= 2 ? 1.5 : 0.83 * (each + 0.3);
    const double us = load * ((tiles + r - 1) / r + 2) * step + (r > 1 ? join + r * partial : 0.0);
    if (r == 1 || us < least) { best = r; least = us; }
  }
  return best;
}

static AttendCodesPlan plan_attend_codes(const obf_attend_t* c, int bits, bool sinks_per_head) {
  AttendCodesPlan p;
  AttendArgs& a = p.c.a;
  a = attend_args(c);
  a.n_keys = 1;
  AttendKeys& k = a.keys[0];
  k = attend_own(c);
  const long own_rows = (long)a.T * a.g, d = c->head_dim;
  const bool few_seen = k.window > 0 && (k.sink > 0 || !sinks_per_head);
  const auto tiles_of = [&](const int tile_rows) { return (own_rows + tile_rows - 1) / tile_rows; };
  const auto seen_by = [&](const int tile_rows) { const long seen = (long)k.window + k.sink + tile_rows / a.g + 1; return few_seen && seen < k.stride ? seen : (long)k.stride; };
  // bf16 calls of more than 64 rows may take the kernel whose rows share the numbers that it makes of the codes; workgroups of 16 rows read the codes as often as they are,
  // and so are the faster ones for 64 rows at any length and for more where their tiles are not many times what the chip holds, the fewer the longer the caches are (us, many
  // rows and few: 16 x 8 heads of 8192 to 32768 rows, 40 query rows 297 - 187, of 2000 to 8192, 64 rows 93 - 69, 80 rows 93 - 97; 8 heads of 300 to 600 rows, 96 to 512 query
  // rows 14 to 20 - 7 to 9, 1000 rows 16.4 - 11.1; 16 heads of 300, 1000 rows (1008 tiles) 16.8 - 19.5; of 4000, 256 rows (256 tiles) 31.5 - 27.5, 64 heads 71 - 80; 8 heads
  // of 12000, 160 rows (80 tiles) 37.8 - 33.2, 256 rows 38.2 - 40.3).  Workgroups of 32 rows: 16 x 8 heads of 4000, 20 rows 33 for 30, 4 x 8 of 1000 15 for 13.
  const long few_tiles = tiles_of(kCodesFewRows) * a.S * a.H, few_rows = seen_by(kCodesFewRows);
  p.tile = c->dtype == OBF_BF16 && own_rows > kCodesManyRows && few_tiles > (few_rows <= 2560 ? 768 : few_rows <= 6144 ? 256 : 96);
  const int tile_rows = p.tile ? kAttendTileRows : kCodesFewRows;
  k.row_tiles = (int)tiles_of(tile_rows);
  const long blocks = (long)k.row_tiles * a.S * a.H, rows = seen_by(tile_rows);
  long ranges = 1;
  p.waves = 8;
  if (p.tile) {
    ranges = tile_ranges(blocks, rows, a.rows, (int)d);
  } else {
    // Few rows: how many ranges of how many waves was measured over 559 shapes (2 to 640 heads of 40 to 32000 rows, of one length and ragged, all types, 1 to 175 tiles of
    // query rows), each with up to 14 launches (profiles/codes_launches.txt); these rules take 1.012 of the best launch's time on average, 1.17 at worst.  us, otherwise and so:
    //   a join takes 3 us: none for short caches (8 heads of 600 rows 10.8 - 7.9, 64 of 1000 11.9 - 10.7);
    //   few sets: a wave with one or two tiles and a join of 16 ranges ends before long ranges do (8 heads of 1500 rows, four of eight waves 12.7 - 9.7);
    //   long caches: as many small workgroups as even out heads of different lengths (136 of 5000 to 20000 rows, 2 of eight waves and 8 of four 82.9 - 65; 72 of them,
    //   four of eight waves and 16 of four 45.2 - 35.8); 128 and 256 heads of one length lose by it (8 bits, 9000 rows: 59.9 - 61.4, 105.7 - 110);
    //   more than 32 ranges take longer to join than they save (8 heads of 32000 rows, 32, 64 and 128 ranges 19 - 24 - 32);
    //   four waves where eight would have nothing to do (8 heads of 256 rows 6.9 - 6.4, 512 of 100 9.2 - 7.6), and where registers leave room for 12 a compute unit and there
    //   is work for them (fp32, d 128, 24 heads of 400 rows, 1332 query rows 65.8 - 37.0).
    const bool wide = few_codes_per_cu(c->head_dim, c->dtype == OBF_F32, bits) == 2;
    if (rows > (wide && blocks > 32 ? 1536 : wide || blocks > 32 ? 1024 : 768)) {
      const long most = rows > 16384 ? 32 : 16, want = rows <= 4096 ? (blocks <= 32 ? 16 * blocks : kNumCU) : blocks <= 16 ? 512 : wide ? 1536 : 768;
      while (2 * ranges * blocks <= want && ranges < most) ranges *= 2;
    }
    const bool four = ranges > 1 ? (rows <= 4096 ? blocks <= 32 : blocks > 16) : rows <= 256 || (!wide && blocks >= 384);
    p.waves = four ? 4 : 8;
  }
  // At most 2^16 rows a range, where the partial results stay under 256 MB: a lane adds up a range's terms in single precision (2^24 rows of equal weights, 2^19 a range: lse
  // 7e-5 off).
  while (rows > ranges << 16 && 2 * ranges * a.rows * d * (long)sizeof(float) <= 1L << 28) ranges *= 2;
  k.nsplit = (int)ranges;
  k.split0 = 0;
  a.ranges = k.nsplit;
  k.blocks = (int)(blocks * k.nsplit);
  size_t at = 0;
  p.part_O = at;
  if (a.ranges > 1) at += (size_t)a.ranges * a.rows * d * sizeof(float);
  p.part_lse = at;
  if (a.ranges > 1) at += ((size_t)a.ranges * a.rows * sizeof(float) + 255) & ~(size_t)255;
  p.least = at ? at : 256;
  // Numbers made once for all workgroups of a head, where 16 or more of them read a row and the copies stay under 4 GiB (us, by every workgroup and once: 8 heads of 8000
  // rows, 4, 8, 16 and 32 tiles of query rows 49 - 58, 66 - 72, 108 - 108, 236 - 190; 8 x 8 heads of 4000, 8 and 16 tiles 189 - 200, 342 - 332).
  const long readers = k.window > 0 && k.window * (long)a.g / kAttendTileRows < k.row_tiles ? k.window * (long)a.g / kAttendTileRows + 1 : k.row_tiles;
  const size_t values = ((size_t)a.S * a.H * k.stride * d * sizeof(uint16_t) + 255) & ~(size_t)255;
  p.rows = p.tile && readers >= 16 && values <= (size_t)1 << 31;
  p.c.flags = (k.stride + kCodeFlagRows - 1) / kCodeFlagRows;
  p.rows_k = at;
  if (p.rows) at += values;
  p.rows_v = at;
  if (p.rows) at += values;
  p.numbers = at;
  if (p.rows) at += ((size_t)a.S * a.H * k.stride * sizeof(uint2) + 255) & ~(size_t)255;
  p.bad = at;
  if (p.rows) at += ((size_t)a.S * a.H * p.c.flags + 255) & ~(size_t)255;
  p.total = p.rows ? at : p.least;
  return p;
}

}  // namespace obf

using namespace obf;

extern "C" {

obf_status_t obf_cache_write(const obf_cache_rows_t* call, const void* K, const void* V, const int32_t* kv_len, const int32_t* n_new,
                             const obf_codes_t* K_cache, const obf_codes_t* V_cache, void* stream) {
  OBF_TRY(check_rows(call));
  OBF_TRY(check_aligned("K", K)); OBF_TRY(check_aligned("V", V));
  OBF_TRY(check_codes("K_cache", K_cache)); OBF_TRY(check_codes("V_cache", V_cache));
  const CacheRowsArgs a = rows_args(call, K, V, kv_len, n_new, K_cache, V_cache);
  OBF_TRY(check_rows_apart(call, a, K_cache, V_cache, true));
  return launch_cache_write(a, call->head_dim, call->dtype, call->bits, (hipStream_t)stream);
}

obf_status_t obf_cache_read(const obf_cache_rows_t* call, const obf_codes_t* K_cache, const obf_codes_t* V_cache, const int32_t* kv_len,
                            const int32_t* idx, void* K, void* V, void* stream) {
  OBF_TRY(check_rows(call));
  OBF_TRY(check_aligned("K", K)); OBF_TRY(check_aligned("V", V));
  OBF_TRY(check_codes("K_cache", K_cache)); OBF_TRY(check_codes("V_cache", V_cache));
  const CacheRowsArgs a = rows_args(call, K, V, kv_len, idx, K_cache, V_cache);
  for (int i = 0; i < 2; ++i) {
    const int64_t strides[3] = {a.stride[i][0], a.stride[i][1], a.stride[i][2]};
    if (rows_meet(strides, {a.S, a.H, a.n_rows}, call->head_dim)) { set_error("cache rows: rows of K and V must not overlap"); return OBF_ERR_INVALID_ARG; }
  }
  OBF_TRY(check_rows_apart(call, a, K_cache, V_cache, false));
  return launch_cache_read(a, call->head_dim, call->dtype, call->bits, (hipStream_t)stream);
}

size_t obf_attend_codes_workspace_bytes(const obf_attend_t* call, int32_t bits) {
  if (check_attend(call) != OBF_OK || check_bits(bits) != OBF_OK) return 0;
  const size_t with = plan_attend_codes(call, bits, true).total, without = plan_attend_codes(call, bits, false).total;
  return with > without ? with : without;
}

size_t obf_attend_codes_workspace_least(const obf_attend_t* call, int32_t bits) {
  if (check_attend(call) != OBF_OK || check_bits(bits) != OBF_OK) return 0;
  const size_t with = plan_attend_codes(call, bits, true).least, without = plan_attend_codes(call, bits, false).least;
  return with > without ? with : without;
}

obf_status_t obf_attend_codes(const obf_attend_t* call, int32_t bits, const void* Q, const obf_codes_t* K, const obf_codes_t* V, const int32_t* kv_len,
                              const int32_t* sink_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  OBF_TRY(check_attend(call));
  OBF_TRY(check_bits(bits));
  OBF_TRY(check_aligned("Q", Q)); OBF_TRY(check_aligned("O", O));
  OBF_TRY(check_codes("K", K)); OBF_TRY(check_codes("V", V));
  AttendCodesPlan p = plan_attend_codes(call, bits, sink_len != nullptr);
  if (ws_bytes < p.total) { p.rows = false; p.total = p.least; }
  OBF_TRY(check_attend_ws(p.total, ws, ws_bytes));
  AttendArgs& a = p.c.a;
  a.Q = Q; a.O = O; a.lse = lse;
  a.part_O = (float*)((char*)ws + p.part_O);
  a.part_lse = (float*)((char*)ws + p.part_lse);
  p.c.rows_k = p.rows ? (uint16_t*)((char*)ws + p.rows_k) : nullptr;
  p.c.rows_v = p.rows ? (uint16_t*)((char*)ws + p.rows_v) : nullptr;
  p.c.numbers = p.rows ? (uint2*)((char*)ws + p.numbers) : nullptr;
  p.c.bad = p.rows ? (uint8_t*)ws + p.bad : nullptr;
  AttendKeys& k = a.keys[0];
  k.len = kv_len; k.sink_len = sink_len;
  p.c.k = {K->codes, K->scale_f16, K->zero_f16};
  p.c.v = {V->codes, V->scale_f16, V->zero_f16};
  const size_t es = call->dtype == OBF_BF16 ? 2 : 4;
  const long hq = (long)a.H * a.g;
  Region codes[6];
  code_regions(codes, K, V, region_cache(a, k), (size_t)call->head_dim * bits / 8);
  const Region outs[] = {{"O", O, region_rows(a.S, hq, a.T, call->head_dim, a.os, a.oh, a.ot) * es}, {"lse", lse, (size_t)a.rows * 4}, {"the workspace", ws, p.total}};
  const Region ins[] = {{"Q", Q, region_rows(a.S, hq, a.T, call->head_dim, a.qs, a.qh, a.qt) * es}, codes[0], codes[1], codes[2], codes[3], codes[4], codes[5],
                        {"kv_len", kv_len, region_lens(a, k) * 4}, {"sink_len", sink_len, region_lens(a, k) * 4}};
  OBF_TRY(check_apart(outs, 3, ins, 9));
  const hipStream_t st = (hipStream_t)stream;
  if (p.tile) OBF_TRY(launch_attend_codes_tile(p.c, call->head_dim, bits, st));
  else OBF_TRY(launch_attend_codes_few(p.c, p.waves, call->head_dim, call->dtype, bits, st));
  return a.ranges > 1 ? launch_attend_join(a, call->head_dim, call->dtype, st) : OBF_OK;
}

}  // extern "C"
