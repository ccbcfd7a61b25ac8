// Entry points around the compression in a model's layer: finch_rotate, finch_rope_frequencies,
// finch_quantize, finch_attend.  Argument checks, launch sizing, launches; no allocation and no
// synchronisation.
#include <algorithm>
#include <cmath>

#include "attend.h"
#include "attend_plan.h"
#include "context.h"

namespace {

using finch::aligned;
using finch::AttendLaunch;
using finch::AttendParams;
using finch::AttendPlan;
using finch::hip_fail;
using finch::overlaps;

// The context's device is current while one of these lives.
struct OnDevice {
  int before = -1;
  hipError_t e;
  explicit OnDevice(const finch_ctx* ctx) {
    e = hipGetDevice(&before);
    if (e == hipSuccess && before != ctx->device) {
      e = hipSetDevice(ctx->device);
    } else {
      before = -1;  // nothing to restore
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

finch_status done(finch_ctx* ctx, hipError_t e) {
  if (e == hipSuccess) return FINCH_OK;
  (void)hipGetLastError();
  return hip_fail(ctx, e);
}

int elem_bytes(const finch_ctx* ctx) { return ctx->cfg.dtype == FINCH_BF16 ? 2 : 4; }

// A stride between rows or heads: not negative, whole 16-byte pieces, and offsets of 2^24 of them fit 63 bits.
bool stride_ok(int64_t s, int bytes) { return s >= 0 && s < (int64_t{1} << 36) && s * bytes % 16 == 0; }

// Bytes from the first to behind the last element of n0 x n1 heads of d channels.
size_t extent(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t d, int bytes) {
  return n0 <= 0 || n1 <= 0 ? 0 : static_cast<size_t>((n0 - 1) * s0 + (n1 - 1) * s1 + d) * bytes;
}

// Whether n0 x n1 heads of d channels keep clear of each other: one stride steps over all of the other's.
bool apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t d) {
  if ((n0 > 1 && s0 < d) || (n1 > 1 && s1 < d)) return false;
  return n0 <= 1 || n1 <= 1 || s0 >= (n1 - 1) * s1 + d || s1 >= (n0 - 1) * s0 + d;
}

// Whether two sets of rows of d bytes, `row` apart, lie between each other's rows and touch none.
bool between_rows(const void* a, const void* b, int64_t n, int64_t row, int64_t d) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  if (n <= 1 || row <= 0) return false;
  const uintptr_t r = (x < y ? y - x : x - y) % static_cast<uintptr_t>(row);
  return r >= static_cast<uintptr_t>(d) && static_cast<uintptr_t>(row) - r >= static_cast<uintptr_t>(d);
}

constexpr int32_t kMostRows = 1 << 24;
constexpr int32_t kMostHeads = 1 << 12;

finch_status check_attention(const finch_ctx* ctx, const finch_attention& a) {
  const int e = elem_bytes(ctx), G = ctx->cfg.group_size;
  const int64_t d = ctx->cfg.head_dim;
  if (a.n_que < 0 || a.c < 0 || a.m < 0 || (a.causal != 0 && a.causal != 1)) return FINCH_ERR_INVALID_ARG;
  if (int64_t{a.c} + a.m > kMostRows || int64_t{a.n_que} * G > kMostRows) return FINCH_ERR_CAPACITY;
  if ((a.k_scale == nullptr) != (a.v_scale == nullptr)) return FINCH_ERR_INVALID_ARG;
  if (a.k_scale && ctx->cfg.dtype != FINCH_BF16) return FINCH_ERR_UNSUPPORTED;
  if (a.n_que == 0) return FINCH_OK;
  const int ce = a.k_scale ? 1 : e;
  if (!a.q || !a.out || !aligned(a.q, 16) || !aligned(a.out, 16) || !aligned(a.lse, 4) || !aligned(a.m_live, 4)) return FINCH_ERR_INVALID_ARG;
  if (!stride_ok(a.q_row, e) || !stride_ok(a.q_head, e) || !stride_ok(a.out_row, e) || !stride_ok(a.out_head, e)) return FINCH_ERR_INVALID_ARG;
  if (!apart(a.n_que, a.out_row, G, a.out_head, d)) return FINCH_ERR_INVALID_ARG;
  const size_t ob = extent(a.n_que, a.out_row, G, a.out_head, d, e);
  if (overlaps(a.out, ob, a.q, extent(a.n_que, a.q_row, G, a.q_head, d, e))) return FINCH_ERR_INVALID_ARG;
  if (a.c > 0) {
    if (!a.k_cache || !a.v_cache || !aligned(a.k_cache, 16) || !aligned(a.v_cache, 16) || !stride_ok(a.cache_row, ce)) return FINCH_ERR_INVALID_ARG;
    const size_t b = extent(a.c, a.cache_row, 1, 0, d, ce);
    if (overlaps(a.out, ob, a.k_cache, b) || overlaps(a.out, ob, a.v_cache, b)) return FINCH_ERR_INVALID_ARG;
  }
  if (a.m > 0) {
    if (!a.k_chunk || !a.v_chunk || !aligned(a.k_chunk, 16) || !aligned(a.v_chunk, 16) || !stride_ok(a.chunk_row, e)) return FINCH_ERR_INVALID_ARG;
    const size_t b = extent(a.m, a.chunk_row, 1, 0, d, e);
    if (overlaps(a.out, ob, a.k_chunk, b) || overlaps(a.out, ob, a.v_chunk, b)) return FINCH_ERR_INVALID_ARG;
  }
  return FINCH_OK;
}

finch_status plan_attention(const finch_ctx* ctx, const finch_attention* hd, int32_t n, AttendPlan& pl) {
  const bool bf16 = ctx->cfg.dtype == FINCH_BF16;
  const int G = ctx->cfg.group_size, d = ctx->cfg.head_dim, cu = ctx->n_cu > 0 ? ctx->n_cu : 256;
  for (int32_t i = 0; i < n; ++i) {
    const finch_status st = check_attention(ctx, hd[i]);
    if (st != FINCH_OK) return st;
    if (hd[i].k_scale) pl.eight = true;
    const int64_t rows = int64_t{hd[i].n_que} * G;
    if (rows > 0) (!bf16 ? pl.some : rows <= pl.few.rows_hi ? pl.few : rows <= pl.some.rows_hi ? pl.some : pl.many).add(hd[i], i, rows);
  }
  // What is little beside the problems of many rows, and no longer than their workgroups, goes along with them: a launch of its own would
  // take longer (five packed prompts on 32 heads, one of them of 58 rows: 114 us with one, 109 without).
  const auto little = [&](const AttendLaunch& l) { return pl.many.tiles > 0 && 8 * l.work <= pl.many.work && 8 * l.keys_max * cu <= pl.many.work; };
  if (pl.few.tiles + pl.some.tiles > 0 && little(pl.some)) {
    const int lo = little(pl.few) ? pl.few.rows_lo : pl.some.rows_lo;
    pl.many = AttendLaunch(finch::kTilesRows, finch::kTilesKeys, lo, INT32_MAX);
    for (int32_t i = 0; i < n; ++i)
      if (int64_t{hd[i].n_que} * G >= lo) pl.many.add(hd[i], i, int64_t{hd[i].n_que} * G);
    pl.some.tiles = 0;
    if (lo == pl.few.rows_lo) pl.few.tiles = 0;
  }
  finch_status st = pl.few.deal(false, cu, d, G, pl.bytes);
  if (st == FINCH_OK) st = pl.some.deal(false, cu, d, G, pl.bytes);
  if (st == FINCH_OK) st = pl.many.deal(true, cu, d, G, pl.bytes);
  return st;
}

finch_status check_rotation(const finch_ctx* ctx, const finch_rotary* how, const finch_rows* hd, int32_t n, int32_t& n_max) {
  if (!how) return FINCH_ERR_INVALID_ARG;
  const int e = elem_bytes(ctx), G = ctx->cfg.group_size;
  const int64_t d = ctx->cfg.head_dim;
  if (how->pairing != FINCH_ROPE_OFF && how->pairing != FINCH_ROPE_HALF && how->pairing != FINCH_ROPE_INTERLEAVED) return FINCH_ERR_INVALID_ARG;
  if (how->pairing != FINCH_ROPE_OFF) {
    if (how->dims < 16 || how->dims > d || how->dims % 16 != 0) return FINCH_ERR_UNSUPPORTED;
    if (!how->freq || !aligned(how->freq, 8) || !std::isfinite(how->gain)) return FINCH_ERR_INVALID_ARG;
  }
  if (!aligned(how->q_norm, 16) || !aligned(how->k_norm, 16)) return FINCH_ERR_INVALID_ARG;
  if ((how->q_norm || how->k_norm) && !(how->eps >= 0.f && std::isfinite(how->eps))) return FINCH_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i) {
    const finch_rows& r = hd[i];
    if (r.n < 0 || r.kv_heads < 1 || (r.slot && r.slots < 0)) return FINCH_ERR_INVALID_ARG;
    if (r.n > kMostRows || r.kv_heads > kMostHeads || (r.slot && r.slots > (1 << 30))) return FINCH_ERR_CAPACITY;
    if (r.n == 0) continue;
    if (!aligned(r.pos, 4) || !aligned(r.slot, 4)) return FINCH_ERR_INVALID_ARG;
    if (how->pairing != FINCH_ROPE_OFF && !r.pos && r.pos0 > INT32_MAX - (r.n - 1)) return FINCH_ERR_INVALID_ARG;
    const struct {
      const void *in, *out;
      int64_t row, head, out_row, out_head;
      int64_t heads;
      bool slots;
    } parts[3] = {{r.q, r.q_out, r.q_row, r.q_head, r.q_out_row, r.q_out_head, int64_t{r.kv_heads} * G, false},
                  {r.k, r.k_out, r.k_row, r.k_head, r.k_out_row, r.k_out_head, r.kv_heads, r.slot != nullptr},
                  {r.v, r.v_out, r.v_row, r.v_head, r.v_out_row, r.v_out_head, r.kv_heads, r.slot != nullptr}};
    for (const auto& p : parts) {
      if (!p.in) continue;
      if (!p.out || !aligned(p.in, 16) || !aligned(p.out, 16)) return FINCH_ERR_INVALID_ARG;
      if (!stride_ok(p.row, e) || !stride_ok(p.head, e) || !stride_ok(p.out_row, e) || !stride_ok(p.out_head, e)) return FINCH_ERR_INVALID_ARG;
      // (up to 2^30 slots: stride_ok has 2^24 rows in mind)
      if (p.slots && r.slots > 0 && p.out_row > (int64_t{1} << 60) / r.slots) return FINCH_ERR_CAPACITY;
      if (!apart(p.slots ? r.slots : r.n, p.out_row, p.heads, p.out_head, d)) return FINCH_ERR_INVALID_ARG;
    }
    if (r.n > n_max) n_max = r.n;
  }
  return FINCH_OK;
}

finch_status check_quantization(const finch_ctx* ctx, const finch_quantization* hd, int32_t n, int32_t& n_max) {
  const int e = elem_bytes(ctx);
  const int64_t d = ctx->cfg.head_dim;
  for (int32_t i = 0; i < n; ++i) {
    const finch_quantization& q = hd[i];
    if (q.n < 0 || q.reserved != 0) return FINCH_ERR_INVALID_ARG;
    if (q.n > kMostRows) return FINCH_ERR_CAPACITY;
    if (q.n == 0) continue;
    if (!q.k || !q.v || !q.k_out || !q.v_out || !q.k_scale || !q.v_scale) return FINCH_ERR_INVALID_ARG;
    if (!aligned(q.k, 16) || !aligned(q.v, 16) || !aligned(q.k_out, 16) || !aligned(q.v_out, 16)) return FINCH_ERR_INVALID_ARG;
    if (!stride_ok(q.in_row, e) || !stride_ok(q.out_row, 1) || !apart(q.n, q.out_row, 1, 0, d)) return FINCH_ERR_INVALID_ARG;
    const size_t ib = extent(q.n, q.in_row, 1, 0, d, e), ob = extent(q.n, q.out_row, 1, 0, d, 1);
    const size_t sb = static_cast<size_t>((q.n + ctx->scale_block - 1) / ctx->scale_block);
    const void* in[2] = {q.k, q.v};
    const void* out[4] = {q.k_out, q.v_out, q.k_scale, q.v_scale};
    const size_t len[4] = {ob, ob, sb, sb};
    for (int a = 0; a < 4; ++a)
      for (const void* s : in)
        if (overlaps(s, ib, out[a], len[a])) return FINCH_ERR_INVALID_ARG;
    for (int a = 0; a < 4; ++a)
      for (int b = a + 1; b < 4; ++b)
        if (overlaps(out[a], len[a], out[b], len[b]) && !(b == 1 && between_rows(q.k_out, q.v_out, q.n, q.out_row, d))) return FINCH_ERR_INVALID_ARG;
    if (q.n > n_max) n_max = q.n;
  }
  return FINCH_OK;
}

finch_status check_batch(const finch_ctx* ctx, const void* hd, const void* dd, int32_t n) {
  if (!ctx || n < 0) return FINCH_ERR_INVALID_ARG;
  if (n > 0 && (!hd || !dd || !aligned(dd, 8))) return FINCH_ERR_INVALID_ARG;
  return FINCH_OK;
}

}  // namespace

extern "C" {

finch_status finch_rope_frequencies(int32_t dims, double base, const finch_rope_scaling* scaling, double* freq, int32_t freq_len,
                                    float* gain) {
  if (dims < 2 || dims % 2 != 0 || !(base > 1.0 && base < 1e30) || !freq || freq_len < 0) return FINCH_ERR_INVALID_ARG;
  finch_rope_scaling s = {FINCH_SCALING_NONE, 0, 1.0, 0.0, 0.0, 0.0};
  if (scaling) s = *scaling;
  if (s.reserved != 0 || s.kind < FINCH_SCALING_NONE || s.kind > FINCH_SCALING_RAMP) return FINCH_ERR_INVALID_ARG;
  if (s.kind != FINCH_SCALING_NONE && !(s.factor >= 1.0 && s.factor < 1e30)) return FINCH_ERR_INVALID_ARG;
  const bool banded = s.kind == FINCH_SCALING_BANDED || s.kind == FINCH_SCALING_RAMP;
  if (banded && !(s.low > 0.0 && s.high > s.low && s.high < 1e30 && s.context > 0.0 && s.context < 1e30)) return FINCH_ERR_INVALID_ARG;
  if (freq_len < dims / 2) return FINCH_ERR_CAPACITY;
  const double two_pi = 6.283185307179586476925;
  double first = 0.0, last = 1.0;  // RAMP: channel pairs
  if (s.kind == FINCH_SCALING_RAMP) {
    const auto pair_of = [&](double turns) { return dims * std::log(s.context / (turns * two_pi)) / (2.0 * std::log(base)); };
    first = std::fmax(std::floor(pair_of(s.high)), 0.0);
    last = std::fmin(std::ceil(pair_of(s.low)), dims - 1.0);
    if (!(last > first)) last = first + 0.001;
  }
  for (int32_t u = 0; u < dims / 2; ++u) {
    const double f = std::pow(base, -2.0 * u / dims);
    double keep = 1.0;  // share of the unscaled frequency
    if (s.kind == FINCH_SCALING_LINEAR) keep = 0.0;
    if (s.kind == FINCH_SCALING_BANDED) keep = (s.context * f / two_pi - s.low) / (s.high - s.low);
    if (s.kind == FINCH_SCALING_RAMP) keep = 1.0 - (u - first) / (last - first);
    keep = std::fmin(std::fmax(keep, 0.0), 1.0);
    freq[u] = s.kind == FINCH_SCALING_NONE ? f : f * keep + f / s.factor * (1.0 - keep);
  }
  if (gain) *gain = s.kind == FINCH_SCALING_RAMP ? static_cast<float>(0.1 * std::log(s.factor) + 1.0) : 1.0f;
  return FINCH_OK;
}

finch_status finch_rotate(finch_ctx* ctx, const finch_rotary* how, const finch_rows* host_desc, const finch_rows* dev_desc,
                          int32_t n, void* stream) {
  finch_status st = check_batch(ctx, host_desc, dev_desc, n);
  if (st != FINCH_OK) return st;
  int32_t n_max = 0;
  if ((st = check_rotation(ctx, how, host_desc, n, n_max)) != FINCH_OK || n_max == 0) return st;
  const OnDevice on(ctx);
  if (on.e != hipSuccess) return done(ctx, on.e);
  return done(ctx, finch::launch_rotate(ctx->cfg.head_dim, ctx->cfg.dtype == FINCH_BF16, *how, dev_desc, n, ctx->cfg.group_size, n_max,
                                        static_cast<hipStream_t>(stream)));
}

finch_status finch_quantize(finch_ctx* ctx, const finch_quantization* host_desc, const finch_quantization* dev_desc, int32_t n,
                            void* stream) {
  finch_status st = check_batch(ctx, host_desc, dev_desc, n);
  if (st != FINCH_OK) return st;
  int32_t n_max = 0;
  if ((st = check_quantization(ctx, host_desc, n, n_max)) != FINCH_OK || n_max == 0) return st;
  const OnDevice on(ctx);
  if (on.e != hipSuccess) return done(ctx, on.e);
  return done(ctx, finch::launch_quantize(ctx->cfg.head_dim, ctx->cfg.dtype == FINCH_BF16, dev_desc, n, n_max, ctx->scale_block,
                                          static_cast<hipStream_t>(stream)));
}

finch_status finch_attend_workspace_size(const finch_ctx* ctx, const finch_attention* host_desc, int32_t n, size_t* bytes) {
  if (!ctx || !bytes || n < 0 || (n > 0 && !host_desc)) return FINCH_ERR_INVALID_ARG;
  AttendPlan pl(ctx->cfg.dtype == FINCH_BF16);
  const finch_status st = plan_attention(ctx, host_desc, n, pl);
  *bytes = st == FINCH_OK ? pl.bytes : 0;
  return st;
}

finch_status finch_attend(finch_ctx* ctx, const finch_attention* host_desc, const finch_attention* dev_desc, int32_t n, void* ws,
                          size_t ws_bytes, void* stream) {
  finch_status st = check_batch(ctx, host_desc, dev_desc, n);
  if (st != FINCH_OK) return st;
  AttendPlan pl(ctx->cfg.dtype == FINCH_BF16);
  if ((st = plan_attention(ctx, host_desc, n, pl)) != FINCH_OK) return st;
  if (pl.bytes > 0 && (!ws || !aligned(ws, 256) || ws_bytes < pl.bytes)) return FINCH_ERR_WORKSPACE;
  if (pl.few.tiles == 0 && pl.some.tiles == 0 && pl.many.tiles == 0) return FINCH_OK;
  const OnDevice on(ctx);
  if (on.e != hipSuccess) return done(ctx, on.e);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = ctx->cfg.dtype == FINCH_BF16;
  const int d = ctx->cfg.head_dim;
  hipError_t e = hipSuccess;
  for (const AttendLaunch* l : {&pl.many, &pl.some, &pl.few}) {
    if (l->tiles == 0) continue;
    AttendParams p;
    p.descs = dev_desc;
    p.group = ctx->cfg.group_size;
    l->table(p);
    p.block_shift = __builtin_ctz(static_cast<unsigned>(ctx->scale_block));
    p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(d)));
    p.part = reinterpret_cast<float*>(static_cast<char*>(ws) + l->off_o);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + l->off_ml);
    // (a graph outlives its context, and graphs may run side by side: what is captured joins by a launch of its own)
    const bool meets = l != &pl.many && l->slots > 0 && (l->most_splits < finch::kJoinApart || l->rows_max == 1) && !finch::being_captured(s);
    p.meet = meets ? ctx->attend_meet : nullptr;
    for (int64_t at = 0; at < l->workgroups && e == hipSuccess; at += finch::kLaunchGrid) {
      const int some = static_cast<int>(std::min<int64_t>(finch::kLaunchGrid, l->workgroups - at));
      p.base = static_cast<int32_t>(at);
      if (!bf16) {
        e = finch::launch_attend_rows_f32(d, p, some, s);
      } else if (l == &pl.few) {
        e = finch::launch_attend_rows16(d, pl.eight, p, some, s);
      } else {
        e = l == &pl.some ? finch::launch_attend_rows(d, pl.eight, p, some, s) : finch::launch_attend_tiles(d, pl.eight, p, some, s);
      }
    }
    if (e == hipSuccess && l->slots > 0 && !meets) {
      int problems = 0;
      const int tiles = l->join_table(p, problems);
      e = finch::launch_attend_join(d, bf16, l->tile_rows, l->tile_keys, l->rows_max, problems, tiles, p, s);
    }
    if (e != hipSuccess) break;
  }
  return done(ctx, e);
}

// (Not in finch.h: for tests without a GPU.)  The checks that the calls above make of their descriptors
// before they launch anything; call: 0 finch_rotate, 1 finch_quantize, 2 finch_attend.
finch_status finch_debug_layer_check(const finch_config* cfg, int32_t scale_block, int32_t call, const finch_rotary* how, const void* desc,
                                     int32_t n) {
  if (!cfg || n < 0 || (n > 0 && !desc)) return FINCH_ERR_INVALID_ARG;
  finch_ctx tmp = {};
  tmp.cfg = *cfg;
  tmp.scale_block = scale_block;
  int32_t n_max = 0;
  AttendPlan pl(cfg->dtype == FINCH_BF16);
  if (call == 0) return check_rotation(&tmp, how, static_cast<const finch_rows*>(desc), n, n_max);
  if (call == 1) return check_quantization(&tmp, static_cast<const finch_quantization*>(desc), n, n_max);
  return plan_attention(&tmp, static_cast<const finch_attention*>(desc), n, pl);
}

// (Likewise.)  How finch_attend launches a batch on a chip of `cu` compute units.  kernel: 0 few rows, 1 some (or fp32), 2 many.
// said: workgroups, tiles of keys of a split at most, most splits, slots of partial results, tiles of rows that are joined, bytes of
// workspace, fewest and most stacked rows of its problems.  pieces, or NULL: [workgroups][5], of each its problem, tile of rows, split, splits and its tile's first slot.
finch_status finch_debug_attend_plan(const finch_config* cfg, int32_t cu, const finch_attention* desc, int32_t n, int32_t kernel, int64_t* said,
                                     int32_t* pieces) {
  if (!cfg || n < 0 || (n > 0 && !desc) || kernel < 0 || kernel > 2 || !said) return FINCH_ERR_INVALID_ARG;
  finch_ctx tmp = {};
  tmp.cfg = *cfg;
  tmp.scale_block = 64;
  tmp.n_cu = cu;
  AttendPlan pl(cfg->dtype == FINCH_BF16);
  const finch_status st = plan_attention(&tmp, desc, n, pl);
  if (st != FINCH_OK) return st;
  const AttendLaunch& l = kernel == 0 ? pl.few : kernel == 1 ? pl.some : pl.many;
  AttendParams p;
  int problems = 0;
  const int64_t got[8] = {l.workgroups, l.span, l.most_splits, l.slots, l.join_table(p, problems), static_cast<int64_t>(pl.bytes), l.rows_lo, l.rows_hi};
  std::copy(got, got + 8, said);
  l.table(p);
  for (int64_t w = 0; pieces && w < l.workgroups; ++w) {
    const finch::AttendPiece x = finch::piece_of(p, static_cast<int>(w));
    const int32_t five[5] = {x.p, x.rt, x.split, x.splits, x.slot};
    std::copy(five, five + 5, pieces + 5 * w);
  }
  return FINCH_OK;
}

}  // extern "C"
