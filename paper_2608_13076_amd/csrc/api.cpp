// C ABI of the speculative-verify library: argument checks, memory layout of
// the caller's buffers, and the launch sequence of one call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <vector>

#include "kvq.h"
#include "spade_internal.h"

using namespace spade;

namespace {

thread_local char g_err[512] = "";

spade_status fail(spade_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return s;
}

spade_status hipfail(hipError_t e, const char* what) {
  return fail(SPADE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Set the host bound of lens[b0..B) (and of the evicted positions) to the
// device values (synchronises).
spade_status refresh_bound(spade_kv kv, int b0, int B, hipStream_t st) {
  const size_t n = (size_t)(B - b0);
  std::vector<int32_t> h(n), ev(n, 0);
  hipError_t e = hipMemcpyAsync(h.data(), kv->lens + b0, n * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess && kv->evicted)
    e = hipMemcpyAsync(ev.data(), kv->evicted + b0, n * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return hipfail(e, "reading lens");
  for (size_t i = 0; i < n; ++i) {
    kv->lens_ub[b0 + i] = std::max(0, (int)h[i]);
    kv->evicted_ub[b0 + i] = ev[i];
  }
  return SPADE_OK;
}

// Whether `rows` more positions of request b fit the cache and the model's
// positions (evicted ones count), by the host bounds.
bool rows_fit(spade_kv kv, int b, int rows) {
  const int64_t end = (int64_t)kv->lens_ub[b] + rows;
  return end <= kv->max_len && end + kv->evicted_ub[b] <= kv->model->max_len;
}

bool capturing(hipStream_t st) {
  hipStreamCaptureStatus c;
  if (hipStreamIsCapturing(st, &c) == hipSuccess) return c != hipStreamCaptureStatusNone;
  (void)hipGetLastError();  // (the default stream beside a capture)
  return true;
}

// Whether rows(b) more positions of every request b0 <= b < B fit.  The host
// bound grows by gamma + 1 per commit (an eviction moves that on to the evicted
// positions) while the lengths grow by k + 1: where it does not allow the rows,
// the device's counts are read once before giving up (a capture cannot wait for
// them).
template <typename Rows>
spade_status make_fit(spade_kv kv, int b0, int B, Rows rows, hipStream_t st) {
  bool refreshed = false;
  for (int b = b0; b < B; ++b) {
    const int n = rows(b);
    if (!rows_fit(kv, b, n) && !refreshed && !capturing(st)) {
      const spade_status rs = refresh_bound(kv, b0, B, st);
      if (rs != SPADE_OK) return rs;
      refreshed = true;
    }
    if (rows_fit(kv, b, n)) continue;
    if ((int64_t)kv->lens_ub[b] + n > kv->max_len)
      return fail(SPADE_ECAPACITY, "request %d: %d cached + %d positions exceed max_len %d", b, kv->lens_ub[b], n, kv->max_len);
    return fail(SPADE_ECAPACITY, "request %d: %d cached, %d evicted + %d exceed the model's %d positions", b, kv->lens_ub[b],
                kv->evicted_ub[b], n, kv->model->max_len);
  }
  return SPADE_OK;
}

spade_status check_config(const spade_config* c) {
  if (!c) return fail(SPADE_EINVAL, "null config");
  if (c->n_layers < 1 || c->d_model < 1 || c->n_heads < 1 || c->head_dim < 1 || c->d_ffn < 1 || c->vocab < 2)
    return fail(SPADE_EINVAL, "config dimensions must be positive (vocab >= 2)");
  if (c->weight_dtype != SPADE_BF16 && c->weight_dtype != SPADE_F32)
    return fail(SPADE_EINVAL, "weight_dtype must be SPADE_BF16 or SPADE_F32");
  if (c->kv_dtype != SPADE_BF16 && c->kv_dtype != SPADE_F32 && c->kv_dtype != SPADE_I4)
    return fail(SPADE_EINVAL, "kv_dtype must be SPADE_BF16, SPADE_F32 or SPADE_I4");
  if (c->d_model != c->n_heads * c->head_dim) return fail(SPADE_EINVAL, "d_model != n_heads * head_dim");
  if (c->n_kv_heads < 0 || (c->n_kv_heads > 0 && c->n_heads % c->n_kv_heads != 0))
    return fail(SPADE_EINVAL, "n_kv_heads must be 0 or a divisor of n_heads");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(SPADE_EUNSUPPORTED, "head_dim must be 64 or 128");
  const int kb = kblock_of(c->weight_dtype);
  if (c->d_model % kb || c->d_ffn % kb)
    return fail(SPADE_EUNSUPPORTED, "d_model and d_ffn must be multiples of %d for this weight dtype", kb);
  if (!(c->rms_eps >= 0.f) || !(c->rope_theta > 0.f)) return fail(SPADE_EINVAL, "bad rms_eps / rope_theta");
  return SPADE_OK;
}

Dims dims_of(const spade_config* c) {
  Dims d{};
  d.L = c->n_layers;
  d.d = c->d_model;
  d.H = c->n_heads;
  d.hd = c->head_dim;
  d.KVH = c->n_kv_heads > 0 ? c->n_kv_heads : c->n_heads;
  d.dkv = d.KVH * c->head_dim;
  d.F = c->d_ffn;
  d.V = c->vocab;
  d.Vpad = (c->vocab + 15) / 16 * 16;
  d.wdt = c->weight_dtype;
  d.kvdt = c->kv_dtype;
  d.eps = c->rms_eps;
  d.theta = c->rope_theta;
  return d;
}

ArenaLayout layout_of(const Dims& D) {
  const size_t e = D.wdt == SPADE_BF16 ? 2 : 4;
  ArenaLayout a{};
  size_t off = 0;
  a.qkv = off;  off += align256((size_t)(D.d + 2 * D.dkv) * D.d * e);
  a.o = off;    off += align256((size_t)D.d * D.d * e);
  a.gu = off;   off += align256((size_t)2 * D.F * D.d * e);
  a.down = off; off += align256((size_t)D.d * D.F * e);
  a.g_attn = off; off += align256((size_t)D.d * 4);
  a.g_ffn = off;  off += align256((size_t)D.d * 4);
  a.layer_bytes = off;
  off = a.layer_bytes * D.L;
  a.embed = off;   off += align256((size_t)D.V * D.d * e);
  a.g_final = off; off += align256((size_t)D.d * 4);
  a.lm = off;      off += align256((size_t)D.Vpad * D.d * e);
  a.total = off;
  return a;
}

struct WsPlan {
  size_t x, act_n, act_o, act_f, ssq, q, attn_o, attn_ml, attn_cnt, logits, stats, rope, err, split_cnt,
      split_part, wide_cnt, wide_part, tile_part, corr_lse, corr_part, corr_cnt, prefill_tok, prefill_cnt, prefill_base,
      prefill_map, prefill_off, stage_k, stage_v, stage_lens, stage_rope, stage_rows, kvq_work, kvq_part_rows, kvq_ml,
      kvq_lse, total;
  size_t wide_items, wide_floats, tile_floats;
  int max_units;
  size_t act_split, actf_split;
  int Mmax, Mrows, NCmax, Rmax;
};

WsPlan plan_ws(const Dims& D, int max_batch, int max_gamma, int max_len) {
  WsPlan p{};
  p.Rmax = std::max(max_gamma + 1, kPrefillRows);
  // rows of a verify call, or of a batched prefill of 16 tokens per request
  p.Mmax = std::max(max_batch * (max_gamma + 1), max_batch * kPrefillRows);
  // rows of any forward: a bf16 cache with head_dim 128 also takes prefill
  // forwards of up to kPrefillMaxRows prompt rows (no more than the caches hold)
  p.Mrows = p.Mmax;
  if (D.kvdt == SPADE_BF16 && D.hd == kAttnHd)
    p.Mrows = std::max(p.Mmax, (int)std::min<long>(kPrefillMaxRows, (long)max_batch * ((max_len + 15) / 16 * 16)));
  p.NCmax = std::min(kAttnMaxChunks, (max_len + kAttnChunk - 1) / kAttnChunk);
  const bool wb = D.wdt == SPADE_BF16;
  const size_t ae = wb ? 2 * kActSplits : 4;  // bf16 terms or one float
  p.act_split = (size_t)p.Mrows * D.d;
  p.actf_split = (size_t)p.Mrows * D.F;
  const int NU = D.Vpad / 16;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += align256(bytes);
    return o;
  };
  p.x = take((size_t)p.Mrows * D.d * 4);
  p.act_n = take((size_t)p.Mrows * D.d * ae);
  p.act_o = take((size_t)p.Mrows * D.d * ae);
  p.act_f = take((size_t)p.Mrows * D.F * ae);
  p.ssq = take((size_t)p.Mrows * (D.d / 16) * 4);
  p.q = take((size_t)p.Mrows * D.d * 4);
  p.attn_o = take((size_t)max_batch * D.H * p.NCmax * p.Rmax * D.hd * 4);
  p.attn_ml = take((size_t)max_batch * D.H * p.NCmax * p.Rmax * 2 * 4);
  p.attn_cnt = take((size_t)max_batch * D.H * 4);
  p.logits = take((size_t)p.Mmax * D.V * 4);
  p.stats = take((size_t)p.Mmax * std::max(NU, kMaxStatGroups) * 3 * 4);  // NU = panels of the LM head
  p.rope = take((size_t)max_len * (D.hd / 2) * 2 * 4);
  p.err = take(4);
  p.max_units = std::max(std::max(D.d + 2 * D.dkv, 2 * D.F), D.Vpad) / 16;
  p.split_cnt = take((size_t)p.max_units * 4);
  p.split_part = take((size_t)p.max_units * 8 * 256 * 4);
  // k-split wide-row O and down projections (d / 16 panels, up to Mmax rows):
  // the most (unit group, row group) items and published floats any tiling
  // needs (17 to 32 rows by default; any where a setting keeps larger calls on
  // that engine, whose k-splits the tests force there)
  if (wb) {
    const int nu = D.d / 16;
    // unit groups of 8 panels (one per wave) x row groups of one 16-row tile
    p.wide_items = (size_t)((nu + 7) / 8) * (size_t)((p.Mmax + 15) / 16);
    for (int rt = 1; rt <= 3; ++rt)
      for (int pp = 1; pp <= 2; ++pp)
        if (!(pp == 2 && rt == 3)) p.wide_floats = std::max(p.wide_floats, wide_split_floats(nu, p.Mmax, rt, pp));
  }
  p.wide_cnt = take(p.wide_items * 4);
  p.wide_part = take(p.wide_floats * 4);
  // k-split launches of the tiled GEMM (forwards of more than 16 rows): the
  // widest projection of 144 rows, or a narrower one of more rows
  if (wb && p.Mrows > kWideMinRows)
    p.tile_floats = (size_t)((std::max(D.d + 2 * D.dkv, 2 * D.F) / 16 + 15) / 16) * tile_split_floats();
  p.tile_part = take(p.tile_floats * 4);
  p.corr_lse = take((size_t)max_batch * 4);
  p.corr_part = take((size_t)max_batch * kCorrPartFloats * 4);
  p.corr_cnt = take((size_t)max_batch * 4);
  p.prefill_tok = take((size_t)p.Mrows * 4);
  p.prefill_cnt = take((size_t)max_batch * 4);
  p.prefill_base = take((size_t)max_batch * 4);
  p.prefill_map = take((size_t)p.Mrows * 4);
  p.prefill_off = take((kPrefillPack + 1) * 4);
  if (D.kvdt == SPADE_I4) {
    const size_t rows = (size_t)max_batch * D.KVH * kVBlock * D.hd * 4;
    p.stage_k = take(rows);
    p.stage_v = take(rows);
    p.stage_lens = take((size_t)max_batch * 4);
    p.stage_rope = take((size_t)kMaxR * D.hd * 4);
    p.stage_rows = take((size_t)max_batch * 4);
    size_t ml, lse;
    const size_t o = kvq_attend_floats(max_batch, D.H, D.KVH, D.hd, p.Rmax, &ml, &lse);
    p.kvq_part_rows = o / D.hd;
    p.kvq_ml = align256(o * 4);
    p.kvq_lse = p.kvq_ml + align256(ml * 4);
    p.kvq_work = take(p.kvq_lse + lse * 4);
  }
  p.total = off;
  return p;
}

spade_status check_kvq(const spade_kvq_shape* s) {
  if (!s) return fail(SPADE_EINVAL, "null shape");
  if (s->n_layers < 1 || s->batch < 1 || s->n_kv_heads < 1 || s->n_heads < 1 || s->n_heads % s->n_kv_heads != 0)
    return fail(SPADE_EINVAL, "shape: layers, batch and heads must be positive, n_heads a multiple of n_kv_heads");
  if (s->head_dim != 64 && s->head_dim != 128) return fail(SPADE_EUNSUPPORTED, "head_dim must be 64 or 128");
  if (s->max_len < 1 || s->max_len > kKvqMaxLen) return fail(SPADE_ECAPACITY, "max_len must be in [1, %d]", kKvqMaxLen);
  // every count of heads fits 31 bits, also times the rows of an attention call
  if ((int64_t)s->n_layers * s->batch > 0x7fffffff / s->n_heads / kKvqMaxRows)
    return fail(SPADE_ECAPACITY, "too many layers, requests and heads");
  return SPADE_OK;
}

spade_status check_kvq_call(const spade_kvq_shape* s, int layer, int B, int dtype) {
  const spade_status r = check_kvq(s);
  if (r != SPADE_OK) return r;
  if (layer < 0 || layer >= s->n_layers) return fail(SPADE_EINVAL, "layer %d out of range", layer);
  if (B < 1 || B > s->batch) return fail(SPADE_ECAPACITY, "B=%d out of range", B);
  if (dtype != SPADE_F32 && dtype != SPADE_BF16) return fail(SPADE_EINVAL, "dtype must be SPADE_F32 or SPADE_BF16");
  return SPADE_OK;
}

// Rows of `heads` heads, ld elements apart: alignment of the vector accesses.
bool kvq_rows_ok(const void* p, int64_t ld, int64_t heads, int hd, int dtype) {
  return ((uintptr_t)p & (dtype == SPADE_F32 ? 15 : 7)) == 0 && ld >= heads * hd && ld % 4 == 0;
}
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
// Whether n rows of na bytes share one with n rows of nb bytes (sa, sb bytes
// from row to row; rows of equal distance may be interleaved).
bool rows_overlap(const void* a, int64_t na, int64_t sa, const void* b, int64_t nb, int64_t sb, int64_t n) {
  const __int128 a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  if (a0 >= b0 + (__int128)(n - 1) * sb + nb || b0 >= a0 + (__int128)(n - 1) * sa + na) return false;
  if (sa != sb || n == 1) return true;
  int64_t d = ((int64_t)((uintptr_t)b - (uintptr_t)a)) % sa;  // of b's row behind the one of a before it
  if (d < 0) d += sa;
  return d < na || sa - d < nb;
}

// the layers' heads of a model's 4-bit cache; the requests' evicted counts follow
size_t kvq_codes_bytes(const Dims& D, int max_batch, int max_len) {
  return align256((size_t)D.L * max_batch * D.KVH * kvq_head_bytes(max_len, D.hd));
}

size_t kvq_layer_bytes(const spade_kvq_shape* s) {
  return (size_t)s->batch * s->n_kv_heads * kvq_head_bytes(s->max_len, s->head_dim);
}

}  // namespace

extern "C" {

const char* spade_last_error(void) { return g_err; }

size_t spade_weight_bytes(const spade_config* cfg) {
  if (check_config(cfg) != SPADE_OK) return 0;
  return layout_of(dims_of(cfg)).total;
}

size_t spade_workspace_bytes(const spade_config* cfg, int max_batch, int max_gamma, int max_len) {
  if (check_config(cfg) != SPADE_OK || max_batch < 1 || max_gamma < 0 || max_gamma + 1 > kMaxR || max_len < 1)
    return 0;
  return plan_ws(dims_of(cfg), max_batch, max_gamma, max_len).total;
}

size_t spade_kv_bytes(const spade_config* cfg, int max_batch, int max_len) {
  if (check_config(cfg) != SPADE_OK || max_batch < 1 || max_len < 1) return 0;
  if (cfg->kv_dtype == SPADE_I4) return kvq_codes_bytes(dims_of(cfg), max_batch, max_len) + align256((size_t)max_batch * 4);
  const size_t e = cfg->kv_dtype == SPADE_BF16 ? 2 : 4;
  const int kvh = cfg->n_kv_heads > 0 ? cfg->n_kv_heads : cfg->n_heads;
  return 2 * align256((size_t)cfg->n_layers * max_batch * kvh * kv_stride_of(max_len) * cfg->head_dim * e);
}

spade_status spade_model_create(const spade_config* cfg, void* d_weights, void* d_workspace, int max_batch,
                                int max_gamma, int max_len, spade_model* out) {
  spade_status s = check_config(cfg);
  if (s != SPADE_OK) return s;
  if (!d_weights || !d_workspace || !out) return fail(SPADE_EINVAL, "null pointer");
  if (((uintptr_t)d_weights | (uintptr_t)d_workspace) & 255) return fail(SPADE_EINVAL, "buffers must be 256-byte aligned");
  if (max_batch < 1 || max_len < 2) return fail(SPADE_EINVAL, "max_batch >= 1 and max_len >= 2 required");
  if (max_len > kMaxLen) return fail(SPADE_ECAPACITY, "max_len must be <= %d", kMaxLen);
  if (max_gamma < 0 || max_gamma + 1 > kMaxR) return fail(SPADE_ECAPACITY, "max_gamma must be in [0, %d]", kMaxR - 1);
  if (cfg->kv_dtype == SPADE_I4 &&
      (size_t)max_batch * dims_of(cfg).KVH * kVBlock * cfg->head_dim * 4 > 0x7fffff00u)
    return fail(SPADE_ECAPACITY, "max_batch times K/V heads is too large for a 4-bit cache");
  spade_model m = new (std::nothrow) spade_model_s();
  if (!m) return fail(SPADE_EINVAL, "out of host memory");
  m->cfg = *cfg;
  m->dims = dims_of(cfg);
  m->lay = layout_of(m->dims);
  m->weights = (uint8_t*)d_weights;
  m->work = (uint8_t*)d_workspace;
  m->max_batch = max_batch;
  m->max_gamma = max_gamma;
  m->max_len = max_len;
  (void)hipGetDevice(&m->device);
  m->n_cu = 0;
  if (hipDeviceGetAttribute(&m->n_cu, hipDeviceAttributeMultiprocessorCount, m->device) != hipSuccess ||
      m->n_cu < 1)
    m->n_cu = 256;
  // one 8-wave GEMM workgroup per compute unit (the kernel needs two waves per
  // SIMD); SPADE_GEMM_WGS overrides for experiments
  m->gemm_wgs = m->n_cu;
  m->wide_rt = 0;
  m->wide_p = 0;
  m->wide_ks = 0;
  m->split_ks = 0;
  m->attn_merge = 0;
  m->corr_split = 0;
  m->attn_grouped = 0;
  m->prefill_rows = 0;
  m->big_gemm = 0;
  m->mid_gemm = 0;
  m->mid_ks = 0;
  m->tile_rt = 0;
  m->tile_p = 0;
  m->tile_ks = 0;
  if (const char* ev = std::getenv("SPADE_GEMM_WGS")) {
    const int v = std::atoi(ev);
    if (v > 0) m->gemm_wgs = std::min(v, kMaxStatGroups);
  }
  const WsPlan p = plan_ws(m->dims, max_batch, max_gamma, max_len);
  Workspace& w = m->ws;
  uint8_t* b = m->work;
  w.x = (float*)(b + p.x);
  w.act_n = b + p.act_n;
  w.act_o = b + p.act_o;
  w.act_f = b + p.act_f;
  w.ssq = (float*)(b + p.ssq);
  w.q = (float*)(b + p.q);
  w.attn_o = (float*)(b + p.attn_o);
  w.attn_ml = (float*)(b + p.attn_ml);
  w.attn_cnt = (uint32_t*)(b + p.attn_cnt);
  w.split_cnt = (uint32_t*)(b + p.split_cnt);
  w.split_part = (float*)(b + p.split_part);
  w.wide_cnt = (uint32_t*)(b + p.wide_cnt);
  w.wide_part = (float*)(b + p.wide_part);
  w.wide_items = p.wide_items;
  w.wide_floats = p.wide_floats;
  w.tile_floats = p.tile_floats;
  w.tile_part = (float*)(b + p.tile_part);
  w.corr_lse = (float*)(b + p.corr_lse);
  w.corr_part = (float*)(b + p.corr_part);
  w.corr_cnt = (uint32_t*)(b + p.corr_cnt);
  w.prefill_tok = (int32_t*)(b + p.prefill_tok);
  w.prefill_cnt = (int32_t*)(b + p.prefill_cnt);
  w.prefill_base = (int32_t*)(b + p.prefill_base);
  w.prefill_map = (int32_t*)(b + p.prefill_map);
  w.prefill_off = (int32_t*)(b + p.prefill_off);
  w.logits = (float*)(b + p.logits);
  w.stats = (float*)(b + p.stats);
  w.rope = (float*)(b + p.rope);
  w.err = (uint32_t*)(b + p.err);
  const bool quant = cfg->kv_dtype == SPADE_I4;
  if (quant) {
    w.stage_k = (float*)(b + p.stage_k);
    w.stage_v = (float*)(b + p.stage_v);
    w.stage_lens = (int32_t*)(b + p.stage_lens);
    w.stage_rope = (float*)(b + p.stage_rope);
    w.stage_rows = (int32_t*)(b + p.stage_rows);
    w.kvq_work = b + p.kvq_work;
    w.kvq_part_rows = p.kvq_part_rows;
    w.kvq_ml = p.kvq_ml;
    w.kvq_lse = p.kvq_lse;
  }
  w.act_split = p.act_split;
  w.actf_split = p.actf_split;
  w.Mmax = p.Mmax;
  w.Mrows = p.Mrows;
  w.NCmax = p.NCmax;
  w.Rmax = p.Rmax;

  // RoPE table: angle pos * theta^(-2i/hd) in double, stored as float.
  const int half = m->dims.hd / 2;
  std::vector<float> rope((size_t)max_len * half * 2);
  for (int pos = 0; pos < max_len; ++pos)
    for (int i = 0; i < half; ++i) {
      const double inv = std::pow((double)cfg->rope_theta, -2.0 * i / (double)m->dims.hd);
      const double ang = (double)pos * inv;
      rope[((size_t)pos * half + i) * 2] = (float)std::cos(ang);
      rope[((size_t)pos * half + i) * 2 + 1] = (float)std::sin(ang);
    }
  hipError_t e = hipMemcpy(w.rope, rope.data(), rope.size() * 4, hipMemcpyHostToDevice);
  if (e == hipSuccess) e = hipMemset(w.attn_cnt, 0, (size_t)max_batch * m->dims.H * 4);
  if (e == hipSuccess) e = hipMemset(w.split_cnt, 0, (size_t)p.max_units * 4);
  if (e == hipSuccess && p.wide_items > 0) e = hipMemset(w.wide_cnt, 0, p.wide_items * 4);
  if (e == hipSuccess) e = hipMemset(w.corr_cnt, 0, (size_t)max_batch * 4);
  if (e == hipSuccess) e = hipMemset(w.err, 0, 4);
  if (quant) {
    float none[kMaxR * 128];  // angles 0
    for (int i = 0; i < kMaxR * 128; i += 2) {
      none[i] = 1.f;
      none[i + 1] = 0.f;
    }
    if (e == hipSuccess) e = hipMemcpy(w.stage_rope, none, (size_t)kMaxR * half * 2 * 4, hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemset(w.stage_lens, 0, (size_t)max_batch * 4);
  }
  // activation buffers start at zero so rows past M never feed NaNs
  if (e == hipSuccess) e = hipMemset(b, 0, p.ssq);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    delete m;
    return hipfail(e, "model_create");
  }
  *out = m;
  return SPADE_OK;
}

void spade_model_destroy(spade_model m) { delete m; }

spade_status spade_model_load_tensor(spade_model m, int kind, int layer, const void* d_src, void* stream) {
  if (!m || !d_src) return fail(SPADE_EINVAL, "null pointer");
  if (kind < SPADE_WQ || kind > SPADE_LM_HEAD) return fail(SPADE_EINVAL, "bad tensor kind %d", kind);
  const bool global = kind == SPADE_EMBED || kind == SPADE_G_FINAL || kind == SPADE_LM_HEAD;
  if (!global && (layer < 0 || layer >= m->dims.L)) return fail(SPADE_EINVAL, "layer %d out of range", layer);
  hipError_t e = launch_pack(m, kind, global ? 0 : layer, d_src, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "load_tensor");
  return SPADE_OK;
}

spade_status spade_kv_create(spade_model m, void* d_kv, int max_batch, int max_len, int32_t* d_lens,
                             int32_t* d_pending, spade_kv* out) {
  if (!m || !d_kv || !d_lens || !d_pending || !out) return fail(SPADE_EINVAL, "null pointer");
  if ((uintptr_t)d_kv & 255) return fail(SPADE_EINVAL, "KV buffer must be 256-byte aligned");
  if (max_batch < 1 || max_batch > m->max_batch) return fail(SPADE_ECAPACITY, "kv max_batch exceeds the model's");
  if (max_len < 2 || max_len > m->max_len) return fail(SPADE_ECAPACITY, "kv max_len exceeds the model's");
  spade_kv kv = new (std::nothrow) spade_kv_s();
  if (!kv) return fail(SPADE_EINVAL, "out of host memory");
  kv->model = m;
  const bool quant = m->dims.kvdt == SPADE_I4;
  const size_t half = spade_kv_bytes(&m->cfg, max_batch, max_len) / 2;
  kv->k = (uint8_t*)d_kv;
  kv->v = quant ? nullptr : (uint8_t*)d_kv + half;
  kv->evicted = quant ? (int32_t*)((uint8_t*)d_kv + kvq_codes_bytes(m->dims, max_batch, max_len)) : nullptr;
  kv->evicted_ub = new (std::nothrow) int[max_batch]();
  kv->weights = nullptr;
  kv->evictions = kv->snap_evictions = 0;
  kv->lens = d_lens;
  kv->pending = d_pending;
  kv->max_batch = max_batch;
  kv->max_len = max_len;
  kv->stride = kv_stride_of(max_len);
  kv->lens_ub = new (std::nothrow) int[max_batch]();
  kv->last_rows = m->max_gamma + 1;
  kv->last_B = 0;
  kv->verified = false;
  kv->snap_ub = new (std::nothrow) int[max_batch]();
  if (!kv->lens_ub || !kv->snap_ub || !kv->evicted_ub) {
    spade_kv_destroy(kv);
    return fail(SPADE_EINVAL, "out of host memory");
  }
  if (quant) {
    hipError_t e = hipMemset(kv->evicted, 0, (size_t)max_batch * 4);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
      spade_kv_destroy(kv);
      return hipfail(e, "kv_create");
    }
  }
  *out = kv;
  return SPADE_OK;
}

void spade_kv_destroy(spade_kv kv) {
  if (!kv) return;
  delete[] kv->lens_ub;
  delete[] kv->snap_ub;
  delete[] kv->evicted_ub;
  delete kv;
}

spade_status spade_kv_set_state(spade_kv kv, int B, const int32_t* h_lens, const int32_t* h_pending, void* stream) {
  if (!kv || !h_lens || !h_pending) return fail(SPADE_EINVAL, "null pointer");
  if (B < 1 || B > kv->max_batch) return fail(SPADE_ECAPACITY, "B out of range");
  for (int b = 0; b < B; ++b) {
    if (h_lens[b] < 0 || h_lens[b] >= kv->max_len) return fail(SPADE_ECAPACITY, "lens[%d] out of range", b);
    if (h_pending[b] < 0 || h_pending[b] >= kv->model->dims.V) return fail(SPADE_EINVAL, "pending[%d] out of range", b);
  }
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipMemcpyAsync(kv->lens, h_lens, (size_t)B * 4, hipMemcpyHostToDevice, st);
  if (e == hipSuccess) e = hipMemcpyAsync(kv->pending, h_pending, (size_t)B * 4, hipMemcpyHostToDevice, st);
  if (e == hipSuccess && kv->evicted) e = launch_kvq_restart(B, kv->lens, kv->evicted, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return hipfail(e, "kv_set_state");
  for (int b = 0; b < B; ++b) {
    kv->lens_ub[b] = h_lens[b];
    if (h_lens[b] == 0 && kv->evicted_ub[b] > 0) {
      kv->evicted_ub[b] = 0;
      ++kv->evictions;  // a snapshot's rows counted them
    }
  }
  kv->verified = false;
  return SPADE_OK;
}

spade_status spade_kv_get_state(spade_kv kv, int B, int32_t* h_lens, int32_t* h_pending, void* stream) {
  if (!kv || !h_lens || !h_pending) return fail(SPADE_EINVAL, "null pointer");
  if (B < 1 || B > kv->max_batch) return fail(SPADE_ECAPACITY, "B out of range");
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipMemcpyAsync(h_lens, kv->lens, (size_t)B * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipMemcpyAsync(h_pending, kv->pending, (size_t)B * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess && kv->evicted)
    e = hipMemcpyAsync(kv->evicted_ub, kv->evicted, (size_t)B * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return hipfail(e, "kv_get_state");
  for (int b = 0; b < B; ++b) kv->lens_ub[b] = h_lens[b];
  return SPADE_OK;
}

spade_status spade_kv_snapshot(spade_kv kv, int B, int32_t* d_lens, int32_t* d_pending, void* stream) {
  if (!kv || !d_lens || !d_pending) return fail(SPADE_EINVAL, "null pointer");
  if (B < 1 || B > kv->max_batch) return fail(SPADE_ECAPACITY, "B out of range");
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = launch_copy_state(B, d_lens, d_pending, kv->lens, kv->pending, st);
  if (e != hipSuccess) return hipfail(e, "kv_snapshot");
  for (int b = 0; b < kv->max_batch; ++b) kv->snap_ub[b] = kv->lens_ub[b];
  kv->snap_evictions = kv->evictions;
  return SPADE_OK;
}

spade_status spade_kv_restore(spade_kv kv, int B, const int32_t* d_lens, const int32_t* d_pending, void* stream) {
  if (!kv || !d_lens || !d_pending) return fail(SPADE_EINVAL, "null pointer");
  if (B < 1 || B > kv->max_batch) return fail(SPADE_ECAPACITY, "B out of range");
  if (kv->evictions != kv->snap_evictions) return fail(SPADE_EINVAL, "positions were evicted since the snapshot");
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = launch_copy_state(B, kv->lens, kv->pending, d_lens, d_pending, st);
  if (e != hipSuccess) return hipfail(e, "kv_restore");
  for (int b = 0; b < B; ++b) kv->lens_ub[b] = kv->snap_ub[b];
  kv->verified = false;
  return SPADE_OK;
}

spade_status spade_prefill(spade_model m, spade_kv kv, int b, const int32_t* d_tokens, int n_tokens, void* stream) {
  if (!m || !kv || !d_tokens) return fail(SPADE_EINVAL, "null pointer");
  if (kv->model != m) return fail(SPADE_EINVAL, "kv belongs to another model");
  if (b < 0 || b >= kv->max_batch) return fail(SPADE_EINVAL, "request %d out of range", b);
  if (n_tokens < 1) return fail(SPADE_EINVAL, "n_tokens must be >= 1");
  const int n_cache = n_tokens - 1;
  const spade_status fit = make_fit(kv, b, b + 1, [&](int) { return n_tokens; }, (hipStream_t)stream);
  if (fit != SPADE_OK) return fit;
  hipError_t e = launch_prefill_one(m, kv, b, d_tokens, n_cache, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "prefill");
  kv->verified = false;
  return SPADE_OK;
}

spade_status spade_verify(spade_model m, spade_kv kv, int B, int gamma, const int32_t* d_draft_tokens,
                          const float* d_draft_probs, const float* d_uniforms, const uint8_t* d_mode,
                          float temperature, int32_t* d_n_accepted, int32_t* d_correction, float* d_logits,
                          void* stream) {
  if (!m || !kv || !d_mode || !d_n_accepted || !d_correction) return fail(SPADE_EINVAL, "null pointer");
  if (kv->model != m) return fail(SPADE_EINVAL, "kv belongs to another model");
  if (B < 1 || B > m->max_batch || B > kv->max_batch) return fail(SPADE_ECAPACITY, "B=%d out of range", B);
  if (gamma < 0 || gamma > m->max_gamma) return fail(SPADE_ECAPACITY, "gamma=%d out of range", gamma);
  if (gamma > 0 && !d_draft_tokens) return fail(SPADE_EINVAL, "draft tokens required when gamma > 0");
  if (d_draft_probs && !d_uniforms) return fail(SPADE_EINVAL, "sampling needs uniforms");
  if (!(temperature > 0.f && std::isfinite(temperature)))
    return fail(SPADE_EINVAL, "temperature must be finite and > 0");
  hipStream_t st = (hipStream_t)stream;
  const spade_status fit = make_fit(kv, 0, B, [&](int) { return gamma + 1; }, st);
  if (fit != SPADE_OK) return fit;
  kv->last_rows = gamma + 1;
  kv->last_B = B;
  kv->verified = true;
  ForwardCall fc{};
  fc.b0 = 0;
  fc.nb = B;
  fc.R = gamma + 1;
  fc.drafts = d_draft_tokens;
  fc.want_logits = true;
  fc.logits_out = d_logits ? d_logits : m->ws.logits;
  fc.mode = d_mode;
  fc.inv_T = 1.0f / temperature;
  fc.have_q = d_uniforms != nullptr && (d_draft_probs != nullptr || gamma == 0);
  AcceptCall ac{};
  ac.B = B;
  ac.gamma = gamma;
  ac.V = m->dims.V;
  ac.logits = fc.logits_out;
  ac.stats = m->ws.stats;
  ac.NU = std::min(m->dims.Vpad / 16, m->gemm_wgs);  // LM-head workgroups
  ac.panels = lm_stats_panels(m, B * (gamma + 1));
  ac.drafts = d_draft_tokens;
  ac.q = d_draft_probs;
  ac.u = d_uniforms;
  ac.mode = d_mode;
  ac.inv_T = fc.inv_T;
  ac.n_out = d_n_accepted;
  ac.corr_out = d_correction;
  hipError_t e = launch_forward(m, kv, fc, st);
  if (e == hipSuccess) e = launch_accept(m, ac, st);
  if (e != hipSuccess) return hipfail(e, "verify");
  return SPADE_OK;
}

spade_status spade_model_set_wide_tiles(spade_model m, int row_tiles, int panels) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (row_tiles < -1 || row_tiles > 3) return fail(SPADE_EINVAL, "row_tiles must be -1, 0, 1, 2 or 3");
  if (panels < 0 || panels > 2) return fail(SPADE_EINVAL, "panels must be 0, 1 or 2");
  m->wide_rt = row_tiles;
  m->wide_p = panels;
  return SPADE_OK;
}

spade_status spade_model_set_attn_merge(spade_model m, int mode) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (mode < 0 || mode > 2) return fail(SPADE_EINVAL, "mode must be 0, 1 or 2");
  m->attn_merge = mode;
  return SPADE_OK;
}

spade_status spade_model_set_attn_grouped(spade_model m, int mode) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (mode < 0 || mode > 1) return fail(SPADE_EINVAL, "mode must be 0 or 1");
  m->attn_grouped = mode;
  return SPADE_OK;
}

spade_status spade_model_set_prefill_rows(spade_model m, int rows) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (rows < 0) return fail(SPADE_EINVAL, "rows must be >= 0");
  m->prefill_rows = rows;
  return SPADE_OK;
}

spade_status spade_model_set_big_gemm(spade_model m, int mode) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (mode < 0 || mode > 2) return fail(SPADE_EINVAL, "mode must be 0, 1 or 2");
  m->big_gemm = mode;
  return SPADE_OK;
}

spade_status spade_model_set_mid_gemm(spade_model m, int mode, int k_splits) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (mode < 0 || mode > 2) return fail(SPADE_EINVAL, "mode must be 0, 1 or 2");
  if (k_splits < 0 || k_splits > 8) return fail(SPADE_EINVAL, "k_splits must be 0..8");
  m->mid_gemm = mode;
  m->mid_ks = k_splits;
  return SPADE_OK;
}

spade_status spade_model_set_tile_gemm(spade_model m, int row_tiles, int panels, int k_splits) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if ((row_tiles != 0 || panels != 0) && !tile_built(row_tiles, panels))
    return fail(SPADE_EINVAL, "no tile of %d row tiles and %d panels", row_tiles, panels);
  if (k_splits < 0 || k_splits > 8) return fail(SPADE_EINVAL, "k_splits must be 0..8");
  m->tile_rt = row_tiles;
  m->tile_p = panels;
  m->tile_ks = k_splits;
  return SPADE_OK;
}

spade_status spade_model_set_correction_slices(spade_model m, int mode) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (mode < 0 || mode > 2) return fail(SPADE_EINVAL, "mode must be 0, 1 or 2");
  m->corr_split = mode;
  return SPADE_OK;
}

spade_status spade_model_set_wide_k_splits(spade_model m, int splits) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (splits != 0 && splits != 1 && splits != 2 && splits != 4) return fail(SPADE_EINVAL, "splits must be 0, 1, 2 or 4");
  m->wide_ks = splits;
  return SPADE_OK;
}

spade_status spade_prefill_batch(spade_model m, spade_kv kv, int B, const int32_t* d_tokens, int ld,
                                 const int32_t* h_n_tokens, void* stream) {
  if (!m || !kv || !d_tokens || !h_n_tokens) return fail(SPADE_EINVAL, "null pointer");
  if (kv->model != m) return fail(SPADE_EINVAL, "kv belongs to another model");
  if (B < 1 || B > kv->max_batch || B > m->max_batch) return fail(SPADE_ECAPACITY, "B=%d out of range", B);
  std::vector<int> n_cache(B);
  for (int b = 0; b < B; ++b) {
    if (h_n_tokens[b] < 1 || h_n_tokens[b] > ld) return fail(SPADE_EINVAL, "request %d: n_tokens must be in [1, ld]", b);
    n_cache[b] = h_n_tokens[b] - 1;
  }
  const spade_status fit = make_fit(kv, 0, B, [&](int b) { return h_n_tokens[b]; }, (hipStream_t)stream);
  if (fit != SPADE_OK) return fit;
  hipError_t e = launch_prefill_batch(m, kv, B, d_tokens, ld, n_cache.data(), (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "prefill_batch");
  kv->verified = false;
  return SPADE_OK;
}

spade_status spade_softmax(const float* d_logits, int rows, int V, float temperature, float* d_probs,
                           void* stream) {
  if (!d_logits || !d_probs) return fail(SPADE_EINVAL, "null pointer");
  if (rows < 1 || V < 2) return fail(SPADE_EINVAL, "rows must be >= 1 and V >= 2");
  if (!(temperature > 0.f && std::isfinite(temperature)))
    return fail(SPADE_EINVAL, "temperature must be finite and > 0");
  hipError_t e = launch_softmax(d_logits, rows, V, 1.0f / temperature, d_probs, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "softmax");
  return SPADE_OK;
}

spade_status spade_model_set_split_k(spade_model m, int splits) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (splits != -1 && splits != 0 && splits != 2 && splits != 4) return fail(SPADE_EINVAL, "splits must be -1, 0, 2 or 4");
  m->split_ks = splits;
  return SPADE_OK;
}

spade_status spade_kv_commit(spade_kv kv, int B, const int32_t* d_n_accepted, const int32_t* d_correction,
                             void* stream) {
  if (!kv || !d_n_accepted || !d_correction) return fail(SPADE_EINVAL, "null pointer");
  if (!kv->verified) return fail(SPADE_EINVAL, "kv_commit needs a spade_verify on this cache since the last commit");
  if (B < 1 || B > kv->last_B) return fail(SPADE_EINVAL, "B=%d: the last spade_verify covered %d requests", B, kv->last_B);
  // the kernel clamps each k to [0, gamma] of that call, so the lengths grow
  // by at most gamma + 1
  hipError_t e = launch_commit(kv, B, kv->last_rows, d_n_accepted, d_correction, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "kv_commit");
  for (int b = 0; b < B; ++b) kv->lens_ub[b] += kv->last_rows;
  kv->verified = false;
  return SPADE_OK;
}

spade_status spade_accept_from_logits(spade_model m, int B, int gamma, int V, const float* d_logits,
                                      const int32_t* d_draft_tokens, const float* d_draft_probs,
                                      const float* d_uniforms, const uint8_t* d_mode, float temperature,
                                      int32_t* d_n_accepted, int32_t* d_correction, void* stream) {
  if (!m || !d_logits || !d_mode || !d_n_accepted || !d_correction) return fail(SPADE_EINVAL, "null pointer");
  if (B < 1 || B > m->max_batch) return fail(SPADE_ECAPACITY, "B out of range");
  if (gamma < 0 || gamma + 1 > kMaxR) return fail(SPADE_ECAPACITY, "gamma out of range");
  if (gamma > 0 && !d_draft_tokens) return fail(SPADE_EINVAL, "draft tokens required when gamma > 0");
  if (V < 2) return fail(SPADE_EINVAL, "V must be >= 2");
  if (d_draft_probs && !d_uniforms) return fail(SPADE_EINVAL, "sampling needs uniforms");
  if (!(temperature > 0.f && std::isfinite(temperature)))
    return fail(SPADE_EINVAL, "temperature must be finite and > 0");
  AcceptCall ac{};
  ac.B = B;
  ac.gamma = gamma;
  ac.V = V;
  ac.logits = d_logits;
  ac.stats = nullptr;
  ac.drafts = d_draft_tokens;
  ac.q = d_draft_probs;
  ac.u = d_uniforms;
  ac.mode = d_mode;
  ac.inv_T = 1.0f / temperature;
  ac.n_out = d_n_accepted;
  ac.corr_out = d_correction;
  hipError_t e = launch_accept(m, ac, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "accept_from_logits");
  return SPADE_OK;
}

spade_status spade_accept_from_logits_noalloc(int B, int gamma, int V, const float* d_logits,
                                              const int32_t* d_draft_tokens, const float* d_draft_probs,
                                              const float* d_uniforms, const uint8_t* d_mode, float temperature,
                                              int32_t* d_n_accepted, int32_t* d_correction, uint32_t* d_err,
                                              void* stream) {
  if (!d_logits || !d_mode || !d_n_accepted || !d_correction || !d_err) return fail(SPADE_EINVAL, "null pointer");
  if (B < 1 || B > kNoAllocMaxB)
    return fail(SPADE_ECAPACITY, "B=%d: the static scratch holds at most %d requests", B, kNoAllocMaxB);
  if (gamma < 0 || gamma + 1 > kMaxR) return fail(SPADE_ECAPACITY, "gamma out of range");
  if (gamma > 0 && !d_draft_tokens) return fail(SPADE_EINVAL, "draft tokens required when gamma > 0");
  if (V < 2) return fail(SPADE_EINVAL, "V must be >= 2");
  if (d_draft_probs && !d_uniforms) return fail(SPADE_EINVAL, "sampling needs uniforms");
  if (!(temperature > 0.f && std::isfinite(temperature)))
    return fail(SPADE_EINVAL, "temperature must be finite and > 0");
  AcceptCall ac{};
  ac.B = B;
  ac.gamma = gamma;
  ac.V = V;
  ac.logits = d_logits;
  ac.drafts = d_draft_tokens;
  ac.q = d_draft_probs;
  ac.u = d_uniforms;
  ac.mode = d_mode;
  ac.inv_T = 1.0f / temperature;
  ac.n_out = d_n_accepted;
  ac.corr_out = d_correction;
  hipError_t e = launch_accept_noalloc(ac, d_err, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "accept_from_logits_noalloc");
  return SPADE_OK;
}

spade_status spade_profile_gemm(spade_model m, spade_kv kv, int kind, int B, int gamma, int launches,
                                void* stream) {
  if (!m || !kv) return fail(SPADE_EINVAL, "null pointer");
  if (kv->model != m) return fail(SPADE_EINVAL, "kv belongs to another model");
  if (kind < GEMM_QKV || kind > GEMM_LM) return fail(SPADE_EINVAL, "bad GEMM kind %d", kind);
  if (B < 1 || B > m->max_batch || B > kv->max_batch) return fail(SPADE_ECAPACITY, "B out of range");
  if (gamma < 0 || gamma > m->max_gamma) return fail(SPADE_ECAPACITY, "gamma out of range");
  if (launches < 1) return fail(SPADE_EINVAL, "launches must be >= 1");
  for (int b = 0; b < B; ++b)
    if (kv->lens_ub[b] + gamma + 1 > kv->max_len) return fail(SPADE_ECAPACITY, "KV capacity");
  const int R = gamma + 1;
  for (int i = 0; i < launches; ++i) {
    ForwardCall fc{};
    fc.b0 = 0;
    fc.nb = B;
    fc.R = R;
    fc.logits_out = m->ws.logits;
    fc.inv_T = 1.0f;
    hipError_t e = launch_layer_gemm(m, kv, kind, i % m->dims.L, fc, (hipStream_t)stream);
    if (e != hipSuccess) return hipfail(e, "profile_gemm");
  }
  return SPADE_OK;
}

spade_status spade_wide_tiling(int kind, int rows, int n_units, int k, int n_cu, int* row_tiles, int* panels,
                               int* k_splits) {
  if (!row_tiles || !panels || !k_splits) return fail(SPADE_EINVAL, "null pointer");
  if (kind < GEMM_QKV || kind > GEMM_LM || rows <= kWideMinRows || n_units < 1 || k < 256 || k % 256 != 0 ||
      n_cu < 1)
    return fail(SPADE_EINVAL, "shape out of range");
  const WideChoice c = wide_choice(kind, rows, n_units, k / 256, k, n_cu, 0, 0, 0, (size_t)-1, (size_t)-1);
  *row_tiles = c.rt;
  *panels = c.p;
  *k_splits = c.ks;
  return SPADE_OK;
}

spade_status spade_model_gemm_engine(spade_model m, int kind, int rows, int* engine) {
  if (!m || !engine) return fail(SPADE_EINVAL, "null pointer");
  if (kind < GEMM_QKV || kind > GEMM_LM || rows < 1) return fail(SPADE_EINVAL, "shape out of range");
  *engine = gemm_engine(m, kind, rows);
  return SPADE_OK;
}

spade_status spade_tile_tiling(int kind, int rows, int n_units, int k, int n_cu, int* row_tiles, int* panels,
                               int* k_splits) {
  if (!row_tiles || !panels || !k_splits) return fail(SPADE_EINVAL, "null pointer");
  if (kind < GEMM_QKV || kind > GEMM_LM || rows <= kWideMinRows || n_units < 1 || k < 256 || k % 256 != 0 ||
      n_cu < 1)
    return fail(SPADE_EINVAL, "shape out of range");
  const TileChoice c = tile_choice(kind, rows, n_units, k / 256, n_cu, 0, 0, 0, (size_t)-1);
  *row_tiles = c.rt;
  *panels = c.p;
  *k_splits = c.ks;
  return SPADE_OK;
}

spade_status spade_model_set_head_norms(spade_model m, const float* d_gain_q, const float* d_gain_k, float eps) {
  if (!m) return fail(SPADE_EINVAL, "null model");
  if (m->dims.kvdt != SPADE_I4) return fail(SPADE_EUNSUPPORTED, "head norms need a 4-bit cache");
  if (!d_gain_q != !d_gain_k) return fail(SPADE_EINVAL, "both gains or none");
  if (!aligned16(d_gain_q) || !aligned16(d_gain_k)) return fail(SPADE_EINVAL, "gains must be 16-byte aligned");
  if (!(eps >= 0.f && std::isfinite(eps))) return fail(SPADE_EINVAL, "eps must be finite and >= 0");
  m->gain_q = d_gain_q;
  m->gain_k = d_gain_k;
  m->head_eps = eps;
  return SPADE_OK;
}

spade_status spade_kv_track_weights(spade_kv kv, float* d_weights) {
  if (!kv) return fail(SPADE_EINVAL, "null cache");
  if (!kv->evicted) return fail(SPADE_EUNSUPPORTED, "running weights need a 4-bit cache");
  kv->weights = d_weights;
  return SPADE_OK;
}

spade_status spade_kv_evict(spade_kv kv, int B, int budget, int recent, int32_t* d_kept, void* stream) {
  if (!kv || !d_kept) return fail(SPADE_EINVAL, "null pointer");
  if (!kv->evicted) return fail(SPADE_EUNSUPPORTED, "eviction needs a 4-bit cache");
  if (!kv->weights) return fail(SPADE_EINVAL, "eviction needs running weights (spade_kv_track_weights)");
  if (B < 1 || B > kv->max_batch) return fail(SPADE_ECAPACITY, "B out of range");
  if (budget < 1 || budget > kv->max_len) return fail(SPADE_ECAPACITY, "budget must be in [1, max_len]");
  if (recent < 0 || recent > budget) return fail(SPADE_EINVAL, "recent must be in [0, budget]");
  const Dims& D = kv->model->dims;
  KvqEvict a{};
  a.cache = kv->k;
  a.out = kv->k;
  a.head_bytes = a.out_head_bytes = kvq_head_bytes(kv->max_len, D.hd);
  a.L = D.L;
  a.batch = a.out_batch = kv->max_batch;
  a.B = B;
  a.KVH = D.KVH;
  a.hd = D.hd;
  a.max_len = a.out_max_len = kv->max_len;
  a.budget = budget;
  a.recent = recent;
  a.w = kv->weights;
  a.w_out = kv->weights;
  a.lens = kv->lens;
  a.lens_out = kv->lens;
  a.kept = d_kept;
  a.evicted = kv->evicted;
  const hipError_t e = launch_kvq_evict(a, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "kv_evict");
  for (int b = 0; b < B; ++b) {
    kv->evicted_ub[b] += std::max(0, kv->lens_ub[b] - budget);
    kv->lens_ub[b] = std::min(kv->lens_ub[b], budget);
  }
  kv->verified = false;
  ++kv->evictions;
  return SPADE_OK;
}

size_t spade_kvq_bytes(const spade_kvq_shape* s) {
  if (check_kvq(s) != SPADE_OK) return 0;
  return align256(s->n_layers * kvq_layer_bytes(s));
}

size_t spade_kvq_workspace_bytes(const spade_kvq_shape* s, int max_rows) {
  if (check_kvq(s) != SPADE_OK) return 0;
  if (max_rows < 1 || max_rows > kKvqMaxRows) {
    fail(SPADE_ECAPACITY, "max_rows must be in [1, %d]", kKvqMaxRows);
    return 0;
  }
  size_t ml, lse;
  const size_t o = kvq_attend_floats(s->batch, s->n_heads, s->n_kv_heads, s->head_dim, max_rows, &ml, &lse);
  return align256(o * 4) + align256(ml * 4) + align256(lse * 4);
}

spade_status spade_kvq_append(const spade_kvq_shape* s, int layer, void* d_cache, int B, int R, int dtype,
                              const void* d_q, int64_t q_ld, const void* d_k, int64_t k_ld, const void* d_v,
                              int64_t v_ld, const float* d_gain_q, const float* d_gain_k, float eps,
                              const float* d_rope, int rope_len, const int32_t* d_pos, const int32_t* d_lens,
                              const int32_t* d_rows, void* d_q_out, int64_t q_out_ld, float* d_weights,
                              uint32_t* d_err, void* stream) {
  const spade_status r = check_kvq_call(s, layer, B, dtype);
  if (r != SPADE_OK) return r;
  if (!d_cache || !d_k || !d_v || !d_lens || (d_q && !d_q_out)) return fail(SPADE_EINVAL, "null pointer");
  if (R < 1) return fail(SPADE_EINVAL, "R must be >= 1");
  const int hd = s->head_dim;
  if (!kvq_rows_ok(d_k, k_ld, s->n_kv_heads, hd, dtype) || !kvq_rows_ok(d_v, v_ld, s->n_kv_heads, hd, dtype) ||
      (d_q && (!kvq_rows_ok(d_q, q_ld, s->n_heads, hd, dtype) || !kvq_rows_ok(d_q_out, q_out_ld, s->n_heads, hd, dtype))))
    return fail(SPADE_EINVAL, "rows: alignment or leading dimension");
  if ((uintptr_t)d_cache & 255) return fail(SPADE_EINVAL, "the cache must be 256-byte aligned");
  if (!aligned16(d_gain_q) || !aligned16(d_gain_k) || !aligned16(d_rope))
    return fail(SPADE_EINVAL, "gains and rope must be 16-byte aligned");
  if (!(eps >= 0.f && std::isfinite(eps))) return fail(SPADE_EINVAL, "eps must be finite and >= 0");
  if (d_rope && rope_len < 1) return fail(SPADE_EINVAL, "rope_len must be >= 1");
  if ((int64_t)B * R > (int64_t)0x7fffffff / (s->n_heads + 2 * s->n_kv_heads))
    return fail(SPADE_ECAPACITY, "too many rows");
  if (d_q) {
    const int64_t e = dtype == SPADE_F32 ? 4 : 2, n = (int64_t)B * R, nq = s->n_heads * hd * e, nk = s->n_kv_heads * hd * e;
    const bool in_place = d_q_out == d_q && (q_out_ld == q_ld || n == 1);
    if ((!in_place && rows_overlap(d_q_out, nq, q_out_ld * e, d_q, nq, q_ld * e, n)) ||
        rows_overlap(d_q_out, nq, q_out_ld * e, d_k, nk, k_ld * e, n) ||
        rows_overlap(d_q_out, nq, q_out_ld * e, d_v, nk, v_ld * e, n))
      return fail(SPADE_EINVAL, "q_out overlaps other rows than q's own");
  }
  KvqAppend a{};
  a.cache = (uint8_t*)d_cache + layer * kvq_layer_bytes(s);
  a.head_bytes = kvq_head_bytes(s->max_len, hd);
  a.B = B;
  a.R = R;
  a.H = s->n_heads;
  a.KVH = s->n_kv_heads;
  a.hd = hd;
  a.max_len = s->max_len;
  a.q = KvqRows{d_q, R * q_ld, q_ld, hd};
  a.k = KvqRows{d_k, R * k_ld, k_ld, hd};
  a.v = KvqRows{d_v, R * v_ld, v_ld, hd};
  a.v_feature = 1;
  a.bf16 = dtype == SPADE_BF16;
  a.gain_q = d_gain_q;
  a.gain_k = d_gain_k;
  a.eps = eps;
  a.rope = d_rope;
  a.rope_len = rope_len;
  a.pos = d_pos;
  a.lens = d_lens;
  a.rows = d_rows;
  a.q_out = d_q_out;
  a.qo_ld = q_out_ld;
  a.weights = d_weights;
  a.err = d_err;
  const hipError_t e = launch_kvq_append(a, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "kvq_append");
  return SPADE_OK;
}

spade_status spade_kvq_read(const spade_kvq_shape* s, int layer, const void* d_cache, int B, int R,
                            const int32_t* d_start, const int32_t* d_rows, int dtype, void* d_k, void* d_v,
                            void* stream) {
  const spade_status r = check_kvq_call(s, layer, B, dtype);
  if (r != SPADE_OK) return r;
  if (!d_cache || !d_k || !d_v) return fail(SPADE_EINVAL, "null pointer");
  if (R < 1) return fail(SPADE_EINVAL, "R must be >= 1");
  if ((uintptr_t)d_cache & 255) return fail(SPADE_EINVAL, "the cache must be 256-byte aligned");
  if (!aligned16(d_k) || !aligned16(d_v)) return fail(SPADE_EINVAL, "outputs must be 16-byte aligned");
  if ((int64_t)B * R > (int64_t)0x7fffffff / s->n_kv_heads) return fail(SPADE_ECAPACITY, "too many rows");
  KvqRead a{};
  a.cache = (const uint8_t*)d_cache + layer * kvq_layer_bytes(s);
  a.head_bytes = kvq_head_bytes(s->max_len, s->head_dim);
  a.B = B;
  a.R = R;
  a.KVH = s->n_kv_heads;
  a.hd = s->head_dim;
  a.max_len = s->max_len;
  a.bf16 = dtype == SPADE_BF16;
  a.start = d_start;
  a.rows = d_rows;
  a.k = d_k;
  a.v = d_v;
  const hipError_t e = launch_kvq_read(a, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "kvq_read");
  return SPADE_OK;
}

spade_status spade_kvq_attend(const spade_kvq_shape* s, int layer, const void* d_cache, int B, int R, int dtype,
                              const void* d_q, int64_t q_ld, float scale, const int32_t* d_lens,
                              const int32_t* d_rows, int max_keys, void* d_out, int64_t out_ld,
                              const float* d_weights_in, float* d_weights_out, int weight_rows, void* d_workspace,
                              size_t workspace_bytes, uint32_t* d_err, void* stream) {
  const spade_status r = check_kvq_call(s, layer, B, dtype);
  if (r != SPADE_OK) return r;
  if (!d_cache || !d_q || !d_out || !d_lens || !d_workspace) return fail(SPADE_EINVAL, "null pointer");
  if (R < 1 || R > kKvqMaxRows) return fail(SPADE_ECAPACITY, "R must be in [1, %d]", kKvqMaxRows);
  const int hd = s->head_dim;
  if (!kvq_rows_ok(d_q, q_ld, s->n_heads, hd, dtype) || !kvq_rows_ok(d_out, out_ld, s->n_heads, hd, dtype))
    return fail(SPADE_EINVAL, "rows: alignment or leading dimension");
  if (((uintptr_t)d_cache | (uintptr_t)d_workspace) & 255)
    return fail(SPADE_EINVAL, "cache and workspace must be 256-byte aligned");
  if (!(scale > 0.f && scale <= 0x1p50f)) return fail(SPADE_EINVAL, "scale must be in (0, 2^50]");
  if (max_keys == 0) max_keys = s->max_len;
  // (a ragged batch of short contexts has a bound below its padded rows)
  const int least = d_rows ? 1 : R;
  if (max_keys < least || max_keys > s->max_len)
    return fail(SPADE_ECAPACITY, "max_keys %d must be in [%d, %d]", max_keys, least, s->max_len);
  if (d_weights_out && (weight_rows < 0 || weight_rows > R)) return fail(SPADE_EINVAL, "weight_rows must be in [0, R]");
  if (d_weights_in && !d_weights_out) return fail(SPADE_EINVAL, "weights_in without weights_out");
  const size_t wb = (size_t)s->batch * s->n_kv_heads * s->max_len * 4;
  if (d_weights_in && d_weights_in != d_weights_out && overlap(d_weights_in, wb, d_weights_out, wb))
    return fail(SPADE_EINVAL, "weights_in and weights_out overlap");
  // the part of the layout that B requests of R rows use
  size_t ml, lse;
  const size_t o = kvq_attend_floats(B, s->n_heads, s->n_kv_heads, hd, R, &ml, &lse);
  if (align256(o * 4) + align256(ml * 4) + align256(lse * 4) > workspace_bytes)
    return fail(SPADE_ECAPACITY, "workspace of %zu bytes is too small", workspace_bytes);
  const int64_t e = dtype == SPADE_F32 ? 4 : 2, nq = s->n_heads * hd * e;
  if (rows_overlap(d_q, nq, q_ld * e, d_out, nq, out_ld * e, (int64_t)B * R)) return fail(SPADE_EINVAL, "q and out overlap");
  KvqAttend a{};
  a.cache = (const uint8_t*)d_cache + layer * kvq_layer_bytes(s);
  a.head_bytes = kvq_head_bytes(s->max_len, hd);
  a.B = B;
  a.R = R;
  a.H = s->n_heads;
  a.KVH = s->n_kv_heads;
  a.G = s->n_heads / s->n_kv_heads;
  a.hd = hd;
  a.max_len = s->max_len;
  a.q = d_q;
  a.q_ld = q_ld;
  a.bf16 = dtype == SPADE_BF16;
  a.scale = scale;
  a.lens = d_lens;
  a.rows = d_rows;
  a.max_keys = max_keys;
  a.out = d_out;
  a.out_ld = out_ld;
  a.w_in = d_weights_in;
  a.w_out = d_weights_out;
  a.w_rows = weight_rows;
  a.part_o = (float*)d_workspace;
  a.part_rows = o / hd;
  a.part_ml = (float*)((uint8_t*)d_workspace + align256(o * 4));
  a.lse = (float*)((uint8_t*)d_workspace + align256(o * 4) + align256(ml * 4));
  a.err = d_err;
  const hipError_t r2 = launch_kvq_attend(a, (hipStream_t)stream);
  if (r2 != hipSuccess) return hipfail(r2, "kvq_attend");
  return SPADE_OK;
}

spade_status spade_kvq_evict(const spade_kvq_shape* s, const void* d_cache, const spade_kvq_shape* s_out,
                             void* d_cache_out, int B, int budget, int recent, const float* d_weights,
                             float* d_weights_out, const int32_t* d_lens, int32_t* d_lens_out, int32_t* d_kept,
                             void* stream) {
  spade_status r = check_kvq_call(s, 0, B, SPADE_F32);
  if (r == SPADE_OK) r = check_kvq_call(s_out, 0, B, SPADE_F32);
  if (r != SPADE_OK) return r;
  if (!d_cache || !d_cache_out || !d_weights || !d_lens || !d_lens_out || !d_kept)
    return fail(SPADE_EINVAL, "null pointer");
  if (s->n_layers != s_out->n_layers || s->n_heads != s_out->n_heads || s->n_kv_heads != s_out->n_kv_heads ||
      s->head_dim != s_out->head_dim)
    return fail(SPADE_EINVAL, "the shapes differ in more than batch and max_len");
  if (budget < 1 || budget > s_out->max_len) return fail(SPADE_ECAPACITY, "budget must be in [1, max_len of the output]");
  if (recent < 0 || recent > budget) return fail(SPADE_EINVAL, "recent must be in [0, budget]");
  if (((uintptr_t)d_cache | (uintptr_t)d_cache_out) & 255) return fail(SPADE_EINVAL, "caches must be 256-byte aligned");
  const bool same = s->batch == s_out->batch && s->max_len == s_out->max_len;
  if (d_cache == d_cache_out) {
    if (!same) return fail(SPADE_EINVAL, "in place the shapes must be the same");
  } else if (overlap(d_cache, spade_kvq_bytes(s), d_cache_out, spade_kvq_bytes(s_out))) {
    return fail(SPADE_EINVAL, "the caches overlap");
  }
  if (d_weights_out) {
    const size_t n = (size_t)s->n_layers * s->n_kv_heads * 4;
    if (d_weights == d_weights_out) {
      if (!same) return fail(SPADE_EINVAL, "in place the shapes must be the same");
    } else if (overlap(d_weights, n * s->batch * s->max_len, d_weights_out, n * s_out->batch * s_out->max_len)) {
      return fail(SPADE_EINVAL, "the weights overlap");
    }
  }
  KvqEvict a{};
  a.cache = (const uint8_t*)d_cache;
  a.head_bytes = kvq_head_bytes(s->max_len, s->head_dim);
  a.out = (uint8_t*)d_cache_out;
  a.out_head_bytes = kvq_head_bytes(s_out->max_len, s->head_dim);
  a.L = s->n_layers;
  a.batch = s->batch;
  a.B = B;
  a.KVH = s->n_kv_heads;
  a.hd = s->head_dim;
  a.max_len = s->max_len;
  a.out_batch = s_out->batch;
  a.out_max_len = s_out->max_len;
  a.budget = budget;
  a.recent = recent;
  a.w = d_weights;
  a.w_out = d_weights_out;
  a.lens = d_lens;
  a.lens_out = d_lens_out;
  a.kept = d_kept;
  const hipError_t e = launch_kvq_evict(a, (hipStream_t)stream);
  if (e != hipSuccess) return hipfail(e, "kvq_evict");
  return SPADE_OK;
}

spade_status spade_get_device_error(spade_model m, uint32_t* h_flags, void* stream) {
  if (!m || !h_flags) return fail(SPADE_EINVAL, "null pointer");
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipMemcpyAsync(h_flags, m->ws.err, 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e == hipSuccess) e = hipMemsetAsync(m->ws.err, 0, 4, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return hipfail(e, "get_device_error");
  return SPADE_OK;
}

}  // extern "C"
