// C ABI of the calls around the decode step: argument validation, workspace sizes, dispatch.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "prr.h"
#include "prr_context.h"
#include "prr_launch.h"

namespace {

using prr::api_fail;
using prr::api_ok;

#define PRR_TRY(expr)             \
  do {                            \
    const prr_status _s = (expr); \
    if (_s != PRR_OK) return _s;  \
  } while (0)

constexpr int kMaxRows = 1 << 24;    // rows of packed tensors
constexpr int kMaxTokens = 1 << 30;  // tokens of one sequence
constexpr int kMaxList = 1 << 20;    // entries of a page list

prr_status hip_status(hipError_t e, const char* what) {
  if (e != hipSuccess) return api_fail(PRR_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return api_ok();
}

int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

prr_status check_batch(const prr_dims* d, const prr_batch* b) {
  if (!b) return api_fail(PRR_ERR_INVALID_ARG, "batch is NULL");
  if (b->n_seqs < 1 || b->n_seqs > PRR_MAX_SEQS)
    return api_fail(PRR_ERR_INVALID_ARG, "n_seqs %d outside [1, %d]", b->n_seqs, PRR_MAX_SEQS);
  if (b->total_q < 1 || b->total_q > kMaxRows)
    return api_fail(PRR_ERR_INVALID_ARG, "total_q %d outside [1, %d]", b->total_q, kMaxRows);
  if (!b->cu_q && b->total_q < b->n_seqs)
    return api_fail(PRR_ERR_INVALID_ARG, "total_q %d < n_seqs %d without cu_q", b->total_q, b->n_seqs);
  if (b->max_q < (b->cu_q ? 0 : 1) || b->max_q > b->total_q)
    return api_fail(PRR_ERR_INVALID_ARG, "max_q %d outside [%d, total_q %d]", b->max_q, b->cu_q ? 0 : 1, b->total_q);
  if (b->max_kv < 0 || b->max_kv > kMaxTokens)
    return api_fail(PRR_ERR_INVALID_ARG, "max_kv %d outside [0, %d]", b->max_kv, kMaxTokens);
  PRR_TRY(prr::api_check_ptr(b->kv_len, "kv_len", 4));
  if (b->cu_q) PRR_TRY(prr::api_check_ptr(b->cu_q, "cu_q", 4));
  int64_t pages = d->max_pages;
  if (b->page_table) {
    PRR_TRY(prr::api_check_ptr(b->page_table, "page_table", 4));
    if (b->table_stride < 1) return api_fail(PRR_ERR_INVALID_ARG, "table_stride %d < 1", b->table_stride);
    pages = b->table_stride;
  } else if (b->n_seqs != 1) {
    return api_fail(PRR_ERR_INVALID_ARG, "page_table is NULL with %d sequences", b->n_seqs);
  }
  if (b->max_kv > pages * d->page_size)
    return api_fail(PRR_ERR_INVALID_ARG, "max_kv %d exceeds %lld pages of %d tokens", b->max_kv, (long long)pages,
                    d->page_size);
  return PRR_OK;
}

prr::BatchArgs batch_args(const prr_batch* b) {
  prr::BatchArgs a;
  a.cu_q = b->cu_q;
  a.kv_len = b->kv_len;
  a.page_table = b->page_table;
  a.n_seqs = b->n_seqs;
  // rows that a sequence can have: the device cuts cu_q to them
  a.total_q = b->cu_q ? (int)std::min((int64_t)b->total_q, (int64_t)b->n_seqs * b->max_q) : b->n_seqs;
  a.max_q = b->cu_q ? b->max_q : 1;
  a.max_kv = b->max_kv;
  a.table_stride = b->table_stride;
  return a;
}

prr_status check_kind(int32_t kind) {
  if (kind != PRR_KV_16 && kind != PRR_KV_E4M3) return api_fail(PRR_ERR_INVALID_ARG, "kv_kind %d", kind);
  return PRR_OK;
}

void cache_shape(const prr_dims* d, prr::CacheArgs& c) {
  c.num_kv_heads = d->num_kv_heads;
  c.max_pages = d->max_pages;
  c.page_size = d->page_size;
  c.page_shift = log2_of(d->page_size);
}

prr_status check_cache(const prr_dims* d, int32_t kind, const void* k, const void* v, const uint8_t* ks,
                       const uint8_t* vs, prr::CacheArgs& c) {
  PRR_TRY(check_kind(kind));
  PRR_TRY(prr::api_check_ptr(k, "k_cache", 16));
  PRR_TRY(prr::api_check_ptr(v, "v_cache", 16));
  if (kind == PRR_KV_E4M3) {
    PRR_TRY(prr::api_check_ptr(ks, "k_scale", 16));
    PRR_TRY(prr::api_check_ptr(vs, "v_scale", 16));
  }
  c.k = const_cast<void*>(k);
  c.v = const_cast<void*>(v);
  c.k_scale = const_cast<uint8_t*>(ks);
  c.v_scale = const_cast<uint8_t*>(vs);
  cache_shape(d, c);
  return PRR_OK;
}

// The grids put KV heads on a dimension of at most 65535.
prr_status check_heads(const prr_dims* d) {
  PRR_TRY(prr::api_check_dims(d));
  if (d->num_kv_heads > 4096) return api_fail(PRR_ERR_UNSUPPORTED, "num_kv_heads %d > 4096", d->num_kv_heads);
  return PRR_OK;
}

prr_status check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return PRR_OK;
  if (!ws) return api_fail(PRR_ERR_WORKSPACE, "workspace is NULL, %zu bytes needed", need);
  if (reinterpret_cast<uintptr_t>(ws) % 256) return api_fail(PRR_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (have < need) return api_fail(PRR_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", have, need);
  return PRR_OK;
}

// Bytes of the partial rows (o of 128 floats, then two floats) of nsplit parts; 0 without parts.
size_t parts_bytes(int64_t rows, int nsplit) {
  if (nsplit <= 1) return 0;
  return ((size_t)rows * nsplit * (128 + 2) * 4 + 255) / 256 * 256;
}

// The shape of a call's scores: its device arguments, and the bits of a kernel's instance (0: NULL, or nothing in it).
prr_status check_shape(const prr_shape* sh, prr::ShapeArgs& a, int& bits) {
  memset(&a, 0, sizeof(a));
  bits = 0;
  if (!sh) return PRR_OK;
  if (sh->cap != 0.0f && !(sh->cap >= 0x1p-10f && sh->cap <= 0x1p20f))
    return api_fail(PRR_ERR_INVALID_ARG, "cap %g is not 0 or in [2^-10, 2^20]", sh->cap);
  if (sh->window < 0 || sh->window > kMaxTokens)
    return api_fail(PRR_ERR_INVALID_ARG, "window %d outside [0, %d]", sh->window, kMaxTokens);
  if (sh->slopes) PRR_TRY(prr::api_check_ptr(sh->slopes, "slopes", 4));
  if (sh->prefix) PRR_TRY(prr::api_check_ptr(sh->prefix, "prefix", 4));
  if (sh->first) PRR_TRY(prr::api_check_ptr(sh->first, "first", 4));
  a.slopes = sh->slopes;
  a.prefix = sh->prefix;
  a.first = sh->first;
  a.window = sh->window;
  if (sh->cap != 0.0f) {
    a.cap = (float)(sh->cap * 11.313708498984761);
    a.inv = 1.0f / a.cap;
    a.small = a.cap * (float)prr::kTanhRange;
    a.wide = sh->cap > prr::kMostCap;
    for (int i = 0; i < 4; ++i) {
      const double k = prr::kTanh[i] * pow((double)a.cap, -2.0 * (i + 1));
      a.k[i] = (float)k;
      a.k2[i] = (float)(k * 0.08838834764831845 * 1.4426950408889634);
    }
    bits |= prr::kShapeCap;
  }
  if (sh->slopes || a.wide) bits |= prr::kShapeSlopes;  // (those instances take NULL for slopes of 0)
  if (bits || sh->window || sh->prefix || sh->first) bits |= prr::kShapeSpan;
  return PRR_OK;
}

prr_status plan(const prr_dims* d, const prr_batch* b, const prr_shape* sh, prr::PromptLaunch& a) {
  PRR_TRY(check_heads(d));
  PRR_TRY(check_batch(d, b));
  memset(&a, 0, sizeof(a));
  PRR_TRY(check_shape(sh, a.sh, a.shape));
  a.b = batch_args(b);
  a.num_kv_heads = d->num_kv_heads;
  a.group = d->num_q_heads / d->num_kv_heads;
  a.max_pages = d->max_pages;
  a.page_shift = log2_of(d->page_size);
  a.bf16 = d->dtype == PRR_BF16;
  // (128 GiB of queries)
  if ((int64_t)a.b.total_q * d->num_q_heads > ((int64_t)1 << 29))
    return api_fail(PRR_ERR_UNSUPPORTED, "%d rows x %d heads: more than 2^29", a.b.total_q, d->num_q_heads);
  prr::plan_prompt(a);
  const int64_t groups = (int64_t)a.tiles * a.num_kv_heads;
  if (groups * a.waves * 64 >= (int64_t)1 << 32)
    return api_fail(PRR_ERR_UNSUPPORTED, "%d sequences, %d rows and %d KV heads: %lld workgroups of %d waves", a.b.n_seqs,
                    a.b.total_q, a.num_kv_heads, (long long)groups, a.waves);
  return PRR_OK;
}

prr_status plan(const prr_dims* d, const prr_batch* b, const prr_shape* sh, int32_t kind, int32_t cap, prr::DecodeLaunch& a) {
  PRR_TRY(check_heads(d));
  PRR_TRY(check_batch(d, b));
  PRR_TRY(check_kind(kind));
  if (b->cu_q) return api_fail(PRR_ERR_INVALID_ARG, "cu_q is set: one token per sequence only");
  if (cap < 0 || cap > kMaxList || (int64_t)cap * d->page_size > kMaxTokens)
    return api_fail(PRR_ERR_INVALID_ARG, "cap %d outside [0, %d]", cap, std::min(kMaxList, kMaxTokens / d->page_size));
  memset(&a, 0, sizeof(a));
  PRR_TRY(check_shape(sh, a.sh, a.shape));
  a.b = batch_args(b);
  cache_shape(d, a.c);
  a.group = d->num_q_heads / d->num_kv_heads;
  a.cap = cap;
  a.bf16 = d->dtype == PRR_BF16;
  a.e4m3 = kind == PRR_KV_E4M3;
  prr::plan_decode(a);
  return PRR_OK;
}

prr_status plan(const prr_dims* d, const prr_batch* b, const prr_shape* sh, int32_t kind, int32_t last, int32_t cap,
                prr::MassLaunch& a) {
  PRR_TRY(check_heads(d));
  PRR_TRY(check_batch(d, b));
  PRR_TRY(check_kind(kind));
  if (last < 0) return api_fail(PRR_ERR_INVALID_ARG, "last %d < 0", last);
  if (cap < 0 || cap > kMaxList || (int64_t)cap * d->page_size > kMaxTokens)
    return api_fail(PRR_ERR_INVALID_ARG, "cap %d outside [0, %d]", cap, std::min(kMaxList, kMaxTokens / d->page_size));
  memset(&a, 0, sizeof(a));
  PRR_TRY(check_shape(sh, a.sh, a.shape));
  a.b = batch_args(b);
  cache_shape(d, a.c);
  a.group = d->num_q_heads / d->num_kv_heads;
  a.cap = cap;
  a.last = last;
  a.bf16 = d->dtype == PRR_BF16;
  a.e4m3 = kind == PRR_KV_E4M3;
  prr::plan_mass(a);
  return PRR_OK;
}

size_t mass_bytes(const prr::MassLaunch& a) {
  if (a.nsplit <= 1) return 0;
  return ((size_t)a.nsplit * a.b.n_seqs * a.c.num_kv_heads * a.part_keys * 4 + 255) / 256 * 256;
}

prr_status plan(const prr_dims* d, const prr_batch* b, int32_t budget, int32_t sink, int32_t recent, prr::KeepLaunch& a) {
  PRR_TRY(check_heads(d));
  PRR_TRY(check_batch(d, b));
  if (budget < 1 || budget > kMaxTokens) return api_fail(PRR_ERR_INVALID_ARG, "budget %d outside [1, %d]", budget, kMaxTokens);
  if (sink < 0 || recent < 0 || (int64_t)sink + recent > budget)
    return api_fail(PRR_ERR_INVALID_ARG, "sink %d and recent %d: negative, or more than the budget %d", sink, recent, budget);
  memset(&a, 0, sizeof(a));
  a.b = batch_args(b);
  a.num_kv_heads = d->num_kv_heads;
  a.max_pages = d->max_pages;
  a.page_size = d->page_size;
  a.page_shift = log2_of(d->page_size);
  a.budget = budget;
  a.sink = sink;
  a.recent = recent;
  prr::plan_keep(a);
  return PRR_OK;
}

size_t keep_bytes(const prr::KeepLaunch& a) {
  return a.chunks == 1 ? 0 : (size_t)a.b.n_seqs * a.num_kv_heads * prr::keep_words(a) * 4;
}

prr_status plan(const prr_dims* d, const prr_batch* b, int32_t kind, int32_t budget, prr::CompactLaunch& a) {
  PRR_TRY(check_heads(d));
  PRR_TRY(check_batch(d, b));
  PRR_TRY(check_kind(kind));
  if (budget < 1 || budget > kMaxTokens) return api_fail(PRR_ERR_INVALID_ARG, "budget %d outside [1, %d]", budget, kMaxTokens);
  memset(&a, 0, sizeof(a));
  a.b = batch_args(b);
  cache_shape(d, a.c);
  a.budget = budget;
  a.stage_rows = std::min(budget, b->max_kv);
  a.e4m3 = kind == PRR_KV_E4M3;
  return PRR_OK;
}

template <class A>
int64_t part_rows(const prr_dims* d, const A& a) {
  return (int64_t)a.b.total_q * d->num_q_heads;
}

}  // namespace

extern "C" {

prr_status prr_rope_freqs(int32_t kind, int32_t rot_dim, double base, double factor, int32_t trained_len, double lo,
                          double hi, double* freqs, float* scale) {
  if (kind < PRR_ROPE_PLAIN || kind > PRR_ROPE_YARN) return api_fail(PRR_ERR_INVALID_ARG, "kind %d", kind);
  if (rot_dim < 2 || rot_dim > 128 || rot_dim % 2 != 0)
    return api_fail(PRR_ERR_INVALID_ARG, "rot_dim %d is not even in [2, 128]", rot_dim);
  if (!(base > 1.0) || !isfinite(base)) return api_fail(PRR_ERR_INVALID_ARG, "base %g", base);
  if (!freqs) return api_fail(PRR_ERR_INVALID_ARG, "freqs is NULL");
  if (!scale) return api_fail(PRR_ERR_INVALID_ARG, "scale is NULL");
  if (kind != PRR_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor)))
    return api_fail(PRR_ERR_INVALID_ARG, "factor %g < 1", factor);
  if (kind == PRR_ROPE_NTK && rot_dim < 4) return api_fail(PRR_ERR_INVALID_ARG, "rot_dim %d < 4", rot_dim);
  const bool ramp = kind == PRR_ROPE_BY_PARTS || kind == PRR_ROPE_YARN;
  if (ramp && trained_len < 1) return api_fail(PRR_ERR_INVALID_ARG, "trained_len %d < 1", trained_len);
  if (ramp && !(lo > 0.0 && hi > lo && isfinite(hi)))
    return api_fail(PRR_ERR_INVALID_ARG, "lo %g, hi %g: not 0 < lo < hi", lo, hi);
  const double two_pi = 6.283185307179586476925;
  const int half = rot_dim / 2;
  const double b = kind == PRR_ROPE_NTK ? base * pow(factor, rot_dim / (double)(rot_dim - 2)) : base;
  const auto index_of = [&](double turns) { return rot_dim * log(trained_len / (turns * two_pi)) / (2.0 * log(base)); };
  double i0 = 0.0, i1 = 0.0;
  if (kind == PRR_ROPE_YARN) {
    i0 = std::max(floor(index_of(hi)), 0.0);
    i1 = std::min(ceil(index_of(lo)), rot_dim - 1.0);
  }
  for (int i = 0; i < half; ++i) {
    const double w = pow(b, -2.0 * i / rot_dim);
    double g = kind == PRR_ROPE_LINEAR ? 0.0 : 1.0;  // the share that keeps its frequency
    if (kind == PRR_ROPE_BY_PARTS) g = (trained_len * w / two_pi - lo) / (hi - lo);
    if (kind == PRR_ROPE_YARN) g = 1.0 - (i - i0) / std::max(i1 - i0, 1e-3);
    g = std::min(std::max(g, 0.0), 1.0);
    freqs[i] = kind == PRR_ROPE_PLAIN || kind == PRR_ROPE_NTK ? w : g * w + (1.0 - g) * (w / factor);
  }
  *scale = kind == PRR_ROPE_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  return api_ok();
}

prr_status prr_rope_append(const prr_dims* dims, const prr_batch* batch, const void* q, const void* k, const void* v,
                           int64_t q_stride, int64_t k_stride, int64_t v_stride, const int32_t* positions,
                           const double* freqs, int32_t rot_dim, int32_t layout, float rope_scale, void* q_out,
                           int32_t kv_kind, void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale,
                           hipStream_t stream) {
  PRR_TRY(check_heads(dims));
  PRR_TRY(check_batch(dims, batch));
  PRR_TRY(check_kind(kv_kind));
  if (!q && !k && !v) return api_fail(PRR_ERR_INVALID_ARG, "q, k and v are NULL");
  if (!k != !v) return api_fail(PRR_ERR_INVALID_ARG, "k and v: one of the two is NULL");
  if (!q != !q_out) return api_fail(PRR_ERR_INVALID_ARG, "q and q_out: one of the two is NULL");
  prr::RopeLaunch a;
  memset(&a, 0, sizeof(a));
  if (q) {
    PRR_TRY(prr::api_check_ptr(q, "q", 8));
    PRR_TRY(prr::api_check_ptr(q_out, "q_out", 8));
    if (q_stride < 0 || q_stride % 4) return api_fail(PRR_ERR_INVALID_ARG, "q_stride %lld", (long long)q_stride);
    if (q == q_out && q_stride != (int64_t)dims->num_q_heads * 128 && batch->total_q > 1)
      return api_fail(PRR_ERR_INVALID_ARG, "q_out = q with q_stride %lld: in place only where q is dense",
                      (long long)q_stride);
  }
  if (k) {
    PRR_TRY(prr::api_check_ptr(k, "k", 8));
    PRR_TRY(prr::api_check_ptr(v, "v", 8));
    if (k_stride < 0 || k_stride % 4) return api_fail(PRR_ERR_INVALID_ARG, "k_stride %lld", (long long)k_stride);
    if (v_stride < 0 || v_stride % 4) return api_fail(PRR_ERR_INVALID_ARG, "v_stride %lld", (long long)v_stride);
    PRR_TRY(check_cache(dims, kv_kind, k_cache, v_cache, k_scale, v_scale, a.c));
  }
  if (rot_dim < 0 || rot_dim > 128) return api_fail(PRR_ERR_INVALID_ARG, "rot_dim %d outside [0, 128]", rot_dim);
  if (rot_dim % 8) return api_fail(PRR_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 8", rot_dim);
  if (rot_dim) PRR_TRY(prr::api_check_ptr(freqs, "freqs", 8));
  if (positions) PRR_TRY(prr::api_check_ptr(positions, "positions", 4));
  if (layout != PRR_ROPE_HALF && layout != PRR_ROPE_INTERLEAVED)
    return api_fail(PRR_ERR_INVALID_ARG, "layout %d", layout);
  if (!isfinite(rope_scale)) return api_fail(PRR_ERR_INVALID_ARG, "rope_scale %g", rope_scale);
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.positions = positions;
  a.freqs = freqs;
  a.q_out = q_out;
  a.c.num_kv_heads = dims->num_kv_heads;
  a.c.max_pages = dims->max_pages;
  a.c.page_size = dims->page_size;
  a.c.page_shift = log2_of(dims->page_size);
  a.b = batch_args(batch);
  a.num_q_heads = dims->num_q_heads;
  a.rot_dim = rot_dim;
  a.scale = rope_scale;
  a.bf16 = dims->dtype == PRR_BF16;
  a.e4m3 = kv_kind == PRR_KV_E4M3;
  a.interleaved = layout == PRR_ROPE_INTERLEAVED;
  if (a.b.total_q == 0) return api_ok();  // (no sequence has a new token)
  return hip_status(prr::launch_rope_append(a, stream), "rope append");
}

prr_status prr_cache_read(const prr_dims* dims, const void* k_codes, const void* v_codes, const uint8_t* k_scale,
                          const uint8_t* v_scale, const int32_t* page_table, int32_t num_tokens, int32_t page_begin,
                          int32_t page_end, void* k_out, void* v_out, hipStream_t stream) {
  PRR_TRY(check_heads(dims));
  prr::CacheReadLaunch a;
  memset(&a, 0, sizeof(a));
  PRR_TRY(check_cache(dims, PRR_KV_E4M3, k_codes, v_codes, k_scale, v_scale, a.c));
  PRR_TRY(prr::api_check_ptr(k_out, "k_out", 16));
  PRR_TRY(prr::api_check_ptr(v_out, "v_out", 16));
  if (page_table) PRR_TRY(prr::api_check_ptr(page_table, "page_table", 4));
  if (num_tokens < 1 || num_tokens > kMaxTokens)
    return api_fail(PRR_ERR_INVALID_ARG, "num_tokens %d outside [1, %d]", num_tokens, kMaxTokens);
  const int pages = (num_tokens + dims->page_size - 1) / dims->page_size;
  if (!page_table && pages > dims->max_pages)
    return api_fail(PRR_ERR_INVALID_ARG, "num_tokens %d exceeds max_pages %d pages of %d tokens", num_tokens,
                    dims->max_pages, dims->page_size);
  if (page_begin < 0 || page_begin > page_end || page_end > pages)
    return api_fail(PRR_ERR_INVALID_ARG, "pages [%d, %d) outside [0, %d)", page_begin, page_end, pages);
  if (page_begin == page_end) return api_ok();
  a.page_table = page_table;
  a.k_out = k_out;
  a.v_out = v_out;
  a.num_tokens = num_tokens;
  a.page_begin = page_begin;
  a.pages = page_end - page_begin;
  a.bf16 = dims->dtype == PRR_BF16;
  return hip_status(prr::launch_cache_read(a, stream), "cache read");
}

size_t prr_prompt_workspace_size(const prr_dims* dims, const prr_batch* batch) {
  return prr_prompt_shaped_workspace_size(dims, batch, nullptr);
}

size_t prr_prompt_shaped_workspace_size(const prr_dims* dims, const prr_batch* batch, const prr_shape* shape) {
  prr::PromptLaunch a;
  if (plan(dims, batch, shape, a) != PRR_OK) return 0;
  return parts_bytes(part_rows(dims, a), a.nsplit);
}

prr_status prr_prompt_attn(const prr_dims* dims, const prr_batch* batch, const void* q, const void* k_cache,
                           const void* v_cache, void* out_o, float* out_m, float* out_l, void* workspace,
                           size_t ws_bytes, hipStream_t stream) {
  return prr_prompt_attn_shaped(dims, batch, nullptr, q, k_cache, v_cache, out_o, out_m, out_l, workspace, ws_bytes, stream);
}

prr_status prr_prompt_attn_shaped(const prr_dims* dims, const prr_batch* batch, const prr_shape* shape, const void* q,
                                  const void* k_cache, const void* v_cache, void* out_o, float* out_m, float* out_l,
                                  void* workspace, size_t ws_bytes, hipStream_t stream) {
  prr::PromptLaunch a;
  PRR_TRY(plan(dims, batch, shape, a));
  PRR_TRY(prr::api_check_ptr(q, "q", 16));
  PRR_TRY(prr::api_check_ptr(k_cache, "k_cache", 16));
  PRR_TRY(prr::api_check_ptr(v_cache, "v_cache", 16));
  PRR_TRY(prr::api_check_ptr(out_o, "out_o", 16));
  if (!out_m != !out_l) return api_fail(PRR_ERR_INVALID_ARG, "out_m and out_l: one of the two is NULL");
  if (out_m) {
    PRR_TRY(prr::api_check_ptr(out_m, "out_m", 4));
    PRR_TRY(prr::api_check_ptr(out_l, "out_l", 4));
  }
  const int64_t rows = part_rows(dims, a);
  PRR_TRY(check_ws(workspace, ws_bytes, parts_bytes(rows, a.nsplit)));
  a.q = q;
  a.k = k_cache;
  a.v = v_cache;
  a.out_o = out_o;
  a.out_m = out_m;
  a.out_l = out_l;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = a.nsplit > 1 ? a.part_o + rows * a.nsplit * 128 : nullptr;
  if (a.tiles == 0) return api_ok();  // (no sequence has a new token)
  return hip_status(prr::launch_prompt(a, stream), "prompt attention");
}

size_t prr_decode_workspace_size(const prr_dims* dims, const prr_batch* batch, int32_t kv_kind, int32_t cap) {
  return prr_decode_shaped_workspace_size(dims, batch, nullptr, kv_kind, cap);
}

size_t prr_decode_shaped_workspace_size(const prr_dims* dims, const prr_batch* batch, const prr_shape* shape, int32_t kv_kind,
                                        int32_t cap) {
  prr::DecodeLaunch a;
  if (plan(dims, batch, shape, kv_kind, cap, a) != PRR_OK) return 0;
  return parts_bytes(part_rows(dims, a), a.nsplit);
}

prr_status prr_decode_attn(const prr_dims* dims, const prr_batch* batch, const void* q, int32_t kv_kind,
                           const void* k_cache, const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale,
                           const int32_t* pages, const int32_t* page_count, int32_t cap, float* out_o32, void* out_o,
                           float* out_m, float* out_l, void* workspace, size_t ws_bytes, hipStream_t stream) {
  return prr_decode_attn_shaped(dims, batch, nullptr, q, kv_kind, k_cache, v_cache, k_scale, v_scale, pages, page_count, cap,
                                out_o32, out_o, out_m, out_l, workspace, ws_bytes, stream);
}

prr_status prr_decode_attn_shaped(const prr_dims* dims, const prr_batch* batch, const prr_shape* shape, const void* q,
                                  int32_t kv_kind, const void* k_cache, const void* v_cache, const uint8_t* k_scale,
                                  const uint8_t* v_scale, const int32_t* pages, const int32_t* page_count, int32_t cap,
                                  float* out_o32, void* out_o, float* out_m, float* out_l, void* workspace, size_t ws_bytes,
                                  hipStream_t stream) {
  if (!pages != !page_count) return api_fail(PRR_ERR_INVALID_ARG, "pages and page_count: one of the two is NULL");
  if (pages && cap < 1) return api_fail(PRR_ERR_INVALID_ARG, "cap %d < 1 with lists", cap);
  prr::DecodeLaunch a;
  PRR_TRY(plan(dims, batch, shape, kv_kind, pages ? cap : 0, a));
  PRR_TRY(check_cache(dims, kv_kind, k_cache, v_cache, k_scale, v_scale, a.c));
  PRR_TRY(prr::api_check_ptr(q, "q", 16));
  if (pages) {
    PRR_TRY(prr::api_check_ptr(pages, "pages", 4));
    PRR_TRY(prr::api_check_ptr(page_count, "page_count", 4));
  }
  PRR_TRY(prr::api_check_ptr(out_o32, "out_o32", 16));
  if (out_o) PRR_TRY(prr::api_check_ptr(out_o, "out_o", 8));
  PRR_TRY(prr::api_check_ptr(out_m, "out_m", 4));
  PRR_TRY(prr::api_check_ptr(out_l, "out_l", 4));
  const int64_t rows = part_rows(dims, a);
  PRR_TRY(check_ws(workspace, ws_bytes, parts_bytes(rows, a.nsplit)));
  a.q = q;
  a.pages = pages;
  a.page_count = page_count;
  a.out_o32 = out_o32;
  a.out_o = out_o;
  a.out_m = out_m;
  a.out_l = out_l;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = a.nsplit > 1 ? a.part_o + rows * a.nsplit * 128 : nullptr;
  return hip_status(prr::launch_decode(a, stream), "decode attention");
}

size_t prr_mass_workspace_size(const prr_dims* dims, const prr_batch* batch, const prr_shape* shape, int32_t kv_kind,
                               int32_t last, int32_t cap) {
  prr::MassLaunch a;
  if (plan(dims, batch, shape, kv_kind, last, cap, a) != PRR_OK) return 0;
  return mass_bytes(a);
}

prr_status prr_key_mass(const prr_dims* dims, const prr_batch* batch, const prr_shape* shape, const void* q, int32_t kv_kind,
                        const void* k_cache, const uint8_t* k_scale, const float* m, const float* l, int32_t last,
                        const int32_t* pages, const int32_t* page_count, int32_t cap, const float* mass_in, float decay,
                        float* mass_out, void* workspace, size_t ws_bytes, hipStream_t stream) {
  if (!pages != !page_count) return api_fail(PRR_ERR_INVALID_ARG, "pages and page_count: one of the two is NULL");
  if (pages && cap < 1) return api_fail(PRR_ERR_INVALID_ARG, "cap %d < 1 with lists", cap);
  prr::MassLaunch a;
  PRR_TRY(plan(dims, batch, shape, kv_kind, last, pages ? cap : 0, a));
  if (pages && batch->cu_q) return api_fail(PRR_ERR_INVALID_ARG, "cu_q is set: lists are of one token per sequence");
  PRR_TRY(prr::api_check_ptr(q, "q", 16));
  PRR_TRY(prr::api_check_ptr(k_cache, "k_cache", 16));
  if (kv_kind == PRR_KV_E4M3) PRR_TRY(prr::api_check_ptr(k_scale, "k_scale", 16));
  PRR_TRY(prr::api_check_ptr(m, "m", 4));
  PRR_TRY(prr::api_check_ptr(l, "l", 4));
  if (pages) {
    PRR_TRY(prr::api_check_ptr(pages, "pages", 4));
    PRR_TRY(prr::api_check_ptr(page_count, "page_count", 4));
  }
  if (mass_in) PRR_TRY(prr::api_check_ptr(mass_in, "mass_in", 4));
  if (mass_in && !isfinite(decay)) return api_fail(PRR_ERR_INVALID_ARG, "decay %g", decay);
  PRR_TRY(prr::api_check_ptr(mass_out, "mass_out", 4));
  PRR_TRY(check_ws(workspace, ws_bytes, mass_bytes(a)));
  a.q = q;
  a.c.k = const_cast<void*>(k_cache);
  a.c.k_scale = const_cast<uint8_t*>(k_scale);
  a.m = m;
  a.l = l;
  a.pages = pages;
  a.page_count = page_count;
  a.before = mass_in;
  a.decay = decay;
  a.mass = mass_out;
  a.part = static_cast<float*>(workspace);
  if (a.b.max_kv == 0) return api_ok();  // (no sequence has a token)
  return hip_status(prr::launch_mass(a, stream), "key mass");
}

prr_status prr_mass_clear(const prr_dims* dims, const prr_batch* batch, const int32_t* from_len, float* mass, hipStream_t stream) {
  prr::MassClearLaunch a;
  PRR_TRY(check_heads(dims));
  PRR_TRY(check_batch(dims, batch));
  PRR_TRY(prr::api_check_ptr(from_len, "from_len", 4));
  PRR_TRY(prr::api_check_ptr(mass, "mass", 4));
  memset(&a, 0, sizeof(a));
  a.mass = mass;
  a.from = from_len;
  a.b = batch_args(batch);
  a.num_kv_heads = dims->num_kv_heads;
  a.max_pages = dims->max_pages;
  a.page_size = dims->page_size;
  a.page_shift = log2_of(dims->page_size);
  if (a.b.max_kv == 0) return api_ok();  // (no sequence has a token)
  return hip_status(prr::launch_mass_clear(a, stream), "mass clear");
}

size_t prr_keep_workspace_size(const prr_dims* dims, const prr_batch* batch, int32_t budget) {
  prr::KeepLaunch a;
  if (plan(dims, batch, budget, 0, 0, a) != PRR_OK) return 0;
  return keep_bytes(a);
}

prr_status prr_keep_tokens(const prr_dims* dims, const prr_batch* batch, const float* mass, int32_t budget, int32_t sink,
                           int32_t recent, int32_t* keep, int32_t* kept_len, void* workspace, size_t ws_bytes,
                           hipStream_t stream) {
  prr::KeepLaunch a;
  PRR_TRY(plan(dims, batch, budget, sink, recent, a));
  PRR_TRY(prr::api_check_ptr(mass, "mass", 16));
  PRR_TRY(prr::api_check_ptr(keep, "keep", 4));
  PRR_TRY(prr::api_check_ptr(kept_len, "kept_len", 4));
  if (kept_len == batch->kv_len)  // (other workgroups still read it, and prr_cache_compact needs both)
    return api_fail(PRR_ERR_INVALID_ARG, "kept_len is the batch's kv_len");
  PRR_TRY(check_ws(workspace, ws_bytes, keep_bytes(a)));
  a.mass = mass;
  a.keep = keep;
  a.kept = kept_len;
  a.counts = static_cast<uint32_t*>(workspace);
  return hip_status(prr::launch_keep(a, stream), "keep tokens");
}

size_t prr_compact_workspace_size(const prr_dims* dims, const prr_batch* batch, int32_t kv_kind, int32_t budget,
                                  int32_t in_place) {
  prr::CompactLaunch a;
  if (plan(dims, batch, kv_kind, budget, a) != PRR_OK) return 0;
  return in_place ? prr::compact_stage_bytes(a) : 0;
}

prr_status prr_cache_compact(const prr_dims* dims, const prr_batch* batch, const int32_t* keep, const int32_t* kept_len,
                             int32_t budget, int32_t kv_kind, void* k_cache, void* v_cache, uint8_t* k_scale,
                             uint8_t* v_scale, float* mass, const int32_t* dst_table, int32_t dst_stride, void* workspace,
                             size_t ws_bytes, hipStream_t stream) {
  prr::CompactLaunch a;
  PRR_TRY(plan(dims, batch, kv_kind, budget, a));
  PRR_TRY(check_cache(dims, kv_kind, k_cache, v_cache, k_scale, v_scale, a.c));
  PRR_TRY(prr::api_check_ptr(keep, "keep", 4));
  PRR_TRY(prr::api_check_ptr(kept_len, "kept_len", 4));
  if (mass) PRR_TRY(prr::api_check_ptr(mass, "mass", 4));
  if (dst_table) {
    PRR_TRY(prr::api_check_ptr(dst_table, "dst_table", 4));
    if (dst_table == batch->page_table)
      return api_fail(PRR_ERR_INVALID_ARG, "dst_table is the batch's page_table: NULL means in place");
    if (dst_stride < 1 || (int64_t)dst_stride * dims->page_size < a.stage_rows)
      return api_fail(PRR_ERR_INVALID_ARG, "dst_stride %d: %d tokens need more pages of %d", dst_stride, a.stage_rows, dims->page_size);
  } else {
    PRR_TRY(check_ws(workspace, ws_bytes, prr::compact_stage_bytes(a)));
  }
  a.mass = mass;
  a.keep = keep;
  a.kept = kept_len;
  a.dst_table = dst_table;
  a.dst_stride = dst_stride;
  a.stage = static_cast<char*>(workspace);
  if (a.b.max_kv == 0) return api_ok();  // (no sequence has a token)
  return hip_status(prr::launch_compact(a, stream), "cache compact");
}

}  // extern "C"
