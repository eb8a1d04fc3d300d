// C-ABI entry points of rotary positions and of the 8-bit cache: host-side validation only, every step is a kernel launch.
// Nothing here allocates or keeps records, so nothing throws.
#include <math.h>

#include "serve_internal.h"

using namespace usp;

namespace {

bool on_16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Whether two sets of `rows` pieces, wa and wb bytes long and sa and sb bytes apart, share memory; true also where it is not
// known (pieces of different distances whose extents meet).
bool rows_meet(const void* a, int64_t wa, int64_t sa, const void* b, int64_t wb, int64_t sb, int64_t rows) {
  const int64_t d = (intptr_t)b - (intptr_t)a;
  if (d >= (rows - 1) * sa + wa || -d >= (rows - 1) * sb + wb) return false;
  if (sa != sb) return true;
  const int64_t r = ((d % sa) + sa) % sa;
  return r < wa || r + wb > sa;
}

int check_rope(const usp_rope* r, int hs) {
  if (!r) return USP_ERR_NULL;
  if (hs != 64 && hs != 128) return USP_ERR_UNSUPPORTED;
  if (r->rotary_dim < 16 || r->rotary_dim > hs || r->rotary_dim % 16) return USP_ERR_SHAPE;
  if (r->layout != USP_ROPE_HALVES && r->layout != USP_ROPE_PAIRS) return USP_ERR_UNSUPPORTED;
  if (!isfinite(r->magnitude)) return USP_ERR_UNSUPPORTED;
  for (int j = 0; j < r->rotary_dim / 2; ++j)
    if (!(fabs(r->freq[j]) <= 1e6)) return USP_ERR_UNSUPPORTED;
  return USP_OK;
}

// The fields that both forms fill alike.
void fill_rope(RopeArgs& a, const usp_rope* r, int hs, int backward) {
  const double turn = 6.283185307179586476925286766559;
  for (int j = 0; j < 64; ++j) a.turns[j] = j < r->rotary_dim / 2 ? r->freq[j] / turn : 0.0;
  a.hs = hs;
  a.rotary_dim = r->rotary_dim;
  a.pairs = r->layout == USP_ROPE_PAIRS;
  a.magnitude = r->magnitude;
  a.sign = backward ? -1.0f : 1.0f;
}

// Outputs against inputs and each other, and what each tensor has to be; tensors of n[t] = 0 heads are not there.
int check_rope_tensors(const RopeArgs& a, int64_t rows, size_t es) {
  const int64_t e = (int64_t)es;
  for (int t = 0; t < 2; ++t) {
    if (!a.heads[t]) continue;
    const int64_t w = (int64_t)a.heads[t] * a.hs * e;
    if (!on_16(a.x[t]) || !on_16(a.y[t]) || (a.stride[t] * e) % 16 || (a.out_stride[t] * e) % 16) return USP_ERR_UNSUPPORTED;
    for (int u = 0; u < 2; ++u) {
      if (!a.heads[u]) continue;
      const int64_t wu = (int64_t)a.heads[u] * a.hs * e;
      const bool itself = t == u && a.x[u] == a.y[t] && a.stride[u] == a.out_stride[t];
      if (!itself && rows_meet(a.y[t], w, a.out_stride[t] * e, a.x[u], wu, a.stride[u] * e, rows)) return USP_ERR_UNSUPPORTED;
      if (u > t && rows_meet(a.y[t], w, a.out_stride[t] * e, a.y[u], wu, a.out_stride[u] * e, rows)) return USP_ERR_UNSUPPORTED;
    }
  }
  return USP_OK;
}

int check_cache(const usp_cache* c) {
  if (!c) return USP_ERR_NULL;
  if (c->hk < 1 || c->pages < 1) return USP_ERR_SHAPE;
  if (c->hs != 64 && c->hs != 128) return USP_ERR_UNSUPPORTED;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return USP_ERR_UNSUPPORTED;
  if (c->pages >= ((int64_t)1 << 31) / c->page) return USP_ERR_UNSUPPORTED;
  if (c->hk > 65536) return USP_ERR_UNSUPPORTED;
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return USP_ERR_NULL;
  if (!on_16(c->k_codes) || !on_16(c->v_codes)) return USP_ERR_UNSUPPORTED;
  return USP_OK;
}

int page_shift(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

}  // namespace

extern "C" int usp_rope_init(usp_rope* r, int hs, int rotary_dim, int layout, double base, int scaling, double factor,
                             double alpha, double beta, int64_t original_len, double magnitude) {
  if (!r) return USP_ERR_NULL;
  if (hs != 64 && hs != 128) return USP_ERR_UNSUPPORTED;
  if (rotary_dim < 16 || rotary_dim > hs || rotary_dim % 16) return USP_ERR_SHAPE;
  if (layout != USP_ROPE_HALVES && layout != USP_ROPE_PAIRS) return USP_ERR_UNSUPPORTED;
  if (scaling < USP_ROPE_UNSCALED || scaling > USP_ROPE_BY_PARTS) return USP_ERR_UNSUPPORTED;
  if (!(base > 0) || isinf(base) || !isfinite((float)magnitude)) return USP_ERR_UNSUPPORTED;
  if (scaling != USP_ROPE_UNSCALED && (!(factor > 0) || isinf(factor))) return USP_ERR_UNSUPPORTED;
  if (scaling == USP_ROPE_BY_PARTS && (!(alpha >= 0) || !(beta > alpha) || isinf(beta) || original_len < 1))
    return USP_ERR_UNSUPPORTED;
  usp_rope made = {};
  made.rotary_dim = rotary_dim;
  made.layout = layout;
  made.magnitude = (float)magnitude;
  const double d = rotary_dim, turn = 6.283185307179586476925286766559;
  if (scaling == USP_ROPE_BASE) base *= pow(factor, d / (d - 2));
  for (int j = 0; j < rotary_dim / 2; ++j) {
    double f = pow(base, -2.0 * j / d);
    if (scaling == USP_ROPE_LINEAR) f /= factor;
    if (scaling == USP_ROPE_BY_PARTS) {
      double kept = ((double)original_len * f / turn - alpha) / (beta - alpha);
      kept = kept < 0 ? 0 : kept > 1 ? 1 : kept;
      f = kept * f + (1 - kept) * f / factor;
    }
    if (!(fabs(f) <= 1e6)) return USP_ERR_UNSUPPORTED;   // (a base or a factor far below 1)
    made.freq[j] = f;
  }
  *r = made;
  return USP_OK;
}

extern "C" int usp_rope_shards(const usp_problem* p, const usp_rope* r, const void* q, const void* k, void* q_out,
                               void* k_out, int backward, int rank_begin, int rank_end, void* stream) {
  int st = usp_validate(p);
  if (st != USP_OK) return st;
  st = check_rope(r, p->hs);
  if (st != USP_OK) return st;
  if (!q != !q_out || !k != !k_out || (!q && !k)) return USP_ERR_NULL;
  const int n = p->ulysses * p->ring;
  if (rank_begin < 0 || rank_end > n || rank_begin > rank_end) return USP_ERR_UNSUPPORTED;
  RopeArgs a = {};
  fill_rope(a, r, p->hs, backward);
  const size_t es = dtype_size(p->dtype);
  a.per_shard = p->L / n;
  a.bs = p->bs;
  const int64_t all = (int64_t)n * p->bs * a.per_shard, first = (int64_t)rank_begin * p->bs * a.per_shard;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  for (int t = 0; t < 2; ++t) {
    a.heads[t] = in[t] ? (t ? p->hk : p->hc) : 0;
    a.x[t] = in[t];
    a.y[t] = out[t];
    a.stride[t] = a.out_stride[t] = (int64_t)a.heads[t] * p->hs;
  }
  st = check_rope_tensors(a, all, es);
  if (st != USP_OK) return st;
  if (rank_begin == rank_end) return USP_OK;
  a.in_place = a.x[0] == a.y[0] && a.x[1] == a.y[1];
  for (int t = 0; t < 2; ++t) {
    if (!a.heads[t]) continue;
    a.x[t] = (const char*)a.x[t] + first * a.stride[t] * es;
    a.y[t] = (char*)a.y[t] + first * a.stride[t] * es;
  }
  a.rows = (int64_t)(rank_end - rank_begin) * p->bs * a.per_shard;
  a.rank0 = rank_begin;
  a.ulysses = p->ulysses;
  a.ring = p->ring;
  a.ring_block = p->L / p->ring;
  a.half_chunk = p->split == USP_SPLIT_ZIGZAG ? p->L / (2 * (int64_t)p->ring) : 0;
  return launch_rope(a, p->dtype, (hipStream_t)stream);
}

extern "C" int usp_rope_rows(const usp_rope* r, const void* q, const void* k, void* q_out, void* k_out,
                             const int32_t* positions, int64_t rows, int hq, int hk, int hs, int64_t q_stride,
                             int64_t k_stride, int64_t q_out_stride, int64_t k_out_stride, int dtype, int backward,
                             void* stream) {
  int st = check_rope(r, hs);
  if (st != USP_OK) return st;
  if (rows < 0 || rows >= (int64_t)1 << 31) return USP_ERR_SHAPE;
  if (dtype != USP_BF16 && dtype != USP_FP32) return USP_ERR_DTYPE;
  if (rows == 0) return USP_OK;
  if (!positions || !q != !q_out || !k != !k_out || (!q && !k)) return USP_ERR_NULL;
  if ((q && hq < 1) || (k && hk < 1)) return USP_ERR_SHAPE;
  if (hq > 65536 || hk > 65536) return USP_ERR_UNSUPPORTED;
  RopeArgs a = {};
  fill_rope(a, r, hs, backward);
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const int64_t stride[2] = {q_stride, k_stride}, out_stride[2] = {q_out_stride, k_out_stride};
  const int64_t most = (int64_t)1 << 30;     // elements between rows
  for (int t = 0; t < 2; ++t) {
    a.heads[t] = in[t] ? (t ? hk : hq) : 0;
    a.x[t] = in[t];
    a.y[t] = out[t];
    a.stride[t] = stride[t];
    a.out_stride[t] = out_stride[t];
    if (in[t]) {
      const int64_t row = (int64_t)a.heads[t] * hs;
      if (stride[t] < row || out_stride[t] < row) return USP_ERR_SHAPE;
      if (stride[t] > most || out_stride[t] > most) return USP_ERR_UNSUPPORTED;
    }
  }
  st = check_rope_tensors(a, rows, dtype_size(dtype));
  if (st != USP_OK) return st;
  a.in_place = a.x[0] == a.y[0] && a.x[1] == a.y[1];
  a.positions = positions;
  a.rows = rows;
  return launch_rope(a, dtype, (hipStream_t)stream);
}

extern "C" int usp_cache_extend(const int32_t* cu_new, const int32_t* len_before, int n_seqs, int64_t total_new,
                                int32_t* block_table, int max_pages, int page, int64_t pages, const int32_t* free_pages,
                                int64_t n_free, int32_t* len_after, int32_t* slots, int32_t* positions, int32_t* taken,
                                void* stream) {
  if (n_seqs < 0 || total_new < 0 || n_free < 0 || max_pages < 1 || pages < 1) return USP_ERR_SHAPE;
  if (page != 16 && page != 32 && page != 64 && page != 128) return USP_ERR_UNSUPPORTED;
  if (n_seqs > USP_CACHE_MAX_REQUESTS || total_new >= (int64_t)1 << 31 || n_free >= (int64_t)1 << 31 ||
      pages >= ((int64_t)1 << 31) / page)
    return USP_ERR_UNSUPPORTED;
  if (!taken) return USP_ERR_NULL;
  if (n_seqs > 0 && (!cu_new || !len_before || !block_table || !len_after)) return USP_ERR_NULL;
  if (total_new > 0 && (!slots || !positions)) return USP_ERR_NULL;
  if (n_free > 0 && !free_pages) return USP_ERR_NULL;
  const int32_t* in[] = {cu_new, len_before, free_pages};
  const int32_t* out[] = {block_table, len_after, slots, positions, taken};
  for (int i = 0; i < 5; ++i) {
    for (const int32_t* x : in)
      if (out[i] && out[i] == x) return USP_ERR_UNSUPPORTED;
    for (int j = 0; j < i; ++j)
      if (out[i] && out[i] == out[j]) return USP_ERR_UNSUPPORTED;
  }
  const CacheExtendArgs a = {cu_new, len_before, free_pages, block_table, len_after, slots,  positions,       taken,
                             total_new, pages,   n_free,     n_seqs,      max_pages, page_shift(page)};
  return launch_cache_extend(a, (hipStream_t)stream);
}

extern "C" int usp_cache_append(const usp_cache* c, const void* k, const void* v, const int32_t* slots, int64_t rows,
                                int64_t k_stride, int64_t v_stride, int dtype, void* stream) {
  int st = check_cache(c);
  if (st != USP_OK) return st;
  if (rows < 0 || rows >= (int64_t)1 << 31) return USP_ERR_SHAPE;
  if (dtype != USP_BF16 && dtype != USP_FP32) return USP_ERR_DTYPE;
  if (rows == 0) return USP_OK;
  if (!k || !v || !slots) return USP_ERR_NULL;
  const int64_t row = (int64_t)c->hk * c->hs, es = (int64_t)dtype_size(dtype), most = (int64_t)1 << 30;
  if (k_stride < row || v_stride < row) return USP_ERR_SHAPE;
  if (k_stride > most || v_stride > most) return USP_ERR_UNSUPPORTED;
  if (!on_16(k) || !on_16(v) || k_stride * es % 16 || v_stride * es % 16) return USP_ERR_UNSUPPORTED;
  CacheAppendArgs a = {};
  a.x[0] = k;
  a.x[1] = v;
  a.codes[0] = (uint8_t*)c->k_codes;
  a.codes[1] = (uint8_t*)c->v_codes;
  a.scale[0] = c->k_scale;
  a.scale[1] = c->v_scale;
  a.stride[0] = k_stride;
  a.stride[1] = v_stride;
  a.slots = slots;
  a.rows = rows;
  a.slots_end = c->pages * c->page;
  a.page_shift = page_shift(c->page);
  a.hk = c->hk;
  a.hs = c->hs;
  return launch_cache_append(a, dtype, (hipStream_t)stream);
}

extern "C" size_t usp_cache_attn_workspace_bytes(const usp_cache* c, int hq, int max_q) {
  if (check_cache(c) != USP_OK || hq < 1 || hq % c->hk || hq / c->hk > 65536) return 0;
  return cache_attn_workspace(hq / c->hk, c->hs, max_q);
}

extern "C" int usp_cache_attn(const usp_cache* c, const void* q, int64_t q_stride, const int32_t* cu_q,
                              const int32_t* kv_len, const int32_t* block_table, int max_pages, int n_seqs,
                              int64_t total_q, int max_q, int hq, float scale, int causal, void* o, float* lse, int o_dtype,
                              void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_cache(c);
  if (st != USP_OK) return st;
  if (n_seqs < 0 || total_q < 0 || max_q < 0 || max_pages < 1 || hq < 1) return USP_ERR_SHAPE;
  if (hq % c->hk) return USP_ERR_DEGREE;
  if (n_seqs > USP_CACHE_MAX_REQUESTS || hq / c->hk > 65536 || total_q >= (int64_t)1 << 31) return USP_ERR_UNSUPPORTED;
  if (total_q * (hq / c->hk) >= ((int64_t)1 << 32) - 256) return USP_ERR_UNSUPPORTED;   // rows of a KV head are counted in 32 bits
  if (o_dtype != USP_BF16 && o_dtype != USP_FP32) return USP_ERR_DTYPE;
  if (!(scale >= 0.0f) || isinf(scale)) return USP_ERR_UNSUPPORTED;
  if (n_seqs == 0 || total_q == 0) return USP_OK;
  if (!q || !cu_q || !kv_len || !block_table || !o || !lse) return USP_ERR_NULL;
  if (q_stride < (int64_t)hq * c->hs) return USP_ERR_SHAPE;
  if (q_stride > (int64_t)1 << 30 || !on_16(q) || !on_16(o) || q_stride % 8) return USP_ERR_UNSUPPORTED;
  const size_t need = cache_attn_workspace(hq / c->hk, c->hs, max_q);
  if (!workspace || workspace_bytes < need) return USP_ERR_WORKSPACE;
  if (!on_16(workspace)) return USP_ERR_UNSUPPORTED;
  // O over Q: a unit's rows are read by the wave that writes them, but other waves that share them may not have read yet
  const int64_t ow = (int64_t)hq * c->hs, oes = (int64_t)dtype_size(o_dtype);
  if (rows_meet(o, ow * oes, ow * oes, q, ow * 2, q_stride * 2, total_q)) return USP_ERR_UNSUPPORTED;
  CacheAttnArgs a = {};
  a.k_codes = (const uint8_t*)c->k_codes;
  a.v_codes = (const uint8_t*)c->v_codes;
  a.k_scale = c->k_scale;
  a.v_scale = c->v_scale;
  a.q = q;
  a.cu_q = cu_q;
  a.kv_len = kv_len;
  a.block_table = block_table;
  a.o = o;
  a.lse = lse;
  a.workspace = workspace;
  a.pages = c->pages;
  a.q_stride = q_stride;
  a.total_q = total_q;
  a.page_shift = page_shift(c->page);
  a.hk = c->hk;
  a.hs = c->hs;
  a.group = hq / c->hk;
  a.max_pages = max_pages;
  a.n_seqs = n_seqs;
  a.causal = causal != 0;
  a.o_dtype = o_dtype;
  a.scale_log2e = (scale == 0.0f ? 1.0f / sqrtf((float)c->hs) : scale) * 1.44269504088896340736f;
  return launch_cache_attn(a, max_q, (hipStream_t)stream);
}
