// C ABI of the receiver's side: rotary positions, the paged four-bit cache and
// attention over it.  Argument validation and launches; declared in
// include/cacheback_cache.h.
#include <math.h>
#include <stdint.h>

#include "../../include/cacheback_cache.h"
#include "cache.h"

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

constexpr int64_t kMaxPositions = (int64_t)0x7fffffff - 0xffff;   // 2^31 - 2^16

bool sizes_ok(const cb_cache* c) {
  if (c->layers < 1 || c->kv_heads < 1 || c->pages < 1 || c->seqs < 1 || c->width < 1) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  const int P = c->page_len;
  if (P != 16 && P != 32 && P != 64 && P != 128 && P != 256) return false;
  if (c->layers > 4096 || c->kv_heads > 4096) return false;
  if (c->pages > cb::kCacheMaxPages || c->seqs > cb::kCacheMaxSeqs) return false;
  return (int64_t)c->width * P <= kMaxPositions;
}

int view_of(const cb_cache* c, cb::CacheView* v) {
  if (!c) return CB_ERR_NULL;
  if (!sizes_ok(c)) return CB_ERR_SHAPE;
  if (!c->pool || !c->refs || !c->table || !c->lens) return CB_ERR_NULL;
  if (!aligned(c->pool, 16) || !aligned(c->refs, 16) || !aligned(c->table, 16) ||
      !aligned(c->lens, 16))
    return CB_ERR_ALIGN;
  v->pool = static_cast<unsigned char*>(c->pool);
  v->refs = c->refs;
  v->table = c->table;
  v->lens = c->lens;
  v->unit_bytes = c->page_len * (c->head_dim + c->head_dim / 16);
  v->page_bytes = (int64_t)c->layers * c->kv_heads * v->unit_bytes;
  v->layers = c->layers;
  v->heads = c->kv_heads;
  v->D = c->head_dim;
  v->page_shift = __builtin_ctz((unsigned)c->page_len);
  v->pages = c->pages;
  v->seqs = c->seqs;
  v->width = c->width;
  return CB_OK;
}

int done(hipError_t e) { return e == hipSuccess ? CB_OK : CB_ERR_HIP; }

// Strides of axes that are walked: whole 16-byte vectors, and for an output no
// two rows in one place.
int check_strides(const int64_t* stride, const int64_t* size, int axes, int bytes, bool output) {
  for (int i = 0; i < axes; ++i) {
    if (size[i] <= 1) continue;
    if ((stride[i] * bytes) % 16 != 0) return CB_ERR_ALIGN;
    if (output && stride[i] == 0) return CB_ERR_SHAPE;
  }
  return CB_OK;
}

bool entries_ok(int32_t n) { return n >= 0 && n <= cb::kCacheMaxEntries; }

int layers_ok(const cb_cache* c, int32_t layer0, int32_t layers, int32_t n) {
  if (layers < 0 || layer0 < 0 || n < 0 || (int64_t)layer0 + layers > c->layers) return CB_ERR_SHAPE;
  if ((int64_t)layers * n * c->kv_heads > 0x7fffffff) return CB_ERR_SHAPE;
  return CB_OK;
}

int rows_args(const cb_cache* c, int32_t layer0, int32_t layers, const int32_t* seqs, int32_t n,
              const int32_t* start, const int32_t* counts, int64_t max_count, const void* k,
              const void* v, const int64_t* stride, int32_t dtype, bool output,
              cb::CacheRowsArgs* a) {
  int st = view_of(c, &a->c);
  if (st != CB_OK) return st;
  if (dtype != CB_F32 && dtype != CB_BF16) return CB_ERR_DTYPE;
  st = layers_ok(c, layer0, layers, n);
  if (st != CB_OK) return st;
  if (max_count < 0 || max_count > kMaxPositions) return CB_ERR_SHAPE;
  if (!seqs && n > c->seqs) return CB_ERR_SHAPE;
  // no rows: their pointers may be null (an empty tensor's is)
  const bool none = layers == 0 || n == 0 || max_count == 0;
  if (!stride || (!none && (!k || !v))) return CB_ERR_NULL;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(seqs, 4) || !aligned(start, 4) ||
      !aligned(counts, 4))
    return CB_ERR_ALIGN;
  const int64_t size[4] = {layers, n, c->kv_heads, max_count};
  st = check_strides(stride, size, 4, dtype == CB_F32 ? 4 : 2, output);
  if (st != CB_OK) return st;
  // a thread for eight values
  const int64_t units = (int64_t)layers * n * c->kv_heads;
  if (units > 0 && max_count > (cb::kMaxThreads - 255) / (c->head_dim / 8) / units)
    return CB_ERR_SHAPE;
  a->k = k;
  a->v = v;
  a->seqs = seqs;
  a->start = start;
  a->counts = counts;
  for (int i = 0; i < 4; ++i) a->stride[i] = stride[i];
  a->max_count = max_count;
  a->layer0 = layer0;
  a->layers = layers;
  a->n = n;
  return CB_OK;
}

}  // namespace

extern "C" {

int cb_rotary_frequencies(const cb_rope* r, double* freq, double* amplitude) {
  if (!r || !freq) return CB_ERR_NULL;
  const int R = r->rotary_dim;
  if (R < 2 || R > 1024 || R % 2 != 0) return CB_ERR_SHAPE;
  if (!(r->base > 1.0) || !isfinite(r->base)) return CB_ERR_SHAPE;
  if (r->scaling != CB_ROPE_NONE && r->scaling != CB_ROPE_LINEAR && r->scaling != CB_ROPE_YARN)
    return CB_ERR_SHAPE;
  const double tau = 2.0 * 3.14159265358979323846;
  double factor = 1.0, lo = 0.0, hi = 0.0;
  if (r->scaling != CB_ROPE_NONE) {
    factor = r->factor;
    if (!(factor >= 1.0) || !isfinite(factor)) return CB_ERR_SHAPE;
  }
  if (r->scaling == CB_ROPE_YARN) {
    const double fast = r->fast_turns == 0.0 ? 32.0 : r->fast_turns;
    const double slow = r->slow_turns == 0.0 ? 1.0 : r->slow_turns;
    if (!(r->original_len >= 1.0) || !isfinite(r->original_len) || !(slow > 0.0) ||
        !(fast >= slow) || !isfinite(fast))
      return CB_ERR_SHAPE;
    // the pair that makes t turns over the original length: base^(-2i/R) L / tau = t
    lo = floor(R * log(r->original_len / (fast * tau)) / (2.0 * log(r->base)));
    hi = ceil(R * log(r->original_len / (slow * tau)) / (2.0 * log(r->base)));
    lo = lo < 0.0 ? 0.0 : lo;
    hi = hi > R - 1.0 ? R - 1.0 : hi;
  }
  const double span = hi - lo > 1e-3 ? hi - lo : 1e-3;
  for (int i = 0; i < R / 2; ++i) {
    const double f = pow(r->base, -2.0 * i / R) / tau;
    double slowed = r->scaling == CB_ROPE_LINEAR ? 1.0 : 0.0;
    if (r->scaling == CB_ROPE_YARN) {
      slowed = (i - lo) / span;
      slowed = slowed < 0.0 ? 0.0 : slowed > 1.0 ? 1.0 : slowed;
    }
    freq[i] = f / factor * slowed + f * (1.0 - slowed);
  }
  if (amplitude) *amplitude = r->scaling == CB_ROPE_YARN ? 0.1 * log(factor) + 1.0 : 1.0;
  return CB_OK;
}

int cb_rotary(const cb_rows* rows, int32_t parts, int32_t head_dim, const double* freq,
              int32_t rotary_dim, double amplitude, int32_t interleaved, int32_t transpose,
              int32_t dtype, void* stream) {
  if (!rows || !freq) return CB_ERR_NULL;
  if (parts < 1 || parts > 2) return CB_ERR_SHAPE;
  if (dtype != CB_F32 && dtype != CB_BF16) return CB_ERR_DTYPE;
  if (head_dim < 8 || head_dim > 1024 || head_dim % 8 != 0 || rotary_dim < 2 ||
      rotary_dim > head_dim || rotary_dim % 2 != 0 || !isfinite((float)amplitude))
    return CB_ERR_SHAPE;
  if (!aligned(freq, 8)) return CB_ERR_ALIGN;
  const int es = dtype == CB_F32 ? 4 : 2;
  cb::RotaryArgs a{};
  for (int i = 0; i < parts; ++i) {
    const cb_rows& r = rows[i];
    int64_t total = 1;   // of rows, at most 2^40; compared by division, as the product may pass 64 bits
    for (int d = 0; d < 3; ++d) {
      if (r.size[d] < 0 || r.size[d] > 0x7fffffff) return CB_ERR_SHAPE;
      const int64_t size = r.size[d] ? r.size[d] : 1;
      if (size > ((int64_t)1 << 40) / total) return CB_ERR_SHAPE;
      total *= size;
    }
    // a thread for eight values of the rows of one head, workgroups of whole rows at least half full
    if (r.size[2] > (cb::kMaxThreads - 255) / (2 * (head_dim / 8 + 1))) return CB_ERR_SHAPE;
    const bool none = r.size[0] == 0 || r.size[1] == 0 || r.size[2] == 0;
    if (!none && (!r.in || !r.out || !r.pos)) return CB_ERR_NULL;
    if (!aligned(r.in, 16) || !aligned(r.out, 16) || !aligned(r.pos, 4) || !aligned(r.from, 4))
      return CB_ERR_ALIGN;
    int st = check_strides(r.in_stride, r.size, 3, es, false);
    if (st != CB_OK) return st;
    st = check_strides(r.out_stride, r.size, 3, es, true);
    if (st != CB_OK) return st;
    cb::RotaryPart& p = a.part[i];
    p.in = r.in;
    p.out = r.out;
    p.pos = r.pos;
    p.from = r.from;
    for (int d = 0; d < 3; ++d) {
      p.size[d] = r.size[d];
      p.in_stride[d] = r.in_stride[d];
      p.out_stride[d] = r.out_stride[d];
      p.pos_stride[d] = r.pos_stride[d];
      p.from_stride[d] = r.from_stride[d];
    }
  }
  a.freq = freq;
  a.amplitude = (float)amplitude;
  a.sign = transpose ? -1.f : 1.f;
  a.D = head_dim;
  a.R = rotary_dim;
  return done(cb::launch_rotary(a, parts, interleaved != 0, dtype == CB_F32,
                                static_cast<hipStream_t>(stream)));
}

size_t cb_cache_page_bytes(const cb_cache* c) {
  if (!c || !sizes_ok(c)) return 0;
  return (size_t)c->layers * c->kv_heads * c->page_len * (c->head_dim + c->head_dim / 16);
}

int cb_cache_status(const int32_t* status, void* stream) {
  if (!status) return CB_ERR_NULL;
  if (!aligned(status, 4)) return CB_ERR_ALIGN;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  int32_t word = 0;
  if (hipStreamSynchronize(s) != hipSuccess) return CB_ERR_HIP;
  if (hipMemcpy(&word, status, sizeof word, hipMemcpyDeviceToHost) != hipSuccess) return CB_ERR_HIP;
  return word == 0 ? CB_OK : word > 0 ? CB_ERR_PAGES : CB_ERR_SHAPE;
}

int cb_cache_extend(const cb_cache* c, const int32_t* seqs, const int32_t* add, int32_t n,
                    int32_t* status, void* stream) {
  cb::CacheView v;
  const int st = view_of(c, &v);
  if (st != CB_OK) return st;
  if (!entries_ok(n)) return CB_ERR_SHAPE;
  if (!status || (n > 0 && (!seqs || !add))) return CB_ERR_NULL;
  if (!aligned(seqs, 4) || !aligned(add, 4) || !aligned(status, 4)) return CB_ERR_ALIGN;
  return done(cb::launch_cache_extend(v, seqs, add, n, status, static_cast<hipStream_t>(stream)));
}

int cb_cache_free(const cb_cache* c, const int32_t* seqs, int32_t n, void* stream) {
  cb::CacheView v;
  const int st = view_of(c, &v);
  if (st != CB_OK) return st;
  if (n < 0 || n > cb::kMaxThreads / 256) return CB_ERR_SHAPE;
  if (n > 0 && !seqs) return CB_ERR_NULL;
  if (!aligned(seqs, 4)) return CB_ERR_ALIGN;
  return done(cb::launch_cache_free(v, seqs, n, static_cast<hipStream_t>(stream)));
}

size_t cb_cache_fork_workspace_bytes(const cb_cache* c, int32_t n) {
  if (!c || !sizes_ok(c) || !entries_ok(n)) return 0;
  return cb::cache_fork_ws(n, c->width);
}

int cb_cache_fork(const cb_cache* c, const int32_t* parents, const int32_t* children, int32_t n,
                  int32_t copy, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
  cb::CacheView v;
  const int st = view_of(c, &v);
  if (st != CB_OK) return st;
  if (!entries_ok(n)) return CB_ERR_SHAPE;
  if (!status || (n > 0 && (!parents || !children))) return CB_ERR_NULL;
  if (!ws || ws_bytes < cb::cache_fork_ws(n, c->width)) return CB_ERR_WORKSPACE;
  if (!aligned(parents, 4) || !aligned(children, 4) || !aligned(status, 4) || !aligned(ws, 16))
    return CB_ERR_ALIGN;
  return done(cb::launch_cache_fork(v, parents, children, n, copy != 0, status, ws,
                                    static_cast<hipStream_t>(stream)));
}

size_t cb_cache_compact_workspace_bytes(const cb_cache* c, int32_t n) {
  if (!c || !sizes_ok(c) || !entries_ok(n)) return 0;
  return cb::cache_compact_ws(n, c->width);
}

int cb_cache_compact(const cb_cache* c, const int32_t* src, const int32_t* dst, int32_t n,
                     const int32_t* idx, const int64_t idx_stride[3], int64_t keep,
                     const int32_t* counts, int32_t* status, void* ws, size_t ws_bytes,
                     void* stream) {
  cb::CacheCompactArgs a{};
  const int st = view_of(c, &a.c);
  if (st != CB_OK) return st;
  if (!entries_ok(n) || keep < 1 || keep > (int64_t)c->width * c->page_len) return CB_ERR_SHAPE;
  if (!idx_stride || !status || (n > 0 && (!src || !dst || !idx))) return CB_ERR_NULL;
  if (!ws || ws_bytes < cb::cache_compact_ws(n, c->width)) return CB_ERR_WORKSPACE;
  if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(idx, 4) || !aligned(counts, 4) ||
      !aligned(status, 4) || !aligned(ws, 16))
    return CB_ERR_ALIGN;
  a.src = src;
  a.dst = dst;
  a.idx = idx;
  a.counts = counts;
  for (int i = 0; i < 3; ++i) a.idx_stride[i] = idx_stride[i];
  a.keep = keep;
  a.n = n;
  a.status = status;
  a.old_rows = static_cast<int32_t*>(ws);
  return done(cb::launch_cache_compact(a, static_cast<hipStream_t>(stream)));
}

int cb_cache_write(const cb_cache* c, int32_t layer0, int32_t layers, const int32_t* seqs,
                   int32_t n, const int32_t* start, const int32_t* counts, int64_t max_count,
                   const void* k, const void* v, const int64_t stride[4], int32_t dtype,
                   void* stream) {
  cb::CacheRowsArgs a{};
  const int st = rows_args(c, layer0, layers, seqs, n, start, counts, max_count, k, v, stride,
                           dtype, false, &a);
  if (st != CB_OK) return st;
  return done(cb::launch_cache_write(a, dtype == CB_F32, static_cast<hipStream_t>(stream)));
}

int cb_cache_read(const cb_cache* c, int32_t layer0, int32_t layers, const int32_t* seqs,
                  int32_t n, const int32_t* start, const int32_t* counts, int64_t max_count,
                  void* k, void* v, const int64_t stride[4], int32_t dtype, void* stream) {
  cb::CacheRowsArgs a{};
  const int st = rows_args(c, layer0, layers, seqs, n, start, counts, max_count, k, v, stride,
                           dtype, true, &a);
  if (st != CB_OK) return st;
  return done(cb::launch_cache_read(a, dtype == CB_F32, static_cast<hipStream_t>(stream)));
}

// Checks shared by the size query and the call.
static int attend_plan(const cb_cache* c, int32_t layers, int32_t n, int32_t q_heads, int64_t q_len,
                       int64_t longest, int32_t dtype, cb::AttendPlan* p) {
  if (!c) return CB_ERR_NULL;
  if (!sizes_ok(c) || layers < 0 || layers > c->layers || n < 0 || n > (1 << 20) || q_heads < 1 ||
      q_heads % c->kv_heads != 0 || q_len < 0 || q_len > (1 << 26) || longest < 0)
    return CB_ERR_SHAPE;
  if (dtype != CB_F32 && dtype != CB_BF16) return CB_ERR_DTYPE;
  if (layers == 0 || n == 0 || q_len == 0) {
    *p = cb::AttendPlan{};
    return CB_OK;
  }
  const int64_t room = (int64_t)c->width * c->page_len;
  return cb::make_attend_plan(layers, n, c->kv_heads, q_heads, q_len, c->head_dim, dtype == CB_F32,
                              longest > 0 && longest < room ? longest : room, p)
             ? CB_OK
             : CB_ERR_SHAPE;
}

size_t cb_cache_attend_workspace_bytes(const cb_cache* c, int32_t layers, int32_t n,
                                       int32_t q_heads, int64_t q_len, int64_t longest) {
  cb::AttendPlan p;
  size_t most = 0;   // of either dtype
  for (int dtype : {CB_F32, CB_BF16})
    if (attend_plan(c, layers, n, q_heads, q_len, longest, dtype, &p) == CB_OK && p.total > most)
      most = p.total;
  return most;
}

int cb_cache_attend(const cb_cache* c, int32_t layer0, int32_t layers, const int32_t* seqs,
                    int32_t n, const void* q, const int64_t q_stride[4], int32_t q_heads,
                    const int32_t* q_lens, int64_t q_len, int32_t causal, int64_t longest,
                    double scale, void* out, const int64_t out_stride[4], float* lse, int32_t dtype, void* ws,
                    size_t ws_bytes, void* stream) {
  cb::AttendArgs a{};
  int st = view_of(c, &a.c);
  if (st != CB_OK) return st;
  st = layers_ok(c, layer0, layers, n);
  if (st != CB_OK) return st;
  cb::AttendPlan p;
  st = attend_plan(c, layers, n, q_heads, q_len, longest, dtype, &p);
  if (st != CB_OK) return st;
  if (!seqs && n > c->seqs) return CB_ERR_SHAPE;
  const double c2 = (scale == 0.0 ? 1.0 / sqrt((double)c->head_dim) : scale) * 1.4426950408889634;
  if (!(scale >= 0.0) || !isfinite((float)c2)) return CB_ERR_SHAPE;
  const bool none = layers == 0 || n == 0 || q_len == 0;
  if (!q_stride || !out_stride || (!none && (!q || !out))) return CB_ERR_NULL;
  if (p.total > 0 && (!ws || ws_bytes < p.total)) return CB_ERR_WORKSPACE;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(seqs, 4) ||
      !aligned(q_lens, 4) || !aligned(ws, 16))
    return CB_ERR_ALIGN;
  const int64_t size[4] = {layers, n, q_heads, q_len};
  const int es = dtype == CB_F32 ? 4 : 2;
  st = check_strides(q_stride, size, 4, es, false);
  if (st != CB_OK) return st;
  st = check_strides(out_stride, size, 4, es, true);
  if (st != CB_OK) return st;
  if (none) return CB_OK;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.seqs = seqs;
  a.q_lens = q_lens;
  unsigned char* w = static_cast<unsigned char*>(ws);
  a.part_o = reinterpret_cast<float*>(w);
  a.part_ml = reinterpret_cast<float2*>(w + (p.total ? p.off_ml : 0));
  for (int i = 0; i < 4; ++i) {
    a.q_stride[i] = q_stride[i];
    a.out_stride[i] = out_stride[i];
  }
  a.q_len = q_len;
  a.layer0 = layer0;
  a.layers = layers;
  a.n = n;
  a.q_heads = q_heads;
  a.group = q_heads / c->kv_heads;
  a.recip = a.group == 1 ? 0xffffffffu : (uint32_t)(((uint64_t)1 << 32) / (uint32_t)a.group);
  a.row_tiles = p.row_tiles;
  a.rows_pad = p.rows_pad;
  a.target = p.target;
  a.whole = p.whole;
  a.slots = p.slots;
  a.room = p.room;
  a.causal = causal != 0;
  a.c2 = fmaxf((float)c2, 1e-37f);   // never 0: a masked logit is -inf times it
  return done(cb::launch_cache_attend(a, p, dtype == CB_F32, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
