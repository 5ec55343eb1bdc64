/*
 * cacheback_cache.h -- C ABI of the receiver's side of a message on MI355X:
 * rotary positions, a paged key/value cache held in four bits, its pages, and
 * attention over it.
 *
 * The selection path of cacheback.h ends with the rows a sender kept.  Here
 * the receiver places their keys at new positions (section 3.1.2, Appendix
 * C.3: selected state enters the receiver at new positions), holds them in
 * pages, lets several answers draw from one message, ranks and thins it again
 * along a chain (Appendix C.2, chain budgets), and attends to it.
 *
 * The conventions of cacheback.h hold: device pointers on the current device,
 * work enqueued on `stream`, no call synchronises, allocates or keeps a
 * pointer, argument errors launch nothing and return a negative CB_ERR_* code.
 * Calls are captured into HIP graphs as any kernel launch is.  Two calls that
 * use the same scratch `ws`, or change the same cache, must not overlap in time.
 *
 * Strided tensors: row strides are given in elements, outermost first; the D
 * values of a row are contiguous, and every row starts on a 16-byte boundary
 * (pointers and strides; CB_ERR_ALIGN otherwise).  A size of zero launches
 * nothing but what writes a call's status.  Outputs must not overlap inputs unless a
 * call says so.  Sizes that pass
 * the limits named at a call, or one launch's (2^32 - 1 threads along an axis: eight
 * values a thread for rows, 16 to 64 query rows a workgroup for attention), give
 * CB_ERR_SHAPE.
 */
#ifndef CACHEBACK_CACHE_H
#define CACHEBACK_CACHE_H

#include "cacheback.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Rotary positions ---------------------------------------------------- */

typedef enum { CB_ROPE_NONE = 0, CB_ROPE_LINEAR = 1, CB_ROPE_YARN = 2 } cb_rope_scaling;

typedef struct cb_rope {
  int32_t rotary_dim;   /* R: rotated values of a row, even, 2..1024 */
  int32_t scaling;      /* cb_rope_scaling */
  double base;          /* > 1 */
  double factor;        /* >= 1; how far the context is stretched */
  double original_len;  /* YaRN: positions of the original context, >= 1 */
  double fast_turns;    /* YaRN: pairs of this many turns and more stay; 0: 32 */
  double slow_turns;    /* YaRN: pairs of this many and fewer slow down; 0: 1 */
} cb_rope;

/* Host-only.  freq[i], i < R/2, receives the turns (of 2 pi) per position of
 * pair i, in 64 bits, and *amplitude (nullable) the factor on sines and cosines:
 *   none    f_i = base^(-2i/R) / (2 pi)
 *   linear  f_i / factor
 *   YaRN    f_i (1 - s_i + s_i / factor), s_i = clamp((i - lo) / (hi - lo), 0, 1),
 *           lo and hi the pairs (rounded outwards, within 0..R-1) that make
 *           fast_turns and slow_turns over original_len positions;
 *           amplitude 0.1 ln(factor) + 1
 * CB_ERR_SHAPE for values outside the ranges above or not finite. */
int cb_rotary_frequencies(const cb_rope* rope, double* freq, double* amplitude);

/* Rows of one tensor, [size0][size1][size2][D]: any strides, in place
 * when `out` = `in` with the same strides.  pos (and from): int32, with strides of
 * their own in entries (0 repeats a position along an axis). */
typedef struct cb_rows {
  const void* in;
  void* out;
  const int32_t* pos;
  const int32_t* from;     /* nullable: zero */
  int64_t size[3];
  int64_t in_stride[3], out_stride[3];
  int64_t pos_stride[3], from_stride[3];
} cb_rows;

/* Rotates the first R = rotary_dim values of every row of `parts` tensors (1
 * or 2: a step's queries and keys go in one call) by the angles
 *   phi_i = 2 pi frac(freq[i] * (pos - from)),
 * `from` being the position that a cached key was rotated to before (a kept
 * key that moves: pass amplitude 1), each pair (x, y) becoming
 *   amplitude * (x cos phi - y sin phi, y cos phi + x sin phi).
 * Pair i is (v[i], v[i + R/2]), or (v[2i], v[2i+1]) if interleaved.  Values
 * from R on are copied.  transpose != 0 rotates by -phi: the gradient of the
 * input given the gradient of the output.  freq: device, R/2 doubles, 8-byte
 * aligned.  Angles are formed in 64 bits, rotations in fp32, each value
 * rounded once to dtype (CB_F32, CB_BF16).  D = head_dim: a multiple of 8,
 * 8..1024, R even, 2..D.  A tensor has at most 2^40 rows.  Rows of an output must not
 * overlap one another. */
int cb_rotary(const cb_rows* rows, int32_t parts, int32_t head_dim, const double* freq,
              int32_t rotary_dim, double amplitude, int32_t interleaved, int32_t transpose,
              int32_t dtype, void* stream);

/* ---- The cache ------------------------------------------------------------
 *
 * Four bits a value: the 32 values of a group (consecutive in a row) share a
 * scale 2^e, stored as the byte e + 127, e the least with max|x| <= 7 * 2^e,
 * clamped to -124..125; a value is held as the nearest of 0, 0.5, 1, 1.5, 2,
 * 3, 4, 6 times the scale (ties to the even code, larger ones to 6) and its
 * sign: bit 3 of the code.  What a code stands for is exact in bf16.  A group
 * with a NaN or an infinity gets the byte 255, and all of it reads as NaN.  The bytes
 * 253 and 254 are never stored: what a group that holds one, in a page's unwritten
 * positions say, reads as is not defined (its values, infinities or NaN).
 *
 * pool  [pages][layers][kv_heads][unit] bytes, unit = P * (D + D/16) for the
 *       P = page_len positions of a page:
 *         key codes    [P][D/2]          even value of a pair in the low half
 *         value codes  [P/4][16][4][D/32]  16 runs of D/16 values, of 4 positions
 *         key scales   [P][D/32]
 *         value scales [P/4][D/32][4]
 * refs  [pages]        how many sequences hold the page; 0: free
 * table [seqs][width]  pages of a sequence in order, -1 behind the last
 * lens  [seqs]         positions of a sequence; it holds ceil(len / P) pages
 *
 * Start: refs and lens zero, table -1; the pool may hold anything.  A page
 * that several sequences hold is never written by cb_cache_extend, _fork,
 * _compact or _free; cb_cache_write writes where it is told.
 */
typedef struct cb_cache {
  int32_t layers, kv_heads;   /* 1..4096 each */
  int32_t head_dim;   /* D: 64 or 128 */
  int32_t page_len;   /* P: 16, 32, 64, 128 or 256 */
  int32_t pages;      /* 1..2^24 */
  int32_t seqs;       /* 1..2^17 */
  int32_t width;      /* >= 1; width * page_len <= 2^31 - 2^16 */
  int32_t reserved;   /* 0 */
  void* pool;         /* 16-byte aligned, like the others */
  int32_t* refs;
  int32_t* table;
  int32_t* lens;
} cb_cache;

/* Bytes of one page (all layers and heads); 0 for invalid sizes. */
size_t cb_cache_page_bytes(const cb_cache* c);

/* The lists of sequences below (seqs, parents, ...) are device int32 arrays
 * of n entries.  Where a call says "all or nothing", *status (device,
 * 4-byte aligned) receives 0 when it was done, the number of pages lacking, or
 * -1 for an invalid entry; unless it is 0 the cache is as it was before.  A call
 * says what became of it alone, over whatever *status held: calls that rest on one
 * another (a fork of what was extended) want a word each, or a look between them.
 * New pages are the free pages of lowest number, in the order of the entries. */

/* Synchronises `stream` and says what *status holds: CB_OK, CB_ERR_PAGES, or
 * CB_ERR_SHAPE for an invalid entry. */
int cb_cache_status(const int32_t* status, void* stream);

/* Room for add[i] (>= 0) more positions behind those of sequence seqs[i]:
 * takes the pages they need and adds add[i] to its length.  All or nothing;
 * invalid: a sequence outside the table or listed twice, add[i] < 0, a length
 * over width * page_len.  One workgroup; n <= 2048. */
int cb_cache_extend(const cb_cache* c, const int32_t* seqs, const int32_t* add, int32_t n,
                    int32_t* status, void* stream);

/* Gives back the pages of the sequences: their lengths become 0 and their
 * table rows -1.  Entries outside the table are passed over, and so is an
 * entry listed again.  n < 2^24. */
int cb_cache_free(const cb_cache* c, const int32_t* seqs, int32_t n, void* stream);

/* children[i] becomes a sequence with the positions of parents[i]: it holds
 * the same full pages and a copy of the page that the last positions fill in
 * part (so that each side can append); copy != 0: a copy of every page.  Pages
 * that a child held before are given back first.  All or nothing; invalid: an
 * entry outside the table, a child listed twice or that is also a parent, a parent
 * whose table row does not name a page for each of its positions.
 * n <= 2048.  ws: cb_cache_fork_workspace_bytes(c, n) bytes, 16-byte aligned. */
size_t cb_cache_fork_workspace_bytes(const cb_cache* c, int32_t n);
int cb_cache_fork(const cb_cache* c, const int32_t* parents, const int32_t* children, int32_t n,
                  int32_t copy, int32_t* status, void* ws, size_t ws_bytes, void* stream);

/* Keeps selected positions: dst[i] becomes a sequence of counts[i] positions
 * (NULL: keep), in new pages, position j of layer l and head h being position
 *   idx[i * idx_stride[0] + l * idx_stride[1] + h * idx_stride[2] + j]
 * of src[i] in that layer and head: codes and scales are moved as they are
 * (strides of 0 use one list for all layers or heads).  A position outside the
 * sequence, or without a page, gives a row of zeros.  dst[i] = src[i] thins a
 * sequence itself; pages that dst[i] held before are given back.  The rest of the
 * last page is cleared.
 * All or nothing; invalid: an entry outside the table, a dst listed twice or
 * that is the src of another entry, a count below 0 or over keep.
 * 1 <= keep <= width * page_len, n <= 2048. */
size_t cb_cache_compact_workspace_bytes(const cb_cache* c, int32_t n);
int cb_cache_compact(const cb_cache* c, const int32_t* src, const int32_t* dst, int32_t n,
                     const int32_t* idx, const int64_t idx_stride[3], int64_t keep,
                     const int32_t* counts, int32_t* status, void* ws, size_t ws_bytes,
                     void* stream);

/* Rows into the cache.  k, v: [layers][n][kv_heads][max_count][D] with the
 * strides of the first four axes, dtype CB_F32 or CB_BF16, for layers
 * layer0..layer0+layers-1.  Row t < counts[i] (NULL: max_count) goes to
 * position start[i] + t of sequence seqs[i] (NULL: sequence i); start = NULL:
 * the sequence's last counts[i] positions.  A row whose position has no page
 * is passed over.  counts[i] below 0 is taken as 0, above max_count as max_count.  No
 * position may be written twice in a call. */
int cb_cache_write(const cb_cache* c, int32_t layer0, int32_t layers, const int32_t* seqs,
                   int32_t n, const int32_t* start, const int32_t* counts, int64_t max_count,
                   const void* k, const void* v, const int64_t stride[4], int32_t dtype,
                   void* stream);

/* The values that the cache's positions stand for: the same arguments, k and v
 * being outputs.  Exact in either dtype.  A position outside the sequence, or without a
 * page, gives a row of zeros; rows t >= counts[i] are left as they are. */
int cb_cache_read(const cb_cache* c, int32_t layer0, int32_t layers, const int32_t* seqs,
                  int32_t n, const int32_t* start, const int32_t* counts, int64_t max_count,
                  void* k, void* v, const int64_t stride[4], int32_t dtype, void* stream);

/* Attention of query rows over the cache.  q, out: [layers][n][q_heads][q_len][D]
 * with the strides of the first four axes.  For query token r < q_lens[i]
 * (NULL: q_len) of row i, sequence seqs[i] (NULL: i) of length len:
 *   out = sum_t p_t V[t],  p = softmax over t < limit of scale * q . K[t],
 * limit = len, or if causal len - q_lens[i] + r + 1 (the query tokens are the
 * sequence's last).  Positions from limit on count for nothing, whatever they
 * hold.  A row with limit <= 0 gives zeros; query tokens from q_lens[i] on are
 * left as they are.  lse (nullable) [layers][n][q_heads][q_len] fp32:
 * ln sum_t exp(scale * q . K[t]), -inf for a row of no position.  scale: >= 0,
 * 0 selects 1/sqrt(D).  q_lens[i] below 0 is taken as 0, above q_len as q_len.
 * dtype of q and out: CB_F32 or CB_BF16; logits, statistics and sums in fp32.  The
 * weights enter the product with V in 24 bits with CB_F32.  With CB_BF16 they enter in
 * 16 bits where q_len * q_heads / kv_heads is at most 16, and for more query rows in 16
 * or in 8 (each off by at most 2^-8 of itself).  A position without a page counts for
 * nothing.  Logits within +-2^28 and values within +-2^60
 * give finite rows; a row that sees larger ones may come out infinite or NaN.
 * longest: what the caller knows of the lengths: sequences longer than this are
 * taken to be this long (0: as long as the table allows).  Short sequences in a
 * wide table are faster with it: none is cut, and no results are joined.  n times
 * its multiples of 128 positions have to stay below 2^31, n is at most 2^20, and q_len and
 * the query rows of a KV head, q_len * q_heads / kv_heads, at most 2^26 (CB_ERR_SHAPE).
 * ws: cb_cache_attend_workspace_bytes bytes (same `longest`), 16-byte aligned;
 * its contents need not be initialised (0 bytes: no scratch is needed, or the call refuses
 * the sizes).  Deterministic.  At most two kernels. */
size_t cb_cache_attend_workspace_bytes(const cb_cache* c, int32_t layers, int32_t n,
                                       int32_t q_heads, int64_t q_len, int64_t longest);
int cb_cache_attend(const cb_cache* c, int32_t layer0, int32_t layers, const int32_t* seqs,
                    int32_t n, const void* q, const int64_t q_stride[4], int32_t q_heads,
                    const int32_t* q_lens, int64_t q_len, int32_t causal, int64_t longest,
                    double scale, void* out, const int64_t out_stride[4], float* lse, int32_t dtype, void* ws,
                    size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CACHEBACK_CACHE_H */
