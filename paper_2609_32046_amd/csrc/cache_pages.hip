// Pages of the four-bit cache (gfx950): taking, sharing, copying, thinning and
// giving back.
//
// The free list is the reference counts themselves: a page of no holder is
// free, and the lowest free ones are taken first.  So there is one state to keep
// right, and every call's outcome is a function of it.  A call that takes pages
// plans in one workgroup (it checks every entry before it changes anything,
// and takes back what it released when pages lack), then moves bytes with the
// whole device.  A plan is a chain of reads that wait for one another (list, length, row, count):
// 5 us to extend 64 sequences, 10 to fork 64 children of 32 pages, 7-8 to compact; giving
// back 64 sequences takes 5.
#include "cache.h"

namespace cb {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kPlan = 1024;         // threads of a planning workgroup
constexpr int kPlanWaves = kPlan / 64;
constexpr int kScan = 16;           // reads of refs a thread has under way
constexpr int kItems = 4;           // pages of rows a thread has under way

__device__ inline int held_pages(const CacheView& c, int len) {
  const int64_t n = ((int64_t)(len > 0 ? len : 0) + (1 << c.page_shift) - 1) >> c.page_shift;
  return n < c.width ? (int)n : c.width;
}

__device__ inline bool known(const CacheView& c, int seq) {
  return (unsigned)seq < (unsigned)c.seqs;
}

// Inclusive sum over the lanes up to this one.
template <typename I>
__device__ inline I wave_scan(I x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const I y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Exclusive prefix of x over the workgroup, and the total, in 64 bits: the rows of a thousand
// sequences can hold more than 2^31 pages.  `sums`: kPlanWaves words; two barriers.
__device__ inline int64_t group_scan(int64_t x, int64_t* sums, int64_t* total) {
  const int wave = threadIdx.x >> 6;
  const int64_t incl = wave_scan(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sums[wave] = incl;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int64_t v = sums[w];
    before += w < wave ? v : 0;
    all += v;
  }
  *total = all;
  return before + incl - x;
}

// Bit set of sequences in LDS; true when the bit was set before.
__device__ inline bool mark(uint32_t* bits, int seq) {
  const uint32_t b = 1u << (seq & 31);
  return (atomicOr(&bits[seq >> 5], b) & b) != 0;
}
__device__ inline bool marked(const uint32_t* bits, int seq) {
  return (bits[seq >> 5] >> (seq & 31)) & 1u;
}

// A list of sequences with their lengths, in LDS: the rows' pages are then one read away.
struct SeqList {
  int seq[kCacheMaxEntries];
  int len[kCacheMaxEntries];
  int most;   // pages of the longest
};

struct PlanShared {
  int64_t sums[kPlanWaves];
  int rows[kScan * kPlanWaves];
  int free;
  int bad;
  int offset[kCacheMaxEntries + 1];   // pages that the entries before need
};

// Fills N lists (a barrier follows), their reads side by side; entries outside the table get no
// pages.  Returns whether one of this thread's is outside.
template <int N>
__device__ inline bool fill_lists(const CacheView& c, SeqList* const (&l)[N],
                                  const int32_t* const (&seqs)[N], int n) {
  bool bad = false;
  int most[N] = {};
  for (int i = threadIdx.x; i < n; i += kPlan) {
    int s[N], len[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = seqs[k][i];
#pragma unroll
    for (int k = 0; k < N; ++k) len[k] = known(c, s[k]) ? c.lens[s[k]] : 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      bad |= !known(c, s[k]) || len[k] < 0;
      l[k]->seq[i] = s[k];
      l[k]->len[i] = len[k];
      const int p = held_pages(c, len[k]);
      most[k] = p > most[k] ? p : most[k];
    }
  }
  // one lane a wave: the compiler would walk the lanes for an atomic of them all (2 us for 64)
  if ((int)(threadIdx.x & ~63u) < n) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_xor(most[k], d);
        most[k] = o > most[k] ? o : most[k];
      }
      if ((threadIdx.x & 63) == 0) atomicMax(&l[k]->most, most[k]);
    }
  }
  return bad;
}

// Gives a page back; a count that was zero (a page listed by mistake) stays.
__device__ inline void drop(int32_t* refs, int page) {
  if (atomicSub(&refs[page], 1) <= 0) atomicAdd(&refs[page], 1);
}

// Offsets of the entries' needs, need(i) pages each; returns the total.
template <typename Need>
__device__ inline int64_t plan_offsets(PlanShared& sh, int n, Need need) {
  if (n <= 64) {   // one wave's work, and one barrier
    if (threadIdx.x < 64) {
      const int i = threadIdx.x;
      const int64_t mine = i < n ? need(i) : 0, incl = wave_scan(mine);
      if (i < n) sh.offset[i] = incl - mine > kCacheMaxPages ? kCacheMaxPages + 1 : (int)(incl - mine);
      if (i == 63) {
        sh.offset[n] = incl > kCacheMaxPages ? kCacheMaxPages + 1 : (int)incl;
        sh.sums[0] = incl;
      }
    }
    __syncthreads();
    return sh.sums[0];
  }
  int64_t base = 0;
  for (int i0 = 0; i0 < n; i0 += kPlan) {
    const int i = i0 + threadIdx.x;
    int64_t total;
    const int64_t at = base + group_scan(i < n ? need(i) : 0, sh.sums, &total);
    if (i < n) sh.offset[i] = at > kCacheMaxPages ? kCacheMaxPages + 1 : (int)at;
    base += total;
  }
  if (threadIdx.x == 0) sh.offset[n] = base > kCacheMaxPages ? kCacheMaxPages + 1 : (int)base;
  __syncthreads();
  return base;
}

// One sweep over kScan rows of kPlan pages, a page of each row to a thread: free pages
// that lie together, as the lowest do, then fall to different threads, which
// enter them in their rows at the same time.
struct Sweep {
  uint32_t free;   // bit j: this thread's page of row j is free
  int64_t p0;
  // Ranks within the sweep go through sh.rows; returns how many pages are free.
  __device__ int load(const CacheView& c, PlanShared& sh, int64_t from) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    p0 = from + threadIdx.x;
    int r[kScan];
#pragma unroll
    for (int j = 0; j < kScan; ++j)
      r[j] = p0 + j * kPlan < c.pages ? c.refs[p0 + j * kPlan] : 1;
    free = 0;
    __syncthreads();   // the last sweep's ranks have been read
#pragma unroll
    for (int j = 0; j < kScan; ++j) {
      free |= r[j] == 0 ? 1u << j : 0u;
      const uint64_t b = __ballot(r[j] == 0);
      if (lane == 0) sh.rows[j * kPlanWaves + wave] = __popcll(b);
    }
    __syncthreads();
    // exclusive prefixes of the kScan * kPlanWaves counts, by the first wave
    constexpr int kEach = kScan * kPlanWaves / 64;
    if (wave == 0) {
      int v[kEach], sum = 0;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        v[k] = sh.rows[lane * kEach + k];
        sum += v[k];
      }
      int at = wave_scan(sum) - sum;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        sh.rows[lane * kEach + k] = at;
        at += v[k];
      }
      if (lane == 63) sh.free = at;
    }
    __syncthreads();
    return sh.free;
  }
  // take(page, rank) for this thread's free pages of rank below want; base: free pages before
  // the sweep.
  template <typename Take>
  __device__ void give(const PlanShared& sh, int64_t base, int64_t want, Take take) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the wave's ranks in lanes 0..kScan-1; rows from the wanted ones on are passed over
    const int first = lane < kScan ? sh.rows[lane * kPlanWaves + wave] : 0;
    uint64_t todo = __ballot(lane < kScan && base + first < want);
#pragma unroll 1
    while (todo != 0) {
      const int j = __ffsll((unsigned long long)todo) - 1;
      todo &= todo - 1;
      const bool is = (free >> j) & 1u;
      const uint64_t b = __ballot(is);
      const int64_t rank =
          base + __builtin_amdgcn_readlane(first, j) + __popcll(b & ((1ull << lane) - 1));
      if (is && rank < want) take((int)(p0 + j * kPlan), (int)rank);
    }
  }
};

// Calls take(page, rank) for the `want` free pages of lowest number, ranks in order of
// their numbers, if there are so many; returns how many there are, at most want.  The
// workgroup's own changes to refs lie before its first barrier.
template <typename Take>
__device__ inline int64_t take_free(const CacheView& c, PlanShared& sh, int64_t want, Take take) {
  constexpr int kStep = kPlan * kScan;
  Sweep sw;
  int64_t base = sw.load(c, sh, 0);
  if (base >= want) {   // within the first sweep: no second look
    sw.give(sh, 0, want, take);
    return want;
  }
  int64_t p0 = kStep;
  for (; p0 < c.pages && base < want; p0 += kStep) base += sw.load(c, sh, p0);
  if (base < want) return base;
  const int64_t end = p0;
  base = 0;
  for (p0 = 0; p0 < end; p0 += kStep) {
    const int k = sw.load(c, sh, p0);
    sw.give(sh, base, want, take);
    base += k;
  }
  return want;
}

// Entry whose pages include rank r.
__device__ inline int entry_of(const PlanShared& sh, int n, int r) {
  int lo = 0, hi = n - 1;   // offset[lo] <= r < offset[hi + 1]
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sh.offset[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// What *status says where pages lack.
__device__ inline int lacking(int64_t k) { return (int)(k < 0x7fffffff ? k : 0x7fffffff); }

__device__ inline void clear_bits(uint32_t* bits, int seqs) {
  for (int i = threadIdx.x; i < (seqs + 31) / 32; i += kPlan) bits[i] = 0u;
}

// ---------------------------------------------------------------------------

__global__ __launch_bounds__(kPlan) void cache_extend_kernel(CacheView c,
                                                             const int32_t* __restrict__ seqs,
                                                             const int32_t* __restrict__ add,
                                                             int n, int32_t* status) {
  extern __shared__ uint32_t bits[];
  __shared__ PlanShared sh;
  __shared__ SeqList l;
  clear_bits(bits, c.seqs);
  if (threadIdx.x == 0) sh.bad = l.most = 0;
  __syncthreads();
  const int64_t room = (int64_t)c.width << c.page_shift;
  const int mine = (int)threadIdx.x < n ? add[threadIdx.x] : 0;   // under way beside the lists
  bool bad = fill_lists<1>(c, {&l}, {seqs}, n);
  for (int i = threadIdx.x; i < n; i += kPlan) {   // this thread's own entries
    const int more = i < kPlan ? mine : add[i];
    bad |= (known(c, l.seq[i]) && mark(bits, l.seq[i])) || more < 0 ||
           (int64_t)l.len[i] + more > room;
  }
  if (bad) sh.bad = 1;
  __syncthreads();
  if (sh.bad) {
    if (threadIdx.x == 0) *status = -1;
    return;
  }
  const int64_t want = plan_offsets(
      sh, n, [&](int i) {   // every thread asks for its own entries
        return held_pages(c, l.len[i] + (i < kPlan ? mine : add[i])) - held_pages(c, l.len[i]);
      });
  const int64_t have = take_free(c, sh, want, [&](int page, int rank) {
    const int i = entry_of(sh, n, rank);
    c.table[(int64_t)l.seq[i] * c.width + held_pages(c, l.len[i]) + rank - sh.offset[i]] = page;
    c.refs[page] = 1;
  });
  if (have < want) {
    if (threadIdx.x == 0) *status = lacking(want - have);
    return;
  }
  for (int i = threadIdx.x; i < n; i += kPlan)
    c.lens[l.seq[i]] = l.len[i] + (i < kPlan ? mine : add[i]);
  if (threadIdx.x == 0) *status = 0;
}

__global__ __launch_bounds__(256) void cache_free_kernel(CacheView c,
                                                         const int32_t* __restrict__ seqs) {
  const int s = seqs[blockIdx.x];
  if (!known(c, s)) return;
  __shared__ int len;
  if (threadIdx.x == 0) len = atomicExch(&c.lens[s], 0);   // an entry listed again finds 0
  __syncthreads();
  const int pages = held_pages(c, len);
  int32_t* row = c.table + (int64_t)s * c.width;
  for (int j = threadIdx.x; j < pages; j += 256) {
    const int p = row[j];
    row[j] = -1;
    if ((unsigned)p < (unsigned)c.pages) drop(c.refs, p);
  }
}

// f(i, j, page) for the pages j of the listed sequences' rows as they stand, kItems of
// them under way in every thread: a row is short, and a row at a time would be all latency.
template <typename F>
__device__ inline void each_page(const CacheView& c, const SeqList& l, int n, F f) {
  // a row's pages are dealt to the next power of two of threads, 16 to 1024
  int shift = 4;
  while ((1 << shift) < l.most && shift < 10) ++shift;
  const int lane = threadIdx.x & ((1 << shift) - 1);
  for (int j0 = 0; j0 < l.most; j0 += 1 << shift) {
    const int j = j0 + lane;
    for (int i0 = threadIdx.x >> shift; i0 < n; i0 += kItems * (kPlan >> shift)) {
      int page[kItems];
#pragma unroll
      for (int e = 0; e < kItems; ++e) {
        const int i = i0 + e * (kPlan >> shift);
        page[e] = i < n && j < held_pages(c, l.len[i]) ? c.table[(int64_t)l.seq[i] * c.width + j] : -1;
      }
#pragma unroll
      for (int e = 0; e < kItems; ++e) {
        const int i = i0 + e * (kPlan >> shift);
        if (i < n && j < held_pages(c, l.len[i])) f(i, j, page[e]);
      }
    }
  }
}

__device__ inline bool is_page(const CacheView& c, int p) { return (unsigned)p < (unsigned)c.pages; }

// ws of a fork: how many pages are copied (padded to 16 bytes), then (from, to).
__global__ __launch_bounds__(kPlan) void cache_fork_kernel(CacheView c,
                                                           const int32_t* __restrict__ parents,
                                                           const int32_t* __restrict__ children,
                                                           int n, int copy, int32_t* status,
                                                           int32_t* count, int2* pairs) {
  extern __shared__ uint32_t bits[];
  __shared__ PlanShared sh;
  __shared__ SeqList from, to;
  // A parent's row names what is no page.  Not sh.bad: a wave may find that out while
  // another still reads sh.bad for the entries.
  __shared__ int no_page;
  clear_bits(bits, c.seqs);
  if (threadIdx.x == 0) {
    sh.bad = no_page = from.most = to.most = 0;
    *count = 0;
  }
  __syncthreads();
  bool bad = fill_lists<2>(c, {&from, &to}, {parents, children}, n);
  for (int i = threadIdx.x; i < n; i += kPlan)   // this thread's own entries
    bad |= known(c, to.seq[i]) && mark(bits, to.seq[i]);
  if (bad) sh.bad = 1;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlan)
    if (known(c, from.seq[i]) && marked(bits, from.seq[i])) sh.bad = 1;
  __syncthreads();
  if (sh.bad) {
    if (threadIdx.x == 0) *status = -1;
    return;
  }
  // every page that a parent says it holds is one
  each_page(c, from, n, [&](int, int, int p) {
    if (!is_page(c, p)) no_page = 1;
  });
  auto hold = [&](int d) {   // the children's pages
    each_page(c, to, n, [&](int, int, int p) {
      if (is_page(c, p)) atomicAdd(&c.refs[p], d);
    });
  };
  hold(-1);
  const int part = (1 << c.page_shift) - 1;
  const int64_t want = plan_offsets(sh, n, [&](int i) {
    const int len = from.len[i];
    return copy ? held_pages(c, len) : (len > 0 && (len & part) != 0);
  });
  __syncthreads();
  const bool refused = no_page != 0;
  // the children's own pages, and what is copied into them
  const int64_t have = refused ? 0 : take_free(c, sh, want, [&](int page, int rank) {
    const int i = entry_of(sh, n, rank);
    const int j = copy ? rank - sh.offset[i] : held_pages(c, from.len[i]) - 1;
    pairs[rank] = make_int2(c.table[(int64_t)from.seq[i] * c.width + j], page);
    c.table[(int64_t)to.seq[i] * c.width + j] = page;
    c.refs[page] = 1;
  });
  if (refused || have < want) {
    hold(1);
    if (threadIdx.x == 0) *status = refused ? -1 : lacking(want - have);
    return;
  }
  // the shared ones, and what the children held beyond their new lengths
  if (!copy)
    each_page(c, from, n, [&](int i, int j, int p) {
      if (j < held_pages(c, from.len[i]) - (sh.offset[i + 1] - sh.offset[i])) {
        atomicAdd(&c.refs[p], 1);
        c.table[(int64_t)to.seq[i] * c.width + j] = p;
      }
    });
  each_page(c, to, n, [&](int i, int j, int) {
    if (j >= held_pages(c, from.len[i])) c.table[(int64_t)to.seq[i] * c.width + j] = -1;
  });
  for (int i = threadIdx.x; i < n; i += kPlan) c.lens[to.seq[i]] = from.len[i];
  if (threadIdx.x == 0) {
    *status = 0;
    *count = (int)want;
  }
}

// Whole pages, 16 bytes a lane, four of them under way.  Stores go past the caches, which keep the
// pages that several children copy: two copies of 8192 positions (1.28 GB moved) take 200 us so
// and 236 through them, 64 copies of part pages 43 and 46.
__global__ __launch_bounds__(256) void cache_copy_kernel(unsigned char* pool, int64_t page_bytes,
                                                         const int32_t* __restrict__ count,
                                                         const int2* __restrict__ pairs,
                                                         int pieces) {
  constexpr int kVec = 4, kPiece = 256 * kVec;
  const int n = *count;
  const int64_t vecs = page_bytes / 16;
  const int64_t items = (int64_t)n * pieces;
  for (int64_t w = blockIdx.x; w < items; w += gridDim.x) {
    const int e = (int)(w / pieces);
    const int64_t v0 = (w - (int64_t)e * pieces) * kPiece + threadIdx.x;
    const int2 pr = pairs[e];
    const u32x4* from = reinterpret_cast<const u32x4*>(pool + pr.x * page_bytes);
    u32x4* to = reinterpret_cast<u32x4*>(pool + pr.y * page_bytes);
    u32x4 x[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if (v0 + j * 256 < vecs) x[j] = from[v0 + j * 256];
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if (v0 + j * 256 < vecs) __builtin_nontemporal_store(x[j], to + v0 + j * 256);
  }
}

// ---------------------------------------------------------------------------
// compaction

__device__ inline int64_t kept(const CacheCompactArgs& a, int i) {
  return a.counts ? (int64_t)a.counts[i] : a.keep;
}

// The plan: dst's pages, and the sources' rows as they were, for the gather
// that follows (dst may be src).
__global__ __launch_bounds__(kPlan) void cache_compact_plan_kernel(CacheCompactArgs a) {
  extern __shared__ uint32_t bits[];
  __shared__ PlanShared sh;
  __shared__ SeqList from, to;
  const CacheView& c = a.c;
  const int n = a.n;
  clear_bits(bits, c.seqs);
  if (threadIdx.x == 0) sh.bad = from.most = to.most = 0;
  __syncthreads();
  bool bad = fill_lists<2>(c, {&from, &to}, {a.src, a.dst}, n);
  for (int i = threadIdx.x; i < n; i += kPlan) {   // this thread's own entries
    const int64_t k = kept(a, i);
    bad |= k < 0 || k > a.keep || (known(c, to.seq[i]) && mark(bits, to.seq[i]));
  }
  if (bad) sh.bad = 1;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlan)
    if (known(c, from.seq[i]) && marked(bits, from.seq[i]) && to.seq[i] != from.seq[i]) sh.bad = 1;
  __syncthreads();
  if (sh.bad) {
    if (threadIdx.x == 0) *a.status = -1;
    return;
  }
  auto hold = [&](int d) {   // what dst held, but for the rows that are read
    each_page(c, to, n, [&](int i, int, int p) {
      if (from.seq[i] != to.seq[i] && is_page(c, p)) atomicAdd(&c.refs[p], d);
    });
  };
  hold(-1);
  const int64_t P = 1 << c.page_shift;
  const int64_t want =
      plan_offsets(sh, n, [&](int i) { return (int)((kept(a, i) + P - 1) >> c.page_shift); });
  // the sources' rows, before any of them changes
  for (int i = threadIdx.x; i < n; i += kPlan)
    a.old_rows[(int64_t)i * (c.width + 1)] = from.len[i];
  each_page(c, from, n, [&](int i, int j, int p) {
    a.old_rows[(int64_t)i * (c.width + 1) + 1 + j] = p;
  });
  __syncthreads();
  const int64_t have = take_free(c, sh, want, [&](int page, int rank) {
    const int i = entry_of(sh, n, rank);
    c.table[(int64_t)to.seq[i] * c.width + rank - sh.offset[i]] = page;
    c.refs[page] = 1;
  });
  if (have < want) {
    hold(1);
    if (threadIdx.x == 0) *a.status = lacking(want - have);
    return;
  }
  // what dst held beyond its new length; a source that is its own dst lets its old pages
  // go, which the gather still reads
  each_page(c, to, n, [&](int i, int j, int) {
    if (j >= sh.offset[i + 1] - sh.offset[i]) c.table[(int64_t)to.seq[i] * c.width + j] = -1;
    if (from.seq[i] == to.seq[i]) {
      const int p = a.old_rows[(int64_t)i * (c.width + 1) + 1 + j];
      if (is_page(c, p)) drop(c.refs, p);
    }
  });
  for (int i = threadIdx.x; i < n; i += kPlan) c.lens[to.seq[i]] = (int)kept(a, i);
  if (threadIdx.x == 0) *a.status = 0;
}

// 16 new positions of one unit a wave: 16 rows of key codes by four (D = 128) or
// two (64) lanes of 16 bytes; four lanes' blocks of value codes, each lane's 16 (8)
// bytes from the four positions' own places.  Bound by HBM in lines of 128 bytes: a quarter of
// three messages of 8192 positions (36 layers, 8 heads: 240 MB kept) takes 151 us, in which 574 MB are
// read and 240 written, 5.4 TB/s: a kept row's 64 bytes of key codes share their line with a
// neighbour's, its value codes lie in two lines of a block of four positions.
template <int D>
__global__ __launch_bounds__(256) void cache_gather_kernel(CacheCompactArgs a, int blocks_per_unit,
                                                           int64_t items) {
  if (*a.status != 0) return;   // the plan changed nothing
  const CacheView& c = a.c;
  const int P = 1 << c.page_shift;
  const int lane = threadIdx.x & 63;
  const int units = c.layers * c.heads;
  constexpr int G = D / 32;
  const int64_t waves = (int64_t)gridDim.x * 4;
  for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < items; w += waves) {
    const int64_t eb = w / units;
    const int u = (int)(w - eb * units);
    const int i = (int)(eb / blocks_per_unit);
    const int64_t j0 = (eb - (int64_t)i * blocks_per_unit) * 16;
    const int64_t cnt = kept(a, i);
    if (j0 >= ((cnt + P - 1) & ~(int64_t)(P - 1))) continue;
    const int layer = u / c.heads, head = u - layer * c.heads;
    const int32_t* old = a.old_rows + (int64_t)i * (c.width + 1);
    const int32_t* idx = a.idx + i * a.idx_stride[0] + layer * a.idx_stride[1] +
                         head * a.idx_stride[2];
    const int page = c.table[(int64_t)a.dst[i] * c.width + (j0 >> c.page_shift)];
    const int64_t unit_off = (int64_t)u * c.unit_bytes;
    unsigned char* to = c.pool + page * c.page_bytes + unit_off;
    const int at0 = (int)(j0 & (P - 1));
    // lane l (of 16) holds the source of new position j0 + l: its unit and place
    const int len = old[0];
    const int l16 = lane & 15;
    int at = -1, spage = 0;
    if (j0 + l16 < cnt) {
      const int s = idx[j0 + l16];
      if (s >= 0 && s < len && (s >> c.page_shift) < c.width) {
        const int p = old[1 + (s >> c.page_shift)];
        if ((unsigned)p < (unsigned)c.pages) {
          spage = p;
          at = s & (P - 1);
        }
      }
    }
    // keys
    constexpr int kRowLanes = D / 32;   // lanes of 16 bytes a row of codes
    if (lane < 16 * kRowLanes) {
      const int row = lane / kRowLanes, b = lane % kRowLanes;
      const int p = __shfl(spage, row), t = __shfl(at, row);
      u32x4 x = {0u, 0u, 0u, 0u};
      if (t >= 0)
        x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
            c.pool + p * c.page_bytes + unit_off + t * (D / 2) + b * 16));
      __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to + (at0 + row) * (D / 2) + b * 16));
    }
    // values: lane (block = lane / 16, run = lane % 16)
    const int blk = lane >> 4, run = lane & 15;
    const unsigned char* vfrom[4];
    int vt[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = __shfl(spage, blk * 4 + e);
      vt[e] = __shfl(at, blk * 4 + e);
      vfrom[e] = c.pool + p * c.page_bytes + unit_off + unit_value_codes(P, D) +
                 (vt[e] >> 2) * (2 * D) + run * (D / 8) + (vt[e] & 3) * (D / 32);
    }
    unsigned char* vto = to + unit_value_codes(P, D) + ((at0 >> 2) + blk) * (2 * D) + run * (D / 8);
    if constexpr (D == 128) {
      u32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[e] = vt[e] >= 0 ? *reinterpret_cast<const uint32_t*>(vfrom[e]) : 0u;
      __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(vto));
    } else {
      uint32_t h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        h[e] = vt[e] >= 0 ? *reinterpret_cast<const uint16_t*>(vfrom[e]) : 0u;
      *reinterpret_cast<uint2*>(vto) = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
    }
    // scales: lane = (position, group); rows without a source get the least
    if (lane < 16 * G) {
      const int row = lane / G, g = lane % G;
      const int p = __shfl(spage, row), t = __shfl(at, row);
      unsigned char ks = 3, vs = 3;
      if (t >= 0) {
        const unsigned char* from = c.pool + p * c.page_bytes + unit_off;
        ks = from[unit_key_scales(P, D) + t * G + g];
        vs = from[unit_value_scales(P, D) + ((t >> 2) * G + g) * 4 + (t & 3)];
      }
      const int q = at0 + row;
      to[unit_key_scales(P, D) + q * G + g] = ks;
      to[unit_value_scales(P, D) + ((q >> 2) * G + g) * 4 + (q & 3)] = vs;
    }
  }
}

size_t bit_bytes(const CacheView& c) { return (size_t)((c.seqs + 31) / 32) * sizeof(uint32_t); }

}  // namespace

hipError_t launch_cache_extend(const CacheView& c, const int32_t* seqs, const int32_t* add, int n,
                               int32_t* status, hipStream_t s) {
  cache_extend_kernel<<<1, kPlan, bit_bytes(c), s>>>(c, seqs, add, n, status);
  return hipGetLastError();
}

hipError_t launch_cache_free(const CacheView& c, const int32_t* seqs, int n, hipStream_t s) {
  if (n == 0) return hipSuccess;
  cache_free_kernel<<<(unsigned)n, 256, 0, s>>>(c, seqs);
  return hipGetLastError();
}

size_t cache_fork_ws(int64_t n, int64_t width) {
  return 16 + (((size_t)n * (size_t)width * sizeof(int2) + 15) & ~(size_t)15);
}

hipError_t launch_cache_fork(const CacheView& c, const int32_t* parents, const int32_t* children,
                             int n, bool copy, int32_t* status, void* ws, hipStream_t s) {
  int32_t* count = static_cast<int32_t*>(ws);
  int2* pairs = reinterpret_cast<int2*>(static_cast<unsigned char*>(ws) + 16);
  cache_fork_kernel<<<1, kPlan, bit_bytes(c), s>>>(c, parents, children, n, copy ? 1 : 0, status,
                                                   count, pairs);
  if (n > 0) {
    const int64_t vecs = c.page_bytes / 16;
    const int pieces = (int)((vecs + 1023) / 1024);
    const int64_t most = (int64_t)n * (copy ? c.width : 1) * pieces;
    const unsigned grid = (unsigned)(most < 4096 ? most : 4096);
    cache_copy_kernel<<<grid, 256, 0, s>>>(c.pool, c.page_bytes, count, pairs, pieces);
  }
  return hipGetLastError();
}

size_t cache_compact_ws(int64_t n, int64_t width) {
  return ((size_t)n * (size_t)(width + 1) * sizeof(int32_t) + 15) & ~(size_t)15;
}

hipError_t launch_cache_compact(const CacheCompactArgs& a, hipStream_t s) {
  cache_compact_plan_kernel<<<1, kPlan, bit_bytes(a.c), s>>>(a);
  if (a.n > 0) {
    const int64_t P = 1 << a.c.page_shift;
    const int blocks = (int)((a.keep + P - 1) / P * (P / 16));
    const int64_t items = (int64_t)a.n * blocks * a.c.layers * a.c.heads;
    const int64_t groups = (items + 3) / 4;
    const unsigned grid = (unsigned)(groups < 4096 ? groups : 4096);
    if (a.c.D == 64) cache_gather_kernel<64><<<grid, 256, 0, s>>>(a, blocks, items);
    else cache_gather_kernel<128><<<grid, 256, 0, s>>>(a, blocks, items);
  }
  return hipGetLastError();
}

}  // namespace cb
