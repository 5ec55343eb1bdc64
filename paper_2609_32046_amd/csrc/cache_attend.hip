// Attention over the paged four-bit cache (gfx950).
//
// A wave holds the query rows of one KV head in blocks of 16 (row = token *
// group + head) and walks positions in steps of 32.  With scores as S^T = K Q^T
// and outputs as O^T = V^T P^T, a lane of the 16 x 16 MFMA results holds one
// query row in both: statistics are two registers a block, no lane exchange
// is needed but for a new maximum, and the weights are the second product's operand
// as they stand: lane (row, g) holds the weights of positions 4g..4g+3 of
// both halves of the step, and the contraction runs over them in that order.
// The order of a head's values is free in the first product, so lane (position,
// g) takes values g*D/4.. of its key, one load with one scale; in the second the
// lanes r of a tile take values r*D/16 + tile, so that a lane's values are
// neighbours too: 16 bytes are four positions of them, with one group's scales.
// Codes become bf16 by conversion with their scale, exactly.  (A scaled MFMA that takes
// the codes as they are, with the query in two fp8 parts, spares the keys' conversions,
// but sums with about 16 bits: log-sums were off by 2e-5.)  fp32 queries and weights go
// in as three bf16 parts, 24 bits; the weights of bf16 calls as two or one (kernel).
//
// The positions of all sequences, in rounds of 128, are dealt to the workgroups in
// equal runs, however ragged they are: a run may end one sequence and begin the next
// (each workgroup finds its own from the lengths).  Four waves take a run's steps in
// turn; their results meet in LDS, and those of a sequence that several runs
// share in a second, small kernel.  Where the table bounds the sequences to short ones, a run
// is a sequence and the second kernel falls away; where there are many, a workgroup is one
// wave and nothing meets at all.
//
// Few rows are bound by HBM: 64 sequences of up to 16384 positions (606 MB) take 119 us in all,
// 5.1 TB/s, against 109 us with the loads alone; one of 131072 (143 MB) takes 29 us and 5 us of
// joining.  Many rows are bound by issue: a step of 64 rows is 64 MFMAs (1060 cycles), 32
// exponentials (380) and about 250 other vector instructions (1150), and the two waves of a
// SIMD overlap little of it: 2500 rows (500 tokens of 40 heads) over 32768 positions
// take 351 us, 950 TFLOP/s.  Tried for them and slower: conversions shared through LDS
// (416-459 us), 32 x 32 x 16 MFMAs (402 us), waves with rows of their own (371 us).
#include <math.h>

#include "cache.h"

namespace cb {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kStep = 32;                   // positions of a wave's step
constexpr int kRound = kStep * kWaves;      // of a workgroup's
constexpr float kNone = -1e38f;             // reference maximum before any position
constexpr float kSlack = 8.f;               // weights may grow to 2^8 before a new reference

typedef const __attribute__((address_space(4))) int32_t* ConstInts;

__device__ inline bf16x2 cvt2(uint32_t c, float s, int byte) {
  switch (byte) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
  }
}

__device__ inline uint32_t u32_of(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }

__device__ inline uint32_t pack_bf16(float a, float b) {   // nearest, ties to even
  const bf16x2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// Eight codes (a dword) times their scale as bf16, in order.
__device__ inline bf16x8 expand8(uint32_t c, float s) {
  u32x4 r = {u32_of(cvt2(c, s, 0)), u32_of(cvt2(c, s, 1)), u32_of(cvt2(c, s, 2)),
             u32_of(cvt2(c, s, 3))};
  return __builtin_bit_cast(bf16x8, r);
}

// x as the sum of three bf16 values, the first two cut, the last rounded: 24 bits.
__device__ inline void split3(float x, float* a, float* b, float* c) {
  *a = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  const float r = x - *a;
  *b = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
  *c = r - *b;
}
__device__ inline uint32_t high_pair(float a, float b) {   // the upper halves of two floats
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

__device__ inline int seq_len(const AttendArgs& a, int b) {
  const int s = a.seqs ? a.seqs[b] : b;
  if ((unsigned)s >= (unsigned)a.c.seqs) return 0;
  const int len = a.c.lens[s];
  return len < 0 ? 0 : len < a.room ? len : a.room;
}

// The same through the scalar cache, for a row that the whole wave asks for.
__device__ inline int seq_of(const AttendArgs& a, int b) {
  return a.seqs ? ((ConstInts)a.seqs)[b] : b;
}
__device__ inline int uniform_len(const AttendArgs& a, int b) {
  const int s = seq_of(a, b);
  if ((unsigned)s >= (unsigned)a.c.seqs) return 0;
  const int len = ((ConstInts)a.c.lens)[s];
  return len < 0 ? 0 : len < a.room ? len : a.room;
}
__device__ inline int query_tokens(const AttendArgs& a, int b) {
  const int m = a.q_lens ? ((ConstInts)a.q_lens)[b] : (int)a.q_len;
  return m < 0 ? 0 : m < (int)a.q_len ? m : (int)a.q_len;
}

// Token of a query row, row / group: by the group's reciprocal, floor(2^32 / group), which gives
// the quotient or one less; the compiler's own division takes four times the instructions.
__device__ inline int token_of(const AttendArgs& a, int row) {
  const int t = (int)__umulhi((uint32_t)row, a.recip);
  return row - t * a.group >= a.group ? t + 1 : t;
}

// Rounds of a sequence; an empty one takes its turn too, to write its zeros.
__device__ inline int rounds_of(int len) { return len <= kRound ? 1 : (len + kRound - 1) / kRound; }

// Sum over the lanes.
__device__ inline uint32_t wave_sum(uint32_t x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

// The same value in scalar registers, where every lane holds the same.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Where run `run` begins: a sequence and the rounds before it (of all sequences), all of them
// below 2^31.  Every wave works it out for itself.
struct Run {
  int b;
  uint32_t before, lo, hi;   // rounds before sequence b; the run
};

__device__ inline uint32_t rounds_per_run(const AttendArgs& a, uint32_t* total) {
  uint32_t t = 0;
  if (a.n == 1) {
    t = rounds_of(uniform_len(a, 0));
  } else {
    for (int i = threadIdx.x & 63; i < a.n; i += 64) t += rounds_of(seq_len(a, i));
    t = wave_sum(t);
  }
  t = uniform(t);
  *total = t;
  return (t + a.target - 1) / (uint32_t)a.target;
}

// False behind the last run.
__device__ inline bool find_run(const AttendArgs& a, int run, Run* r) {
  if (a.whole) {   // a run a sequence
    *r = {run, 0, 0, (uint32_t)rounds_of(uniform_len(a, run))};
    return true;
  }
  uint32_t total;
  const uint32_t per = rounds_per_run(a, &total);
  r->lo = run * per;   // below total + target
  r->hi = r->lo + per < total ? r->lo + per : total;
  r->b = 0;
  r->before = 0;
  if (r->lo >= total) return false;
  if (a.n == 1 || r->lo == 0) return true;
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < a.n; i0 += 64) {
    const int i = i0 + lane;
    const uint32_t k = i < a.n ? rounds_of(seq_len(a, i)) : 0;
    uint32_t incl = k;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(incl, d);
      if (lane >= d) incl += y;
    }
    const uint64_t mine = __ballot(r->before + incl > r->lo);
    if (mine) {
      const int l = __ffsll((unsigned long long)mine) - 1;
      r->b = i0 + uniform(l);
      r->before += uniform(__shfl(incl - k, l));
      return true;
    }
    r->before += uniform(__shfl(incl, 63));
  }
  return false;
}

// What a step reads, as it lies in memory: per half (16 positions) a lane's key codes,
// key scale, value codes of four positions and their scales.
template <int D>
struct Raw {
  uint32_t k[2][D / 32], v[2][D / 32];
  uint32_t ks[2], vs[2];
  uint32_t here;   // uniform: bit h, the half has a page
};

// Byte offsets of a lane's pieces within 16 positions of a unit: 32 bits beside a uniform base.
struct LaneAt {
  uint32_t k, v, ks, vs;
};

template <int D>
__device__ inline LaneAt lane_at(int r, int g) {
  constexpr int G = D / 32;
  return {(uint32_t)(r * (D / 2) + g * (D / 8)), (uint32_t)(g * (2 * D) + r * (D / 8)),
          (uint32_t)(r * G + g * G / 4), (uint32_t)((g * G + r * G / 16) * 4)};
}

// Loads through a buffer descriptor of the unit: the lane's 32-bit offset and a scalar one, so
// that no address is formed in vector registers.
template <int D>
__device__ inline void load_half(const unsigned char* unit, int P, int at, const LaneAt& la,
                                 Raw<D>* w, int h) {
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<unsigned char*>(unit), 0, P * (D + D / 16), 0x00027000);
  const int ko = at * (D / 2), vo = ko + unit_value_codes(P, D);
  const int kso = unit_key_scales(P, D) + at * (D / 32), vso = kso + P * (D / 32);
  if constexpr (D == 128) {
    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)la.k, ko, 0);
    const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)la.v, vo, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w->k[h][i] = x[i];
      w->v[h][i] = y[i];
    }
  } else {
    const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(rs, (int)la.k, ko, 0);
    const u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(rs, (int)la.v, vo, 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w->k[h][i] = x[i];
      w->v[h][i] = y[i];
    }
  }
  w->ks[h] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rs, (int)la.ks, kso, 0);
  w->vs[h] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, (int)la.vs, vso, 0);
}

// The larger, NaN if one is: one instruction for three of them, where fmaxf would quiet each
// operand first.
__device__ inline float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A lane's part of a block of 16 query rows: values g*D/4 .. of its row, the keys' own order.
template <int D, bool F32>
struct Query;
template <int D>
struct Query<D, true> {
  bf16x8 x[D / 32][3];
  __device__ void load(const float* p, int g, bool live) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      f32x4 u = {0, 0, 0, 0}, v = {0, 0, 0, 0};
      if (live) {
        u = *reinterpret_cast<const f32x4*>(p + g * (D / 4) + 8 * j);
        v = *reinterpret_cast<const f32x4*>(p + g * (D / 4) + 8 * j + 4);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float a, b, c;
        split3(i < 4 ? u[i & 3] : v[i & 3], &a, &b, &c);
        x[j][0][i] = (__bf16)a;
        x[j][1][i] = (__bf16)b;
        x[j][2][i] = (__bf16)c;
      }
    }
  }
};
template <int D>
struct Query<D, false> {
  bf16x8 x[D / 32][1];
  __device__ void load(const __bf16* p, int g, bool live) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if (live) w = *reinterpret_cast<const u32x4*>(p + g * (D / 4) + 8 * j);
      x[j][0] = __builtin_bit_cast(bf16x8, w);
    }
  }
};

template <bool F32>
struct RowType;
template <>
struct RowType<false> { typedef __bf16 type; };
template <>
struct RowType<true> { typedef float type; };

// N neighbouring values of an output row: 4 or 8.
template <int N>
__device__ inline void put_row(float* p, const float (&x)[N]) {
#pragma unroll
  for (int v = 0; v < N; v += 4)
    *reinterpret_cast<f32x4*>(p + v) = f32x4{x[v], x[v + 1], x[v + 2], x[v + 3]};
}
template <int N>
__device__ inline void put_row(__bf16* p, const float (&x)[N]) {
  uint32_t w[N / 2];
#pragma unroll
  for (int v = 0; v < N; v += 2) w[v / 2] = pack_bf16(x[v], x[v + 1]);
  if constexpr (N == 8) *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]};
  else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
}

// Values of one tile pair (values 2b and 2b + 1 of the lane's run) for the step's 32 positions:
// conversions give (value 2b, value 2b+1) of a position; the product wants pairs of
// positions.
template <int D>
__device__ inline void value_tiles(const uint32_t (&wv)[2][D / 32], const float vscale[8], int b, bf16x8* even,
                                   bf16x8* odd) {
  u32x4 lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {   // positions 2i, 2i + 1 of the lane's eight
    const int h = i >> 1, e = (2 * i) & 3;
    uint32_t x, y;
    if constexpr (D == 128) {     // a dword a position
      x = u32_of(cvt2(wv[h][e], vscale[2 * i], b));
      y = u32_of(cvt2(wv[h][e + 1], vscale[2 * i + 1], b));
    } else {                      // two bytes a position
      x = u32_of(cvt2(wv[h][e >> 1], vscale[2 * i], b));
      y = u32_of(cvt2(wv[h][e >> 1], vscale[2 * i + 1], 2 + b));
    }
    lo[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
    hi[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
  *even = __builtin_bit_cast(bf16x8, lo);
  *odd = __builtin_bit_cast(bf16x8, hi);
}

template <int D, bool F32, int RT, int W>
__global__ __launch_bounds__(64 * W, RT == 1 && !F32 ? 3 : 2) void attend_kernel(AttendArgs a) {
  typedef typename RowType<F32>::type T;
  constexpr int KS = D / 32;              // first product: MFMAs of a block and half
  constexpr int VT = D / 16;              // second: tiles of 16 values
  constexpr int NQ = F32 ? 3 : 1;
  // bf16 parts of a weight.  Two, 16 bits, where a wave holds one block: outputs are then as near as
  // their own rounding lets them be (0.0016 of their size over thousands of positions; 0.0023 with one part)
  // for 0 to 4% of the time of a call (131072 positions 31.7 and 32.1 us, 64 sequences up to 16384 121.5 and
  // 122.0), 7 or 8% where a wave has few steps (16 of 2048: 16.0 and 17.3; 16 tokens of 32 heads behind 1024
  // 9.9 and 10.5).  With more rows the products weigh more: 2500 rows
  // over 32768 positions take 354 us with one part and 490 with two, 32 tokens of 32 heads 34.6 and 40.3.
  constexpr int NW = F32 ? 3 : RT == 1 ? 2 : 1;
  // Steps of codes in registers, the next under way.  With three the loop is half as long again, which a
  // short sequence pays in instruction fetches: 131072 positions 34.6 us, 32.4 with two; 512
  // positions 8.2 and 7.4.
  constexpr int NB = 2;
  constexpr bool kSharedQ = !F32 && RT > 1;       // the four waves' query rows are the same
  constexpr int kPad = 4;
  constexpr int kTurn = kStep * W;                // positions of a workgroup's step
  __shared__ float so[W > 1 ? W : 1][W > 1 ? 16 : 1][D + kPad];
  __shared__ float sm[W][RT * 16], sl[W][RT * 16];
  __shared__ bf16x8 sq[kSharedQ ? RT : 1][KS][kSharedQ ? 64 : 1];

  const int lane = threadIdx.x & 63;
  const int wave = uniform((int)threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  // heads fastest: the units of a page lie side by side, and with eight heads
  // each L2 (one per XCD, workgroups in turn) sees one head's positions
  uint32_t id = blockIdx.x;
  const int head = (int)(id % (uint32_t)a.c.heads);
  id /= (uint32_t)a.c.heads;
  const int tile = (int)(id % (uint32_t)a.row_tiles);
  id /= (uint32_t)a.row_tiles;
  const int run_id = (int)(id % (uint32_t)a.target);
  const int layer = (int)(id / (uint32_t)a.target);

  Run run;
  if (!find_run(a, run_id, &run)) return;
  const int G = a.group;
  const int P = 1 << a.c.page_shift;
  const int row0 = tile * (RT * 16);
  const LaneAt la = lane_at<D>(r, g);
  const unsigned char* pool = a.c.pool + ((int64_t)(a.layer0 + layer) * a.c.heads + head) *
                                             a.c.unit_bytes;

  // The run's sequences, one after the other.
  for (; run.b < a.n && run.before < run.hi; ++run.b) {
    const int b = run.b;
    const int seq = seq_of(a, b);
    const int len = uniform_len(a, b);
    const uint32_t before = run.before;
    const int rounds = rounds_of(len);
    run.before += rounds;
    const int m = query_tokens(a, b);
    const int rows = m * G;   // at most 2^26
    if (row0 >= rows) continue;   // also m = 0; uniform over the workgroup
    const int rlo = (int)(run.lo > before ? run.lo - before : 0);
    const int rhi = (int)(run.hi < run.before ? run.hi - before : rounds);
    const bool whole = rlo == 0 && rhi == rounds;
    const int lo = rlo * kRound;   // below 2^31 - 2^16
    const int end = (int64_t)rhi * kRound < len ? rhi * kRound : len;

    // The positions that all rows of the tile see, and that any sees: rows ascend with tokens, so the
    // first row sees least, the last live one most
    const int row_last = (row0 + RT * 16 < rows ? row0 + RT * 16 : rows) - 1;
    const int see_first = a.causal ? len - m + token_of(a, row0) + 1 : len;
    const int see_last = a.causal ? len - m + token_of(a, row_last) + 1 : len;
    const int full = see_first < end ? (see_first > 0 ? see_first : 0) : end;
    const int hi = see_last < end ? (see_last > 0 ? see_last : 0) : end;

    const int steps = hi <= lo ? 0 : (hi - lo + kTurn - 1) / kTurn;
    // The page table through the scalar cache: its waits are apart from those for the codes,
    // so that these stay under way.  A half without a page (behind the end, or a
    // table entry that is none) reads page 0, in bounds, and is masked.  Steps behind the
    // last read it again: a load that is always issued lets the compiler count.
    const ConstInts row_pages = (ConstInts)(a.c.table + (int64_t)seq * a.c.width);
    const int mine = lo + wave * kStep;
    int id0 = 0, id1 = 0;
    auto look_up = [&](int k) {
      const int t0 = mine + (k < steps ? k : steps - 1) * kTurn, t1 = t0 + 16;
      id0 = row_pages[(t0 < hi ? t0 : hi - 1) >> a.c.page_shift];
      id1 = row_pages[(t1 < hi ? t1 : hi - 1) >> a.c.page_shift];
    };
    auto fetch = [&](int k, Raw<D>& w) {
      const int t0 = mine + (k < steps ? k : steps - 1) * kTurn;
      const bool ok0 = t0 < hi && (unsigned)id0 < (unsigned)a.c.pages;
      const bool ok1 = t0 + 16 < hi && (unsigned)id1 < (unsigned)a.c.pages;
      w.here = (ok0 ? 1u : 0u) | (ok1 ? 2u : 0u);
      load_half<D>(pool + (ok0 ? id0 : 0) * a.c.page_bytes, P, t0 & (P - 1), la, &w, 0);
      load_half<D>(pool + (ok1 ? id1 : 0) * a.c.page_bytes, P, (t0 + 16) & (P - 1), la, &w, 1);
      look_up(k + 1);
    };
    Raw<D> raw[NB];
    if (steps > 0) {
      look_up(0);
#pragma unroll
      for (int i = 0; i < NB - 1; ++i) fetch(i, raw[i]);
    }

    // Limits of this lane's rows.
    int pr = r;
    if constexpr (RT > 1) asm volatile("" : "+v"(pr));
    int limit[RT];
    const T* qp[RT];
    bool live[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = row0 + t * 16 + pr;
      live[t] = row < rows;
      const int tok = live[t] ? token_of(a, row) : 0;
      const int qh = head * G + (live[t] ? row - tok * G : 0);
      const int see = a.causal ? len - m + tok + 1 : len;
      limit[t] = !live[t] || see < 0 ? 0 : see < end ? see : end;
      qp[t] = static_cast<const T*>(a.q) + layer * a.q_stride[0] + b * a.q_stride[1] +
              qh * a.q_stride[2] + tok * a.q_stride[3];
    }
    Query<D, F32> q[kSharedQ ? 1 : RT];
#pragma unroll
    for (int t = 0; t < RT && steps > 0; ++t) {
      if constexpr (kSharedQ) {
        // held in LDS, in the lanes' order: 16 reads a step of 64 rows, against 64 registers
        if (t % W == wave) {
          q[0].load(qp[t], g, live[t]);
#pragma unroll
          for (int j = 0; j < KS; ++j) sq[t][j][lane] = q[0].x[j][0];
        }
      } else {
        q[t].load(qp[t], g, live[t]);
      }
    }
    if (kSharedQ) __syncthreads();

    float top[RT], sum[RT];
    f32x4 o[RT][VT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      top[t] = kNone;
      sum[t] = 0.f;
#pragma unroll
      for (int i = 0; i < VT; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    auto step = [&](int k, const Raw<D>& cur) {
      const int t0 = mine + k * kTurn;
      if (t0 >= hi) return;
      const bool masked = t0 + kStep > full || cur.here != 3u;   // uniform
      uint32_t vs[2] = {cur.vs[0], cur.vs[1]};
      uint32_t nans[2] = {0u, 0u};   // 0x80 in the byte of a position whose value group may not be finite
      if (masked) {
        // what a masked position holds counts for nothing: 0 times a NaN or an infinity would be
        // NaN.  A scale of 255 is NaN, with 253 and 254 (never stored, but a page may hold anything
        // before its positions are written) codes pass bf16's range.
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int left = ((cur.here >> h) & 1u) ? hi - (t0 + 16 * h + 4 * g) : 0;   // of the lane's four
          const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
          // bytes of 253 and up: bit 7 is set, and the seven below reach 125
          nans[h] = ((vs[h] & 0x7f7f7f7fu) + 0x03030303u) & vs[h] & 0x80808080u & keep;
          vs[h] &= keep & ~((nans[h] >> 7) * 255u);
        }
      }
      float vscale[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        vscale[i] = __uint_as_float(((vs[i >> 2] >> (8 * (i & 3))) & 255u) << 23);
      bf16x8 p[RT][NW];
      {
        bf16x8 kk[2][KS];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float s = __uint_as_float(cur.ks[h] << 23);
#pragma unroll
          for (int j = 0; j < KS; ++j) kk[h][j] = expand8(cur.k[h][j], s);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          f32x4 s[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = NQ - 1; u >= 0; --u)   // small parts first
#pragma unroll
              for (int j = 0; j < KS; ++j)
                s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    kk[h][j], kSharedQ ? sq[t][j][lane] : q[kSharedQ ? 0 : t].x[j][u], s[h], 0, 0, 0);
          }
          if (masked) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int pos = t0 + (i >> 2) * 16 + 4 * g + (i & 3);
              if (pos >= limit[t] || !((cur.here >> (i >> 2)) & 1u)) s[i >> 2][i & 3] = -INFINITY;
            }
          }
          float mx = max2(max2(s[0][0], s[0][1]), s[0][2]);
          mx = max2(max2(mx, s[0][3]), s[1][0]);
          mx = max2(max2(mx, s[1][1]), s[1][2]);
          mx = max2(mx, s[1][3]) * a.c2;   // a NaN is no new maximum, and makes its row NaN
          if (__any(mx > top[t] + kSlack)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            // only rows that outgrew their reference get a new one
            const float next = mx > top[t] + kSlack ? mx : top[t];
            const float f = next == top[t] ? 1.f : __builtin_amdgcn_exp2f(top[t] - next);
            top[t] = next;
            sum[t] *= f;
#pragma unroll
            for (int i = 0; i < VT; ++i) o[t][i] *= f;
          }
          float e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 2][i & 3], a.c2, -top[t]));
          sum[t] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
          if constexpr (F32) {
            u32x4 w[3];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float a0, a1, a2, b0, b1, b2;
              split3(e[2 * i], &a0, &a1, &a2);
              split3(e[2 * i + 1], &b0, &b1, &b2);
              w[0][i] = high_pair(a0, b0);
              w[1][i] = high_pair(a1, b1);
              w[2][i] = pack_bf16(a2, b2);
            }
#pragma unroll
            for (int u = 0; u < 3; ++u) p[t][u] = __builtin_bit_cast(bf16x8, w[u]);
          } else {
            // the rounding of a weight: at most 2^-8 of it, as much as an output's own; what is
            // left of it, rounded again, leaves 2^-16
            u32x4 w, lo;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i] = pack_bf16(e[2 * i], e[2 * i + 1]);
              if constexpr (NW == 2)
                lo[i] = pack_bf16(e[2 * i] - __uint_as_float(w[i] << 16),
                                  e[2 * i + 1] - __uint_as_float(w[i] & 0xffff0000u));
            }
            p[t][0] = __builtin_bit_cast(bf16x8, w);
            if constexpr (NW == 2) p[t][1] = __builtin_bit_cast(bf16x8, lo);
          }
        }
      }
#pragma unroll
      for (int v = 0; v < VT / 2; ++v) {
        bf16x8 even, odd;
        value_tiles<D>(cur.v, vscale, v, &even, &odd);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int u = NW - 1; u >= 0; --u) {
            o[t][2 * v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, p[t][u], o[t][2 * v], 0, 0, 0);
            o[t][2 * v + 1] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, p[t][u], o[t][2 * v + 1], 0, 0, 0);
          }
      }
      if (masked && __any((nans[0] | nans[1]) != 0u)) {
        // a value that is not finite reaches the rows that see its position, as NaN in its group
        constexpr int kRun = 16 / (D / 32);               // lanes r of one group
        const int r0 = (g * (D / 32) / 4) * kRun;         // the group that this lane's outputs lie in
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
          const uint64_t who = __ballot(((i < 4 ? nans[0] : nans[1]) >> (8 * (i & 3) + 7)) & 1u);
#pragma unroll 1
          for (int gg = 0; gg < 4; ++gg) {
            const int pos = t0 + (i >> 2) * 16 + 4 * gg + (i & 3);
            if ((who >> (16 * gg + r0)) & 1u) {
#pragma unroll
              for (int t = 0; t < RT; ++t)
                if (pos < limit[t]) {
#pragma unroll
                  for (int v = 0; v < VT; ++v) o[t][v] += __uint_as_float(0x7fc00000u);
                }
            }
          }
        }
      }
    };
    for (int k0 = 0; k0 < steps; k0 += NB)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        fetch(k0 + i + NB - 1, raw[(i + NB - 1) % NB]);
        if (k0 + i < steps) step(k0 + i, raw[i]);
      }

    if constexpr (W == 1) {
      // the wave has its rows to itself: a lane's D/16 neighbouring values at a time
      int er = r;
      if constexpr (RT > 1) asm volatile("" : "+v"(er));
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        sum[t] += __shfl_xor(sum[t], 16);
        sum[t] += __shfl_xor(sum[t], 32);
        const int row = row0 + t * 16 + er;
        if (row >= rows) continue;
        const float inv = sum[t] == 0.f ? 0.f : 1.f / sum[t];
        const int tok = token_of(a, row);
        const int qh = head * G + row - tok * G;
        T* out = static_cast<T*>(a.out) + layer * a.out_stride[0] + b * a.out_stride[1] +
                 qh * a.out_stride[2] + tok * a.out_stride[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x[VT];
#pragma unroll
          for (int v = 0; v < VT; ++v) x[v] = o[t][v][i] * inv;
          put_row<VT>(out + (4 * g + i) * VT, x);
        }
        if (a.lse && g == 0)
          a.lse[(((int64_t)layer * a.n + b) * a.q_heads + qh) * a.q_len + tok] =
              sum[t] == 0.f ? -INFINITY : (top[t] + log2f(sum[t])) * 0.69314718055994531f;
      }
      if (kSharedQ) __syncthreads();   // the next sequence writes the same LDS
      continue;
    }
    // The four lane groups' sums, then the four waves' results.  With several blocks the thread's
    // number is taken anew, or what follows from it would be worked out before the loop and
    // spilled.
    int tid = (int)threadIdx.x;
    if constexpr (RT > 1) asm volatile("" : "+v"(tid));
    const int er = tid & 15, eg = (tid >> 4) & 3;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      sum[t] += __shfl_xor(sum[t], 16);
      sum[t] += __shfl_xor(sum[t], 32);
      if (eg == 0) {
        sm[wave][t * 16 + er] = top[t];
        sl[wave][t * 16 + er] = sum[t];
      }
    }
    // run and sequence both ascend, so their sum names a piece
    const int64_t piece = ((int64_t)layer * a.c.heads + head) * a.slots + run_id + b;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (t > 0) __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < VT; v += 4) {
          // values (4g + i) * D/16 + v ..: one from each of four tiles
          const f32x4 x = {o[t][v][i], o[t][v + 1][i], o[t][v + 2][i], o[t][v + 3][i]};
          *reinterpret_cast<f32x4*>(&so[wave][er][(4 * eg + i) * VT + v]) = x;
        }
      __syncthreads();
      // thread: row tid / 16, D/16 of its values
      const int qr = tid >> 4, d0 = (tid & 15) * VT;
      const int row = row0 + t * 16 + qr;
      float mw[kWaves], M = kNone, L = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        mw[w] = sm[w][t * 16 + qr];
        M = fmaxf(M, mw[w]);
      }
      float acc[VT];
#pragma unroll
      for (int v = 0; v < VT; ++v) acc[v] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = mw[w] == M ? 1.f : __builtin_amdgcn_exp2f(mw[w] - M);
        L += sl[w][t * 16 + qr] * f;
#pragma unroll
        for (int v = 0; v < VT; ++v) acc[v] += so[w][qr][d0 + v] * f;
      }
      if (row < rows) {
        if (whole) {
          const float inv = L == 0.f ? 0.f : 1.f / L;
          const int tok = token_of(a, row);
          const int qh = head * G + row - tok * G;
          T* out = static_cast<T*>(a.out) + layer * a.out_stride[0] + b * a.out_stride[1] +
                   qh * a.out_stride[2] + tok * a.out_stride[3] + d0;
#pragma unroll
          for (int v = 0; v < VT; ++v) acc[v] *= inv;
          put_row<VT>(out, acc);
          if (a.lse && (tid & 15) == 0)
            a.lse[(((int64_t)layer * a.n + b) * a.q_heads + qh) * a.q_len + tok] =
                L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
        } else {
          const int64_t at = piece * a.rows_pad + row;
          float* po = a.part_o + at * D + d0;
#pragma unroll
          for (int v = 0; v < VT; v += 4)
            *reinterpret_cast<f32x4*>(po + v) = f32x4{acc[v], acc[v + 1], acc[v + 2], acc[v + 3]};
          if ((tid & 15) == 0) a.part_ml[at] = make_float2(M, L);
        }
      }
    }
    __syncthreads();   // the next sequence writes the same LDS
  }
}

// Rows of sequences that several runs share.  SETS groups of D/4 lanes read a row's pieces in
// turn, then join in order: as many as a workgroup holds where a row has dozens of
// pieces (one answer's long context), one where it has a few (a prompt's thousands of rows).
template <int D, bool F32, int SETS>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, uint32_t row_blocks) {
  typedef typename RowType<F32>::type T;
  constexpr int kLanes = D / 4, kRows = 256 / kLanes / SETS;
  constexpr int kAhead = SETS > 1 ? 12 : 4;   // pieces under way: 96 of a row in one turn
  __shared__ f32x4 so[SETS][kLanes];
  __shared__ float2 sml[SETS];
  uint32_t id = blockIdx.x;
  const int set = (int)threadIdx.x / kLanes % SETS;
  const int row = (int)(id % row_blocks) * kRows + (int)threadIdx.x / (kLanes * SETS);
  id /= row_blocks;
  const int head = (int)(id % (uint32_t)a.c.heads);
  id /= (uint32_t)a.c.heads;
  const int b = (int)(id % (uint32_t)a.n);
  const int layer = (int)(id / (uint32_t)a.n);
  const int rows = query_tokens(a, b) * a.group;
  const bool live = row < rows;
  if (SETS > 1 && !live) return;   // one row a workgroup
  uint32_t total;
  const uint32_t per = rounds_per_run(a, &total);
  uint32_t before = 0;
  if (b > 0) {
    for (int i = (int)threadIdx.x & 63; i < b; i += 64) before += rounds_of(seq_len(a, i));
    before = uniform(wave_sum(before));
  }
  const uint32_t first = before / per;
  const int count = (int)((before + rounds_of(uniform_len(a, b)) - 1) / per - first) + 1;
  if (count == 1 || !live) return;
  const int d0 = ((int)threadIdx.x % kLanes) * 4;
  const int64_t base = ((int64_t)layer * a.c.heads + head) * a.slots + first + b;
  float M = kNone, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = set; k0 < count; k0 += SETS * kAhead) {
    float2 ml[kAhead];
    f32x4 x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int k = k0 + j * SETS;
      ml[j] = make_float2(kNone, 0.f);
      x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k < count) {
        const int64_t at = (base + k) * a.rows_pad + row;
        ml[j] = a.part_ml[at];
        x[j] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + d0);
      }
    }
    float next = M;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) next = fmaxf(next, ml[j].x);
    const float f0 = M == next ? 1.f : __builtin_amdgcn_exp2f(M - next);
    L *= f0;
    acc *= f0;
    M = next;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const float f = ml[j].x == M ? 1.f : __builtin_amdgcn_exp2f(ml[j].x - M);
      L += ml[j].y * f;
      acc += x[j] * f;
    }
  }
  if constexpr (SETS > 1) {
    so[set][threadIdx.x % kLanes] = acc;
    if (d0 == 0) sml[set] = make_float2(M, L);
    __syncthreads();
    if (set != 0) return;
#pragma unroll
    for (int w = 0; w < SETS; ++w) M = fmaxf(M, sml[w].x);
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    L = 0.f;
#pragma unroll
    for (int w = 0; w < SETS; ++w) {
      const float f = sml[w].x == M ? 1.f : __builtin_amdgcn_exp2f(sml[w].x - M);
      L += sml[w].y * f;
      acc += so[w][threadIdx.x] * f;
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int tok = token_of(a, row);
  const int qh = head * a.group + row - tok * a.group;
  T* out = static_cast<T*>(a.out) + layer * a.out_stride[0] + b * a.out_stride[1] +
           qh * a.out_stride[2] + tok * a.out_stride[3] + d0;
  acc *= inv;
  if constexpr (F32) {
    *reinterpret_cast<f32x4*>(out) = acc;
  } else {
    *reinterpret_cast<u32x2*>(out) = u32x2{pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3])};
  }
  if (a.lse && d0 == 0)
    a.lse[(((int64_t)layer * a.n + b) * a.q_heads + qh) * a.q_len + tok] =
        L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

template <int D, bool F32>
hipError_t launch(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  constexpr int kMost = !F32 ? 4 : D == 64 ? 2 : 1;   // blocks of a wave, as in make_attend_plan
  const int64_t grid = (int64_t)a.c.heads * a.row_tiles * a.target * a.layers;
  if (grid * kThreads > kMaxThreads) return hipErrorInvalidValue;
  if (p.alone) {
    if (p.blocks == 1) attend_kernel<D, F32, 1, 1><<<(unsigned)grid, 64, 0, s>>>(a);
    else if (F32 || p.blocks == 2) attend_kernel<D, F32, kMost < 2 ? kMost : 2, 1><<<(unsigned)grid, 64, 0, s>>>(a);
    else attend_kernel<D, F32, kMost, 1><<<(unsigned)grid, 64, 0, s>>>(a);
    return hipGetLastError();
  }
  if (p.blocks == 1) attend_kernel<D, F32, 1, kWaves><<<(unsigned)grid, kThreads, 0, s>>>(a);
  else if (F32 || p.blocks == 2) attend_kernel<D, F32, kMost < 2 ? kMost : 2, kWaves><<<(unsigned)grid, kThreads, 0, s>>>(a);
  else attend_kernel<D, F32, kMost, kWaves><<<(unsigned)grid, kThreads, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.total == 0) return e;   // one run: nothing to join
  // Pieces of a row: about the runs over the sequences.  A workgroup a row where few rows have
  // many (32 rows of 64 pieces: 5 us); where the rows are many for their pieces it would be all
  // launch (4096 rows of 8 pieces 24 us, 20000 of 9 86 us; eight rows a workgroup 6 and 9 us).
  constexpr int kRows = 256 / (D / 4);
  const int64_t rows = a.q_len * a.group, pieces = a.target / a.n;
  const bool many = pieces >= 8 && rows * a.c.heads * a.n * a.layers <= 32 * pieces;
  const int64_t blocks = many ? rows : (rows + kRows - 1) / kRows;
  const int64_t g2 = blocks * a.c.heads * a.n * a.layers;
  if (g2 * 256 > kMaxThreads) return hipErrorInvalidValue;
  if (many)
    attend_join_kernel<D, F32, kRows><<<(unsigned)g2, 256, 0, s>>>(a, (uint32_t)blocks);
  else
    attend_join_kernel<D, F32, 1><<<(unsigned)g2, 256, 0, s>>>(a, (uint32_t)blocks);
  return hipGetLastError();
}

}  // namespace

// Workgroups at a time: 256 compute units with two each, and with three of the 16-row kernels at
// D = 64, whose steps are half the bytes: 64 sequences up to 16384 positions at D = 64 take 75.0 us
// so and 78.2 with two; at D = 128 one of 32768 takes 16.9 us with three and 15.6 with two, its fp32 form 20.9
// and 16.9 (fewer pieces to join).
constexpr int64_t kUnits = 256;
constexpr int64_t kFewSteps = 24;
// Rounds of the shortest run, where a table is short for as many runs as the device holds: one
// sequence of 4096 positions takes 9.4 us in runs of one round, 9.7 of two, 11.1 of four, 13.1 of eight; one
// of 8192 11.1, 10.2, 11.2 and 14.1, two of 4096 12.6, 11.7, 13.1 and 14.9.
constexpr int64_t kShortest = 2;
// Where no sequence can be longer than so many rounds, each stays whole, a run of its own, and
// nothing is joined: kWhole of them where the workgroups are few, up to kWholeFull where they
// fill half the device.  Decoding over 8 KV heads, cut and whole: one of 2048 positions 9.4 and
// 16.4 us; 16 of 1024 13.1 and 11.0, of 4096 21.2 and 28.9; 64 of 1024 20.4 and 16.6, of 4096 60.6 and
// 56.9.  128 tokens of 32 heads behind up to 300 positions, 64 times: 160 and 59.  On the border, 16 of
// 2048 (whole) lose a microsecond, 16.3 and 17.4, and one of 1024 two of them in a graph, 8.4 and 10.3, but
// gains one where the host has one launch less to make, 10.9 and 9.9.  Longer ones are cut however many they
// are: one among many short ones would be a single workgroup's work.
constexpr int64_t kWhole = 8, kWholeFull = 32;
// And where the waves that the device holds are taken often enough for their length, once for every
// kAlone rounds, a workgroup is one wave, which has its rows to itself: nothing meets in
// LDS.  With four waves and with one: 64 times 128 tokens of 32 heads over 300 positions 96 and 55 us,
// over 1000 143 and 118; 20 times over 1000 57 and 58, over 4000 131 and 191; 8 times over 300 15.7 and
// 23.1; 150 decoding over 256 positions 14.9 and 14.5, over 512 20.6 and 23.4.
constexpr int64_t kAlone = 8;

bool make_attend_plan(int layers, int n, int heads, int q_heads, int64_t q_len, int D, bool f32,
                      int64_t capacity, AttendPlan* p) {
  const int64_t rows = q_len * (q_heads / heads);
  const int64_t units = (int64_t)heads * layers * n;
  if (rows > (1 << 26) || units > 0x7fffffff) return false;
  // no run shorter than kShortest rounds even where every sequence is full
  const int64_t most = (int64_t)n * ((capacity + kShortest * kRound - 1) / (kShortest * kRound));
  // Blocks of a wave share a step's conversions (64 instructions); with fp32 rows two do not fit the
  // registers at D = 128.  A call that cannot fill the device takes one block to a wave: more
  // workgroups, each sooner done (32 fp32 rows over 512 positions: 7.2 us, 10.3 with two).
  const int64_t single = (rows + 15) / 16 * heads * layers;
  // And one of few steps a SIMD takes two blocks rather than four, whose beginning and end weigh
  // more than the conversions they spare: 256 tokens of 32 heads behind 1024 positions (4 steps of
  // 64 rows) 14.5 and 21.1 us, 64 behind 8192 (8) 26.4 and 31.8, 32 behind 32768 (16) 37.0 and
  // 39.2, 64 behind 32768 (32) 57.0 and 53.8.
  const int64_t steps = (capacity + kStep - 1) / kStep, quads = (rows + 63) / 64;
  const bool few = quads * units <= kFewSteps * 4 * kUnits / steps;
  p->blocks = rows <= 16 || (f32 && D == 128) || (single <= kUnits && single * most <= kUnits)
                  ? 1 : rows <= 32 || f32 || few ? 2 : 4;
  const int64_t per = p->blocks * 16;
  const int64_t tiles = (rows + per - 1) / per;
  const int64_t sets = tiles * heads * layers;
  const int64_t resident = kUnits * (p->blocks == 1 && D == 64 ? 3 : 2);
  // Workgroups run in rounds of `resident`: the number of runs that leaves least of the last
  // one idle, the pieces of a further run counting for a fiftieth.
  int64_t target = 1;
  double best = 0.0;
  const int64_t first = resident / sets > 1 ? resident / sets : 1;
  for (int64_t t = first; t <= first + 7; ++t) {
    const int64_t turns = (sets * t + resident - 1) / resident;
    const double used = (double)(sets * t) / (double)(turns * resident) - 0.02 * (double)(t - first);
    if (used > best) {
      best = used;
      target = t;
    }
  }
  if (target > most) target = most;
  const int64_t longest = (capacity + kRound - 1) / kRound, groups = sets * n;
  if (n * longest > 0x7fffffff) return false;   // rounds are counted in 32 bits
  p->whole = longest <= kWholeFull && groups * kThreads <= kMaxThreads &&
             longest <= kWhole + (kWholeFull - kWhole) * groups / (resident / 2);
  if (p->whole) target = n;
  const int64_t waves = kWaves * kUnits * (p->blocks == 1 ? 3 : 2);   // that the device holds
  p->alone = p->whole && longest * waves <= kAlone * groups;
  const bool joins = target > 1 && !p->whole;
  p->room = (int32_t)capacity;   // below 2^31 - 2^16
  p->row_tiles = (int32_t)tiles;
  p->rows_pad = (int32_t)(tiles * per);
  p->target = (int32_t)target;
  p->slots = (int32_t)(target + n);
  // threads of the two grids
  const int64_t joined = 256 / (D / 4);   // rows a workgroup of the join
  if (sets * p->slots > 0x7fffffff || rows * units > 0x7fffffff ||
      sets * target * kThreads > kMaxThreads ||
      (joins && (rows + joined - 1) / joined * units * 256 > kMaxThreads))
    return false;
  const size_t cells = (size_t)layers * heads * p->slots * p->rows_pad;
  p->off_ml = joins ? cells * (size_t)D * sizeof(float) : 0;
  p->total = joins ? p->off_ml + ((cells * sizeof(float2) + 15) & ~(size_t)15) : 0;
  return true;
}

hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, bool f32, hipStream_t s) {
  if (a.c.D == 64)
    return f32 ? launch<64, true>(a, p, s) : launch<64, false>(a, p, s);
  return f32 ? launch<128, true>(a, p, s) : launch<128, false>(a, p, s);
}

}  // namespace cb
