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
// g) takes values g*D/4.. of its key, one 16-byte load with one scale; in the second the
// lanes r of a tile take values r*D/16 + tile, so that a lane's values are
// neighbours too: 16 bytes are four positions of them, with one group's scales.
// Codes become bf16 by conversion with their scale, exactly.
//
// The positions of all sequences are cut into chunks of equal length, as many
// as fill the device (each workgroup finds its own chunk from the lengths), and
// four waves take a chunk's steps in turn; their results meet in LDS, and
// those of several chunks in a second, small kernel.
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

// A chunk of a sequence: batch row, its index among the row's chunks, how many there are.
struct Chunk {
  int b, index, count, len;
};

__device__ inline int seq_len(const AttendArgs& a, int b) {
  const int s = a.seqs ? a.seqs[b] : b;
  if ((unsigned)s >= (unsigned)a.c.seqs) return 0;
  const int len = a.c.lens[s];
  const int64_t room = (int64_t)a.c.width << a.c.page_shift;
  return len < 0 ? 0 : (int64_t)len < room ? len : (int)room;
}

__device__ inline int query_tokens(const AttendArgs& a, int b) {
  const int m = a.q_lens ? a.q_lens[b] : (int)a.q_len;
  return m < 0 ? 0 : m < (int)a.q_len ? m : (int)a.q_len;
}

// Chunk length: the positions of all rows over the chunks wanted, in whole rounds, at
// least two.
__device__ inline int chunk_len(int64_t total, int target) {
  const int64_t c = (total + target - 1) / target;
  const int64_t r = (c + kRound - 1) / kRound * kRound;
  return r < 2 * kRound ? 2 * kRound : (int)(r < 0x7fffff00 ? r : 0x7fffff00);
}
__device__ inline int chunks_of(int len, int c) {
  return len <= c ? 1 : (int)(((int64_t)len + c - 1) / c);
}

__device__ inline int64_t wave_sum64(int64_t x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

// The chunk of slot `slot`, by one wave: every wave works it out for itself.  False
// behind the last chunk.  *size: the chunk length.
__device__ inline bool find_chunk(const AttendArgs& a, int slot, Chunk* ch, int* size) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int i = lane; i < a.n; i += 64) total += seq_len(a, i);
  const int c = chunk_len(wave_sum64(total), a.target);
  *size = c;
  int before = 0;
  for (int i0 = 0; i0 < a.n; i0 += 64) {
    const int i = i0 + lane;
    const int len = i < a.n ? seq_len(a, i) : 0;
    const int k = i < a.n ? chunks_of(len, c) : 0;
    int incl = k;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(incl, d);
      if (lane >= d) incl += y;
    }
    const uint64_t mine = __ballot(i < a.n && before + incl > slot);
    if (mine) {
      const int l = __ffsll((unsigned long long)mine) - 1;
      ch->b = i0 + l;
      ch->count = __shfl(k, l);
      ch->index = slot - (before + __shfl(incl, l) - ch->count);
      ch->len = __shfl(len, l);
      return true;
    }
    before += __shfl(incl, 63);
  }
  return false;
}

// What a step reads, as it lies in memory: per half (16 positions) a lane's key codes,
// key scale, value codes of four positions and their scales.
template <int D>
struct Raw {
  uint32_t k[2][D / 32], v[2][D / 32];
  uint32_t ks[2], vs[2];
};

template <int D>
__device__ inline void load_half(const unsigned char* unit, int P, int at, int r, int g, Raw<D>* w,
                                 int h) {
  const unsigned char* kp = unit + at * (D / 2) + r * (D / 2) + g * (D / 8);
  const unsigned char* vp = unit + unit_value_codes(P, D) + (at >> 2) * (2 * D) + g * (2 * D) +
                            r * (D / 8);
  if constexpr (D == 128) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(kp), y = *reinterpret_cast<const u32x4*>(vp);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w->k[h][i] = x[i];
      w->v[h][i] = y[i];
    }
  } else {
    const u32x2 x = *reinterpret_cast<const u32x2*>(kp), y = *reinterpret_cast<const u32x2*>(vp);
    w->k[h][0] = x[0];
    w->k[h][1] = x[1];
    w->v[h][0] = y[0];
    w->v[h][1] = y[1];
  }
  constexpr int G = D / 32;
  const int kg = g * G / 4, vg = r * G / 16;
  w->ks[h] = unit[unit_key_scales(P, D) + (at + r) * G + kg];
  w->vs[h] = *reinterpret_cast<const uint32_t*>(unit + unit_value_scales(P, D) +
                                                (((at >> 2) + g) * G + vg) * 4);
}

template <bool F32>
struct RowType;
template <>
struct RowType<false> { typedef __bf16 type; };
template <>
struct RowType<true> { typedef float type; };

// Values of one tile pair (values 2b and 2b + 1 of the lane's run) for the step's 32 positions:
// conversions give (value 2b, value 2b+1) of a position; the product wants pairs of
// positions.
template <int D>
__device__ inline void value_tiles(const Raw<D>& w, const float vscale[8], int b, bf16x8* even,
                                   bf16x8* odd) {
  u32x4 lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {   // positions 2i, 2i + 1 of the lane's eight
    const int h = i >> 1, e = (2 * i) & 3;
    uint32_t x, y;
    if constexpr (D == 128) {     // a dword a position
      x = u32_of(cvt2(w.v[h][e], vscale[2 * i], b));
      y = u32_of(cvt2(w.v[h][e + 1], vscale[2 * i + 1], b));
    } else {                      // two bytes a position
      x = u32_of(cvt2(w.v[h][e >> 1], vscale[2 * i], b));
      y = u32_of(cvt2(w.v[h][e >> 1], vscale[2 * i + 1], 2 + b));
    }
    lo[i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
    hi[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
  *even = __builtin_bit_cast(bf16x8, lo);
  *odd = __builtin_bit_cast(bf16x8, hi);
}

template <int D, bool F32, int RT>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendArgs a) {
  typedef typename RowType<F32>::type T;
  constexpr int KS = D / 32;              // first product: MFMAs of a block and half
  constexpr int VT = D / 16;              // second: tiles of 16 values
  constexpr int NQ = F32 ? 3 : 1;
  constexpr int kPad = 4;
  __shared__ float so[kWaves][16][D + kPad];
  __shared__ float sm[kWaves][RT * 16], sl[kWaves][RT * 16];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  // heads fastest: the units of a page lie side by side, and with eight heads
  // each L2 (one per XCD, workgroups in turn) sees one head's positions
  uint32_t id = blockIdx.x;
  const int head = (int)(id % (uint32_t)a.c.heads);
  id /= (uint32_t)a.c.heads;
  const int tile = (int)(id % (uint32_t)a.row_tiles);
  id /= (uint32_t)a.row_tiles;
  const int slot = (int)(id % (uint32_t)a.slots);
  const int layer = (int)(id / (uint32_t)a.slots);

  Chunk ch;
  int size;
  if (!find_chunk(a, slot, &ch, &size)) return;
  const int G = a.group;
  const int m = query_tokens(a, ch.b);
  const int rows = m * G;   // at most 2^26
  const int row0 = tile * (RT * 16);
  if (row0 >= rows) return;   // also m <= 0; uniform over the workgroup
  const int seq = a.seqs ? a.seqs[ch.b] : ch.b;
  const int P = 1 << a.c.page_shift;

  // Limits of this lane's rows; the positions that any row of the tile sees, and that all see.
  const int64_t first = (int64_t)ch.index * size;
  int lo64 = (int)first;
  const int end = (int)(first + size < ch.len ? first + size : (int64_t)ch.len);
  int limit[RT];
  const T* qp[RT];
  bool live[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = row0 + t * 16 + r;
    live[t] = row < rows;
    const int tok = live[t] ? row / G : 0;
    const int qh = head * G + (live[t] ? row - tok * G : 0);
    const int64_t see = a.causal ? (int64_t)ch.len - m + tok + 1 : (int64_t)ch.len;
    limit[t] = !live[t] ? 0 : see < end ? (int)(see > 0 ? see : 0) : end;
    qp[t] = static_cast<const T*>(a.q) + layer * a.q_stride[0] + ch.b * a.q_stride[1] +
            qh * a.q_stride[2] + tok * a.q_stride[3];
  }
  // rows ascend with tokens, so the first row sees least, the last live one most
  const int tok_first = row0 / G;
  const int row_last = (row0 + RT * 16 < rows ? row0 + RT * 16 : rows) - 1;
  const int64_t see_first = a.causal ? (int64_t)ch.len - m + tok_first + 1 : (int64_t)ch.len;
  const int64_t see_last = a.causal ? (int64_t)ch.len - m + row_last / G + 1 : (int64_t)ch.len;
  const int full = (int)(see_first < end ? (see_first > 0 ? see_first : 0) : end);
  const int hi = (int)(see_last < end ? (see_last > 0 ? see_last : 0) : end);

  // Queries: values g * D/4 + 8j .. of the lane's row, the keys' own order.
  bf16x8 q[RT][KS][NQ];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      if constexpr (F32) {
        f32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
        if (live[t]) {
          x = *reinterpret_cast<const f32x4*>(qp[t] + g * (D / 4) + 8 * j);
          y = *reinterpret_cast<const f32x4*>(qp[t] + g * (D / 4) + 8 * j + 4);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float u0, u1, u2;
          split3(i < 4 ? x[i & 3] : y[i & 3], &u0, &u1, &u2);
          q[t][j][0][i] = (__bf16)u0;
          q[t][j][1][i] = (__bf16)u1;
          q[t][j][2][i] = (__bf16)u2;
        }
      } else {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (live[t]) x = *reinterpret_cast<const u32x4*>(qp[t] + g * (D / 4) + 8 * j);
        q[t][j][0] = __builtin_bit_cast(bf16x8, x);
      }
    }

  float top[RT], sum[RT];
  f32x4 o[RT][VT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    top[t] = kNone;
    sum[t] = 0.f;
#pragma unroll
    for (int i = 0; i < VT; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const unsigned char* pool = a.c.pool + ((int64_t)(a.layer0 + layer) * a.c.heads + head) *
                                             a.c.unit_bytes;
  const int32_t* row_pages = a.c.table + (int64_t)seq * a.c.width;
  const int steps = hi <= lo64 ? 0 : (hi - lo64 + kRound - 1) / kRound;   // rounds
  int ids = 0;   // lane 2k, 2k+1: pages of the halves of round k of the next 32
  Raw<D> cur, nxt;
  auto ids_for = [&](int k0) {
    const int64_t p = (int64_t)lo64 + (int64_t)(k0 + (lane >> 1)) * kRound + wave * kStep +
                      (lane & 1) * 16;
    ids = p < hi ? row_pages[p >> a.c.page_shift] : -1;
  };
  // A half without a page (behind the end, or a table entry that is none) reads
  // page 0, in bounds, and is masked.
  auto fetch = [&](int k, Raw<D>* w) {
    const int t0 = lo64 + k * kRound + wave * kStep;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int id0 = __builtin_amdgcn_readlane(ids, 2 * (k & 31) + h);
      const int pg = (unsigned)id0 < (unsigned)a.c.pages ? id0 : 0;
      load_half<D>(pool + pg * a.c.page_bytes, P, (t0 + h * 16) & (P - 1), r, g, w, h);
    }
  };
  auto valid = [&](int k, int h) {
    return (unsigned)__builtin_amdgcn_readlane(ids, 2 * (k & 31) + h) < (unsigned)a.c.pages;
  };

  if (steps > 0) {
    ids_for(0);
    fetch(0, &cur);
  }
  bool ok0 = steps > 0 && valid(0, 0), ok1 = steps > 0 && valid(0, 1);
  for (int k = 0; k < steps; ++k) {
    const int t0 = lo64 + k * kRound + wave * kStep;
    const bool here0 = ok0, here1 = ok1;
    if (k + 1 < steps) {
      if (((k + 1) & 31) == 0) ids_for(k + 1);
      fetch(k + 1, &nxt);
      ok0 = valid(k + 1, 0);
      ok1 = valid(k + 1, 1);
    }
    if (t0 < hi) {
      const bool masked = t0 + kStep > full || !here0 || !here1;   // uniform
      float vscale[8];
      uint32_t nan_bits = 0;   // positions of the lane whose value group reads as NaN
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t b = (cur.vs[i >> 2] >> (8 * (i & 3))) & 255u;
        if (masked) {
          const int pos = t0 + (i >> 2) * 16 + 4 * g + (i & 3);
          const bool in = pos < hi && (i < 4 ? here0 : here1);
          // what a masked position holds counts for nothing: 0 times a NaN or an
          // infinity would be NaN
          if (in && b == 255u) nan_bits |= 1u << i;
          if (!in || b == 255u) b = 0u;
        }
        vscale[i] = __uint_as_float(b << 23);
      }
      bf16x8 kk[2][KS];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float s = __uint_as_float(cur.ks[h] << 23);
#pragma unroll
        for (int j = 0; j < KS; ++j) kk[h][j] = expand8(cur.k[h][j], s);
      }
      bf16x8 p[RT][NQ];
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
              s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[h][j], q[t][j][u], s[h], 0, 0, 0);
        }
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[i >> 2][i & 3] * a.c2;
        if (masked) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int pos = t0 + (i >> 2) * 16 + 4 * g + (i & 3);
            if (pos >= limit[t] || !(i < 4 ? here0 : here1)) x[i] = -INFINITY;
          }
        }
        float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                         fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
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
        for (int i = 0; i < 8; ++i) {
          e[i] = __builtin_amdgcn_exp2f(x[i] - top[t]);
        }
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
          // the weights' rounding: at most 2^-9 of each, in either direction, under
          // the rounding of the bf16 output itself
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = pack_bf16(e[2 * i], e[2 * i + 1]);
          p[t][0] = __builtin_bit_cast(bf16x8, w);
        }
      }
#pragma unroll
      for (int b = 0; b < VT / 2; ++b) {
        bf16x8 even, odd;
        value_tiles<D>(cur, vscale, b, &even, &odd);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int u = NQ - 1; u >= 0; --u) {
            o[t][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, p[t][u], o[t][2 * b], 0, 0, 0);
            o[t][2 * b + 1] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, p[t][u], o[t][2 * b + 1], 0, 0, 0);
          }
      }
      if (masked && __any(nan_bits != 0)) {
        // a value that reads as NaN reaches the rows that see its position, in its group
        constexpr int kRun = 16 / (D / 32);               // lanes r of one group
        const int r0 = (g * (D / 32) / 4) * kRun;         // the group that this lane's outputs lie in
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
          const uint64_t who = __ballot((nan_bits >> i) & 1u);
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
    }
    cur = nxt;
  }

  // The four lane groups' sums, then the four waves' results.
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    sum[t] += __shfl_xor(sum[t], 16);
    sum[t] += __shfl_xor(sum[t], 32);
    if (g == 0) {
      sm[wave][t * 16 + r] = top[t];
      sl[wave][t * 16 + r] = sum[t];
    }
  }
  const bool whole = ch.count == 1;
  const int64_t out_slot = ((int64_t)layer * a.c.heads + head) * a.slots + slot;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int v = 0; v < VT; v += 4) {
        // values (4g + i) * D/16 + v ..: one from each of four tiles
        const f32x4 x = {o[t][v][i], o[t][v + 1][i], o[t][v + 2][i], o[t][v + 3][i]};
        *reinterpret_cast<f32x4*>(&so[wave][r][(4 * g + i) * VT + v]) = x;
      }
    __syncthreads();
    // thread: row tid / 16, D/16 of its values
    const int qr = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * VT;
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
        const int tok = row / G;
        const int qh = head * G + row - tok * G;
        T* out = static_cast<T*>(a.out) + layer * a.out_stride[0] + ch.b * a.out_stride[1] +
                 qh * a.out_stride[2] + tok * a.out_stride[3] + d0;
        if constexpr (F32) {
#pragma unroll
          for (int v = 0; v < VT; v += 4)
            *reinterpret_cast<f32x4*>(out + v) =
                f32x4{acc[v] * inv, acc[v + 1] * inv, acc[v + 2] * inv, acc[v + 3] * inv};
        } else {
          uint32_t w[VT / 2];
#pragma unroll
          for (int v = 0; v < VT; v += 2) w[v / 2] = pack_bf16(acc[v] * inv, acc[v + 1] * inv);
          if constexpr (D == 128)
            *reinterpret_cast<u32x4*>(out) = u32x4{w[0], w[1], w[2], w[3]};
          else
            *reinterpret_cast<u32x2*>(out) = u32x2{w[0], w[1]};
        }
        if (a.lse && (threadIdx.x & 15) == 0)
          a.lse[(((int64_t)layer * a.n + ch.b) * a.q_heads + qh) * a.q_len + tok] =
              L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
      } else {
        const int64_t at = out_slot * a.rows_pad + row;
        float* po = a.part_o + at * D + d0;
#pragma unroll
        for (int v = 0; v < VT; v += 4)
          *reinterpret_cast<f32x4*>(po + v) = f32x4{acc[v], acc[v + 1], acc[v + 2], acc[v + 3]};
        if ((threadIdx.x & 15) == 0) a.part_ml[at] = make_float2(M, L);
      }
    }
  }
}

// Rows of sequences that were cut into several chunks: D/4 lanes a row, chunks in order.
template <int D, bool F32>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, int64_t blocks_per_row_set) {
  typedef typename RowType<F32>::type T;
  constexpr int kLanes = D / 4, kRows = 256 / kLanes;
  uint32_t id = blockIdx.x;
  const int64_t rb = id % (uint32_t)blocks_per_row_set;
  id /= (uint32_t)blocks_per_row_set;
  const int head = (int)(id % (uint32_t)a.c.heads);
  id /= (uint32_t)a.c.heads;
  const int b = (int)(id % (uint32_t)a.n);
  const int layer = (int)(id / (uint32_t)a.n);
  // the row's first slot and its chunks
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int i = lane; i < a.n; i += 64) total += seq_len(a, i);
  const int c = chunk_len(wave_sum64(total), a.target);
  int64_t before = 0;
  for (int i = lane; i < b; i += 64) before += chunks_of(seq_len(a, i), c);
  const int slot0 = (int)wave_sum64(before);
  const int count = chunks_of(seq_len(a, b), c);
  if (count == 1) return;
  const int rows = query_tokens(a, b) * a.group;
  const int row = (int)(rb * kRows) + (int)(threadIdx.x / kLanes);
  if (row >= rows) return;
  const int d0 = (threadIdx.x % kLanes) * 4;
  const int64_t base = ((int64_t)layer * a.c.heads + head) * a.slots + slot0;
  float M = kNone;
  for (int k = 0; k < count; ++k) M = fmaxf(M, a.part_ml[(base + k) * a.rows_pad + row].x);
  float L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < count; ++k) {
    const int64_t at = (base + k) * a.rows_pad + row;
    const float2 ml = a.part_ml[at];
    const float f = ml.x == M ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + at * D + d0);
    L += ml.y * f;
    acc += x * f;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int tok = row / a.group;
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
  const int64_t grid = (int64_t)a.c.heads * a.row_tiles * a.slots * a.layers;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (p.blocks == 1) attend_kernel<D, F32, 1><<<(unsigned)grid, kThreads, 0, s>>>(a);
  else attend_kernel<D, F32, 2><<<(unsigned)grid, kThreads, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t room = (int64_t)a.c.width << a.c.page_shift;
  if (a.target == 1 || room <= 2 * kRound) return hipSuccess;   // no sequence is cut
  const int64_t rows = a.q_len * a.group;
  const int64_t per = (rows + 256 / (D / 4) - 1) / (256 / (D / 4));
  const int64_t g2 = per * a.c.heads * a.n * a.layers;
  if (g2 > 0x7fffffff) return hipErrorInvalidValue;
  attend_join_kernel<D, F32><<<(unsigned)g2, 256, 0, s>>>(a, per);
  return hipGetLastError();
}

}  // namespace

// Workgroups that fill the device: 256 compute units, two workgroups each at a
// time, two rounds of them.
constexpr int64_t kFill = 1024;

bool make_attend_plan(int layers, int n, int heads, int q_heads, int64_t q_len, int D, bool f32,
                      int64_t capacity, AttendPlan* p) {
  const int64_t rows = q_len * (q_heads / heads);
  if (rows > (1 << 26)) return false;
  // two blocks share a step's conversions; with fp32 rows of 128 they do not fit the
  // registers (72 spills)
  p->blocks = rows <= 16 || (f32 && D == 128) ? 1 : 2;
  const int64_t per = p->blocks * 16;
  const int64_t tiles = (rows + per - 1) / per;
  int64_t target = kFill / (tiles * heads * layers);
  const int64_t most = (int64_t)n * ((capacity + 2 * kRound - 1) / (2 * kRound));
  target = target < 1 ? 1 : target > most ? most : target;
  p->row_tiles = (int32_t)tiles;
  p->rows_pad = (int32_t)(tiles * per);
  p->target = (int32_t)target;
  p->slots = (int32_t)(target + n);
  if ((int64_t)heads * tiles * p->slots * layers > 0x7fffffff) return false;
  const size_t cells = (size_t)layers * heads * p->slots * p->rows_pad;
  const bool cut = target > 1 && capacity > 2 * kRound;
  p->off_ml = cut ? cells * (size_t)D * sizeof(float) : 0;
  p->total = cut ? p->off_ml + ((cells * sizeof(float2) + 15) & ~(size_t)15) : 0;
  return true;
}

hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, bool f32, hipStream_t s) {
  if (a.c.D == 64)
    return f32 ? launch<64, true>(a, p, s) : launch<64, false>(a, p, s);
  return f32 ? launch<128, true>(a, p, s) : launch<128, false>(a, p, s);
}

}  // namespace cb
