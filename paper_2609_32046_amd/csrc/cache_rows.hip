// Rows into and out of the four-bit cache (gfx950).
//
// Eight lanes' worth of a row: a lane holds eight of its values, so that a
// group of 32 values that share a scale is four lanes, and their largest
// magnitude two lane exchanges away.  A wave holds consecutive positions of
// one head: key codes are stored as one contiguous piece, value codes into the
// 4-position blocks that the attention kernel loads as 16 bytes a lane.
// Bound by HBM: 2 or 4 bytes of a row's value for 17/32 byte of cache.  The rows go past
// the caches: the 302 MB of 2048 positions of the 8B shape are written in 74 us and read in 55
// (5.2 and 6.9 TB/s with the cache's bytes), against 85 and 89 through them; at 9 MB there is
// no difference.  Two or four items a thread were no faster.
#include "cache.h"

namespace cb {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

// Where a row's codes and scales live.
struct Place {
  bool held;
  unsigned char* unit;
  int at;   // position within the page
};

__device__ inline Place place_of(const CacheView& c, int seq, int64_t pos, int layer, int head) {
  Place r;
  r.at = (int)(pos & ((1 << c.page_shift) - 1));
  const int64_t slot = pos >> c.page_shift;
  r.held = pos >= 0 && slot < c.width && (unsigned)seq < (unsigned)c.seqs;
  const int page = r.held ? c.table[(int64_t)seq * c.width + slot] : -1;
  r.held = r.held && (unsigned)page < (unsigned)c.pages;
  r.unit = c.pool + (r.held ? page : 0) * c.page_bytes +
           (int64_t)(layer * c.heads + head) * c.unit_bytes;
  return r;
}

// Work of a lane: row (layer, entry, head, t) and its eight values from 8 * sub.
struct Item {
  bool live;
  int layer, entry, head, sub;
  int64_t t;
};

template <int D>
__device__ inline Item item_of(const CacheRowsArgs& a, int64_t thread) {
  constexpr int kLanes = D / 8;
  Item it;
  it.sub = (int)(thread & (kLanes - 1));
  const int64_t row = thread / kLanes;
  const int64_t rows = (int64_t)a.layers * a.n * a.c.heads * a.max_count;
  it.live = row < rows;
  int64_t u;
  if (rows <= 0x7fffffff) {
    u = (uint32_t)row / (uint32_t)a.max_count;
  } else {
    u = row / a.max_count;
  }
  it.t = row - u * a.max_count;
  const uint32_t w = (uint32_t)u;   // at most layers * n * heads < 2^31
  const uint32_t eh = w / (uint32_t)a.c.heads;
  it.head = (int)(w - eh * a.c.heads);
  it.layer = (int)(eh / (uint32_t)a.n);
  it.entry = (int)(eh - (uint32_t)it.layer * a.n);
  return it;
}

// Sequence and position of an item; not live behind its entry's rows.
__device__ inline int64_t position_of(const CacheRowsArgs& a, Item* it, int* seq) {
  int64_t count = a.max_count;
  if (a.counts) count = a.counts[it->entry] < count ? a.counts[it->entry] : count;
  it->live = it->live && it->t < count;
  *seq = a.seqs ? a.seqs[it->entry] : it->entry;
  const bool known = (unsigned)*seq < (unsigned)a.c.seqs;
  const int64_t first = a.start ? (int64_t)a.start[it->entry]
                                : (known ? (int64_t)a.c.lens[*seq] : 0) - count;
  return first + it->t;
}

template <typename T>
__device__ inline void load8(const T* p, float x[8]);
template <>
__device__ inline void load8<float>(const float* p, float x[8]) {
  const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
  const f32x4 b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}
template <>
__device__ inline void load8<__bf16>(const __bf16* p, float x[8]) {
  const u32x4 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(a[i] << 16);
    x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
  }
}

// Codes of eight values and the group's scale byte.  The scale: the least e
// with max|x| <= 1.75 * 2^(e + 2), so that every value lies within half a step
// (of the step between 4 and 6) of a code, the largest included.
__device__ inline uint32_t encode8(const float x[8], int* scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    top = b > top ? b : top;
  }
  uint32_t o = (uint32_t)__shfl_xor((int)top, 1);
  top = o > top ? o : top;
  o = (uint32_t)__shfl_xor((int)top, 2);
  top = o > top ? o : top;
  if (top >= 0x7f800000u) {   // a NaN or an infinity: the whole group reads as NaN
    *scale = 255;
    return 0u;
  }
  int e = (int)(top >> 23) - 129 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = e < -124 ? -124 : e > 125 ? 125 : e;
  *scale = e + 127;
  const float s = __uint_as_float((uint32_t)(e + 127) << 23);
  uint32_t r = 0;
  // nearest, ties to even, saturating at 6; the scale's exponent only counts
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
  return r;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CacheRowsArgs a) {
  Item it = item_of<D>(a, (int64_t)blockIdx.x * kThreads + threadIdx.x);
  if (!it.live) return;   // whole rows, so whole groups of four lanes
  int seq;
  const int64_t pos = position_of(a, &it, &seq);
  if (!it.live) return;
  const int64_t off = it.layer * a.stride[0] + it.entry * a.stride[1] + it.head * a.stride[2] +
                      it.t * a.stride[3] + it.sub * 8;
  float xk[8], xv[8];
  load8<T>(static_cast<const T*>(a.k) + off, xk);
  load8<T>(static_cast<const T*>(a.v) + off, xv);
  const Place pl = place_of(a.c, seq, pos, a.layer0 + it.layer, it.head);
  int sk, sv;
  const uint32_t ck = encode8(xk, &sk), cv = encode8(xv, &sv);
  if (!pl.held) return;
  const int P = 1 << a.c.page_shift;
  constexpr int G = D / 32;
  *reinterpret_cast<uint32_t*>(pl.unit + pl.at * (D / 2) + it.sub * 4) = ck;
  unsigned char* vc = pl.unit + unit_value_codes(P, D) + (pl.at >> 2) * (2 * D);
  if (D == 128) {
    *reinterpret_cast<uint32_t*>(vc + it.sub * 16 + (pl.at & 3) * 4) = cv;
  } else {   // two runs of four values
    *reinterpret_cast<uint16_t*>(vc + it.sub * 16 + (pl.at & 3) * 2) = (uint16_t)cv;
    *reinterpret_cast<uint16_t*>(vc + it.sub * 16 + 8 + (pl.at & 3) * 2) = (uint16_t)(cv >> 16);
  }
  if ((it.sub & 3) == 0) {
    const int g = it.sub >> 2;
    pl.unit[unit_key_scales(P, D) + pl.at * G + g] = (unsigned char)sk;
    pl.unit[unit_value_scales(P, D) + ((pl.at >> 2) * G + g) * 4 + (pl.at & 3)] =
        (unsigned char)sv;
  }
}

template <typename T>
__device__ inline void decode8(uint32_t c, int scale, T* p);
template <>
__device__ inline void decode8<__bf16>(uint32_t c, int scale, __bf16* p) {
  const float s = __uint_as_float((uint32_t)scale << 23);
  bf16x2 r[4];
  r[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
  r[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
  r[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
  r[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
  __builtin_nontemporal_store(*reinterpret_cast<u32x4*>(r), reinterpret_cast<u32x4*>(p));
}
template <>
__device__ inline void decode8<float>(uint32_t c, int scale, float* p) {
  const float s = __uint_as_float((uint32_t)scale << 23);
  f32x2 r[4];
  r[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0);
  r[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
  r[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2);
  r[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
  f32x4 a = {r[0][0], r[0][1], r[1][0], r[1][1]}, b = {r[2][0], r[2][1], r[3][0], r[3][1]};
  __builtin_nontemporal_store(a, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(b, reinterpret_cast<f32x4*>(p + 4));
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheRowsArgs a) {
  Item it = item_of<D>(a, (int64_t)blockIdx.x * kThreads + threadIdx.x);
  if (!it.live) return;
  int seq;
  const int64_t pos = position_of(a, &it, &seq);
  if (!it.live) return;
  const int64_t off = it.layer * a.stride[0] + it.entry * a.stride[1] + it.head * a.stride[2] +
                      it.t * a.stride[3] + it.sub * 8;
  Place pl = place_of(a.c, seq, pos, a.layer0 + it.layer, it.head);
  const bool held = pl.held && pos < a.c.lens[seq];
  const int P = 1 << a.c.page_shift;
  constexpr int G = D / 32;
  uint32_t ck = 0, cv = 0;
  int sk = 0, sv = 0;
  if (held) {
    const int g = it.sub >> 2;
    ck = *reinterpret_cast<const uint32_t*>(pl.unit + pl.at * (D / 2) + it.sub * 4);
    const unsigned char* vc = pl.unit + unit_value_codes(P, D) + (pl.at >> 2) * (2 * D);
    if (D == 128) {
      cv = *reinterpret_cast<const uint32_t*>(vc + it.sub * 16 + (pl.at & 3) * 4);
    } else {
      cv = *reinterpret_cast<const uint16_t*>(vc + it.sub * 16 + (pl.at & 3) * 2) |
           (uint32_t)*reinterpret_cast<const uint16_t*>(vc + it.sub * 16 + 8 + (pl.at & 3) * 2)
               << 16;
    }
    sk = pl.unit[unit_key_scales(P, D) + pl.at * G + g];
    sv = pl.unit[unit_value_scales(P, D) + ((pl.at >> 2) * G + g) * 4 + (pl.at & 3)];
  }
  decode8<T>(ck, sk, static_cast<T*>(const_cast<void*>(a.k)) + off);
  decode8<T>(cv, sv, static_cast<T*>(const_cast<void*>(a.v)) + off);
}

template <typename F64, typename F128>
hipError_t launch_rows(const CacheRowsArgs& a, F64 f64, F128 f128, hipStream_t s) {
  const int64_t rows = (int64_t)a.layers * a.n * a.c.heads * a.max_count;
  if (rows == 0) return hipSuccess;
  const int64_t blocks = (rows * (a.c.D / 8) + kThreads - 1) / kThreads;
  if (blocks * kThreads > kMaxThreads) return hipErrorInvalidValue;
  if (a.c.D == 64) f64<<<(unsigned)blocks, kThreads, 0, s>>>(a);
  else f128<<<(unsigned)blocks, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheRowsArgs& a, bool f32, hipStream_t s) {
  return f32 ? launch_rows(a, cache_write_kernel<float, 64>, cache_write_kernel<float, 128>, s)
             : launch_rows(a, cache_write_kernel<__bf16, 64>, cache_write_kernel<__bf16, 128>, s);
}

hipError_t launch_cache_read(const CacheRowsArgs& a, bool f32, hipStream_t s) {
  return f32 ? launch_rows(a, cache_read_kernel<float, 64>, cache_read_kernel<float, 128>, s)
             : launch_rows(a, cache_read_kernel<__bf16, 64>, cache_read_kernel<__bf16, 128>, s);
}

}  // namespace cb
