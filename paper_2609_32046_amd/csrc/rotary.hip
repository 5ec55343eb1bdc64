// Rotary positions (gfx950): rows of up to two tensors, each pair of values
// turned by freq[i] * (pos - from).  A message's keys are bound by HBM: 2048 moved keys of 36 layers
// and 8 heads (302 MB in and out) take 55 us, 5.5 TB/s.  A step's rows are bound by the launch
// and its host side: 16 answers' queries and keys in 6 us.
#include <math.h>

#include "cache.h"

namespace cb {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kHeads = 4;   // rows of one position that a thread turns by the same angles
constexpr int64_t kStreamBytes = (int64_t)256 << 20;

// 16 bytes; STREAM: past the caches, for calls that would only flush them.
template <bool STREAM, typename V, typename T>
__device__ inline V get16(const T* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  return *reinterpret_cast<const V*>(p);
}
template <bool STREAM, typename V, typename T>
__device__ inline void put16(T* p, V x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<V*>(p));
  else *reinterpret_cast<V*>(p) = x;
}

// Eight consecutive values of a row, as they lie in memory.
template <typename T>
struct Vec8;
template <>
struct Vec8<float> {
  f32x4 a, b;
  __device__ void load_any(const float* p) { __builtin_memcpy(this, p, sizeof *this); }
  __device__ void store_any(float* p) const { __builtin_memcpy(p, this, sizeof *this); }
  template <bool S>
  __device__ void load(const float* p) {
    a = get16<S, f32x4>(p);
    b = get16<S, f32x4>(p + 4);
  }
  template <bool S>
  __device__ void store(float* p) const {
    put16<S>(p, a);
    put16<S>(p + 4, b);
  }
  __device__ float get(int i) const { return i < 4 ? a[i & 3] : b[i & 3]; }
  __device__ void set(const float* x) {
    a = f32x4{x[0], x[1], x[2], x[3]};
    b = f32x4{x[4], x[5], x[6], x[7]};
  }
};
template <>
struct Vec8<__bf16> {
  u32x4 a;
  __device__ void load_any(const __bf16* p) { __builtin_memcpy(this, p, sizeof *this); }
  __device__ void store_any(__bf16* p) const { __builtin_memcpy(p, this, sizeof *this); }
  template <bool S>
  __device__ void load(const __bf16* p) { a = get16<S, u32x4>(p); }
  template <bool S>
  __device__ void store(__bf16* p) const { put16<S>(p, a); }
  __device__ float get(int i) const {
    const uint32_t w = a[i >> 1];
    return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  __device__ void set(const float* x) {   // each value's one rounding
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 r = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
      a[i] = __builtin_bit_cast(uint32_t, r);
    }
  }
};

__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const __bf16* p) { return (float)*p; }

// Turns reduced in 64 bits (a position of 2^31 times a frequency keeps 22
// bits of the turn), then sine and cosine of the remainder by the hardware's
// instructions, which take turns: off by 1.25e-7 at most (over all multiples of 2^-25
// of a turn), two fp32 half steps at one.  They halve the time of moved keys, where
// every row has angles of its own, against sincospif.
__device__ inline void angle(double delta, double freq, float amplitude, float sign, float* cs,
                             float* sn) {
  const double t = delta * freq;
  const float r = (float)(t - rint(t));
  *cs = __builtin_amdgcn_cosf(r) * amplitude;
  *sn = __builtin_amdgcn_sinf(r) * (amplitude * sign);
}

// A piece of a row: mode 0, half layout with halves of whole vectors of eight: eight pairs
// from both halves, then copied vectors; 1, interleaved: eight consecutive values; 2, half
// layout with other halves: up to eight pairs, the upper ones from anywhere, then up to
// eight copied values.  Mode 2 is the slow one: its upper halves and copied values begin off any
// vector's border, and its last pairs are stored one by one.  2048 moved keys with 70 of 128 bf16 values
// turned (302 MB) take 103 us, with 64 of them 55; 38 of 64 fp32 values 94.
template <typename T, int MODE, bool STREAM>
struct Turn {
  static constexpr int PAIRS = MODE == 1 ? 4 : 8;

  // N rows of consecutive heads, chunk ch.  No branch between the loads: the rows, the positions
  // and the frequencies are all under way together.
  template <int N>
  __device__ static void rows(const RotaryArgs& a, const RotaryPart& p, const T* in, T* out,
                              const int32_t* pos, const int32_t* from, int ch) {
    const int half = a.R / 2;
    Vec8<T> lo[N], hi[MODE == 1 ? 1 : N];
    // mode 2: pairs of this piece; the last one, of fewer than eight, begins earlier so that it reads
    // eight too, and keeps those of its own
    const int some = half - ch * 8;
    const int base = MODE == 2 && some < 8 && half >= 8 ? half - 8 : ch * PAIRS;
    int64_t to[N], old[N];
    double freq[PAIRS];
#pragma unroll
    for (int h = 0; h < N; ++h) {
      const T* r = in + h * p.in_stride[1];
      if constexpr (MODE == 0) {
        lo[h].template load<STREAM>(r + ch * 8);
        hi[h].template load<STREAM>(r + half + ch * 8);
      } else if constexpr (MODE == 1) {
        lo[h].template load<STREAM>(r + ch * 8);
      } else if (half >= 8) {
        lo[h].load_any(r + base);
        hi[h].load_any(r + half + base);
      } else {
        float u[8] = {}, v[8] = {};
        for (int i = 0; i < half; ++i) {
          u[i] = load1(r + i);
          v[i] = load1(r + half + i);
        }
        lo[h].set(u);   // exact: the values are of this type
        hi[h].set(v);
      }
    }
#pragma unroll
    for (int h = 0; h < N; ++h) {
      to[h] = pos[h * p.pos_stride[1]];
      old[h] = 0;
    }
    if (from) {   // the same for all rows of the call
#pragma unroll
      for (int h = 0; h < N; ++h) old[h] = from[h * p.from_stride[1]];
    }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      const int pair = base + i;
      freq[i] = a.freq[MODE != 0 && pair >= half ? half - 1 : pair];
    }
    const bool shared = p.pos_stride[1] == 0 && (!from || p.from_stride[1] == 0);
    float cs[PAIRS], sn[PAIRS];
#pragma unroll
    for (int h = 0; h < N; ++h) {
      if (h == 0 || !shared) {
        const double delta = (double)(to[h] - old[h]);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i)
          angle(delta, freq[i], a.amplitude, a.sign, &cs[i], &sn[i]);
      }
      T* w = out + h * p.out_stride[1];
      if constexpr (MODE != 1) {
        float u[8], v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = lo[h].get(i), y = hi[h].get(i);
          u[i] = x * cs[i] - y * sn[i];
          v[i] = y * cs[i] + x * sn[i];
        }
        lo[h].set(u);
        hi[h].set(v);
        if (MODE == 0) {
          lo[h].template store<STREAM>(w + ch * 8);
          hi[h].template store<STREAM>(w + half + ch * 8);
        } else if (some >= 8) {
          lo[h].template store<STREAM>(w + ch * 8);
          hi[h].store_any(w + half + ch * 8);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (base + i >= ch * 8 && base + i < half) {
              w[base + i] = (T)u[i];
              w[half + base + i] = (T)v[i];
            }
        }
      } else {
        float u[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool turn = ch * 4 + i < half;   // pairs behind the rotated ones stay as they are
          const float x = lo[h].get(2 * i), y = lo[h].get(2 * i + 1);
          u[2 * i] = turn ? x * cs[i] - y * sn[i] : x;
          u[2 * i + 1] = turn ? y * cs[i] + x * sn[i] : y;
        }
        lo[h].set(u);
        lo[h].template store<STREAM>(w + ch * 8);
      }
    }
  }
};

template <typename T, int MODE, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  const RotaryPart& p = a.part[blockIdx.z];
  const int half = a.R / 2;
  const int turned = MODE == 1 ? a.D / 8 : (half + 7) / 8;
  const int copied = MODE == 1 ? 0 : (a.D - a.R + 7) / 8;
  const int64_t head_blocks = (p.size[1] + kHeads - 1) / kHeads;
  const int64_t outer = p.size[0] * head_blocks;
  int64_t t;
  int ch;
  if (copied == 0) {
    const int64_t items = p.size[2] * turned;
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (item >= items) return;
    t = items <= 0x7fffffff ? (int64_t)((uint32_t)item / (uint32_t)turned) : item / turned;
    ch = (int)(item - t * turned);
  } else {
    // Whole rows a workgroup, their turned pieces first, then their copied ones, so that one wave
    // at most does both: a quarter of 64 fp32 values turned (190 MB) takes 35 us so and 44 with a
    // row's pieces side by side, half of 128 bf16 values (336 MB) 62 and 64.
    const int rows = kThreads / (turned + copied);
    int at = threadIdx.x, per = turned;
    ch = 0;
    if (at >= rows * turned) {
      at -= rows * turned;
      ch = turned;
      per = copied;
    }
    if (at >= rows * per) return;
    const int row = (int)((uint32_t)at / (uint32_t)per);
    ch += at - row * per;
    t = (int64_t)blockIdx.x * rows + row;
    if (t >= p.size[2]) return;
  }
  for (int64_t y = blockIdx.y; y < outer; y += gridDim.y) {
    const int64_t o = outer <= 0x7fffffff
                          ? (int64_t)((uint32_t)y / (uint32_t)head_blocks) : y / head_blocks;
    const int64_t h0 = (y - o * head_blocks) * kHeads;
    const T* in = static_cast<const T*>(p.in) + o * p.in_stride[0] + h0 * p.in_stride[1] +
                  t * p.in_stride[2];
    T* out = static_cast<T*>(p.out) + o * p.out_stride[0] + h0 * p.out_stride[1] +
             t * p.out_stride[2];
    const int nh = (int)(p.size[1] - h0 < kHeads ? p.size[1] - h0 : kHeads);
    const int32_t* pos = p.pos + o * p.pos_stride[0] + h0 * p.pos_stride[1] + t * p.pos_stride[2];
    const int32_t* from = p.from ? p.from + o * p.from_stride[0] + h0 * p.from_stride[1] +
                                       t * p.from_stride[2]
                                 : nullptr;
    if (ch >= turned) {   // behind the rotated values
      for (int h = 0; h < nh; ++h) {
        const int at = a.R + (ch - turned) * 8;
        const T* from_row = in + h * p.in_stride[1] + at;
        T* to_row = out + h * p.out_stride[1] + at;
        Vec8<T> x;
        if (MODE == 0) {
          x.template load<STREAM>(from_row);
          x.template store<STREAM>(to_row);
        } else if (at + 8 <= a.D) {
          x.load_any(from_row);
          x.store_any(to_row);
        } else {
          for (int i = 0; i < 8 && at + i < a.D; ++i) to_row[i] = from_row[i];
        }
      }
    } else if (nh == kHeads) {
      Turn<T, MODE, STREAM>::template rows<kHeads>(a, p, in, out, pos, from, ch);
    } else {
      for (int h = 0; h < nh; ++h)
        Turn<T, MODE, STREAM>::template rows<1>(
            a, p, in + h * p.in_stride[1], out + h * p.out_stride[1], pos + h * p.pos_stride[1],
            from ? from + h * p.from_stride[1] : nullptr, ch);
    }
  }
}

template <typename T, bool STREAM>
void launch_mode(const RotaryArgs& a, int mode, dim3 grid, hipStream_t s) {
  if (mode == 0) rotary_kernel<T, 0, STREAM><<<grid, kThreads, 0, s>>>(a);
  else if (mode == 1) rotary_kernel<T, 1, STREAM><<<grid, kThreads, 0, s>>>(a);
  else rotary_kernel<T, 2, STREAM><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int parts, bool interleaved, bool f32,
                         hipStream_t s) {
  const int half = a.R / 2;
  const int mode = interleaved ? 1 : half % 8 == 0 ? 0 : 2;
  const int turned = mode == 1 ? a.D / 8 : (half + 7) / 8;
  const int copied = mode == 1 ? 0 : (a.D - a.R + 7) / 8;
  int64_t gx = 0, gy = 0, values = 0;
  for (int i = 0; i < parts; ++i) {
    const RotaryPart& p = a.part[i];
    if (p.size[0] == 0 || p.size[1] == 0 || p.size[2] == 0) continue;
    const int rows = kThreads / (turned + copied);
    const int64_t x = copied == 0 ? (p.size[2] * turned + kThreads - 1) / kThreads
                                  : (p.size[2] + rows - 1) / rows;
    const int64_t y = p.size[0] * ((p.size[1] + kHeads - 1) / kHeads);
    gx = x > gx ? x : gx;
    gy = y > gy ? y : gy;
    values += p.size[0] * p.size[1] * p.size[2] * a.D;
  }
  if (gx == 0) return hipSuccess;
  if (gy > 65535) gy = 65535;   // the kernel strides over the rest
  const dim3 grid((unsigned)gx, (unsigned)gy, (unsigned)parts);
  // More than the last-level cache holds of in and out: 304 MB take 55 us past the caches,
  // 61 through them (5.5 and 5.0 TB/s); what a smaller call writes is there for the next kernel.
  const bool stream = values * (f32 ? 8 : 4) > kStreamBytes;
  if (f32) {
    if (stream) launch_mode<float, true>(a, mode, grid, s);
    else launch_mode<float, false>(a, mode, grid, s);
  } else {
    if (stream) launch_mode<__bf16, true>(a, mode, grid, s);
    else launch_mode<__bf16, false>(a, mode, grid, s);
  }
  return hipGetLastError();
}

}  // namespace cb
