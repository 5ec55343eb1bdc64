// Rotary positions (gfx950): rows of up to two tensors, each pair of values
// turned by freq[i] * (pos - from).
#include <math.h>

#include "cache.h"

namespace cb {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kHeads = 4;   // rows of one position that a thread turns by the same angles

// Eight values of a row as fp32.
template <typename T>
struct Vec8;
template <>
struct Vec8<float> {
  f32x4 a, b;
  __device__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4*>(p);
    b = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ void store(float* p) const {
    *reinterpret_cast<f32x4*>(p) = a;
    *reinterpret_cast<f32x4*>(p + 4) = b;
  }
  __device__ float get(int i) const { return i < 4 ? a[i & 3] : b[i & 3]; }
  __device__ void set(int i, float x) {
    if (i < 4) a[i & 3] = x; else b[i & 3] = x;
  }
};
template <>
struct Vec8<__bf16> {
  u32x4 a;
  __device__ void load(const __bf16* p) { a = *reinterpret_cast<const u32x4*>(p); }
  __device__ void store(__bf16* p) const { *reinterpret_cast<u32x4*>(p) = a; }
  __device__ float get(int i) const {
    const uint32_t w = a[i >> 1];
    return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  __device__ void set(int i, float x) {
    const __bf16 r = (__bf16)x;   // the value's one rounding
    const uint32_t h = __builtin_bit_cast(uint16_t, r);
    a[i >> 1] = (i & 1) ? ((a[i >> 1] & 0xffffu) | (h << 16)) : ((a[i >> 1] & 0xffff0000u) | h);
  }
};

__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const __bf16* p) { return (float)*p; }

// Turns reduced in 64 bits (a position of 2^31 times a frequency keeps 22
// bits of the turn), then sine and cosine of the remainder in fp32.
__device__ inline void angle(double delta, double freq, float amplitude, float sign, float* cs,
                             float* sn) {
  const double t = delta * freq;
  const float r = (float)(t - rint(t));
  float s, c;
  sincospif(2.f * r, &s, &c);
  *cs = c * amplitude;
  *sn = s * (amplitude * sign);
}

// Kind of a work item's chunk of a row: 0, half layout in 16-byte vectors: eight pairs
// from both halves, then copied vectors of eight; 1, interleaved: eight consecutive
// values; 2, half layout with halves that are no multiple of eight: one pair,
// then single copied values.
template <typename T, int MODE>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  const RotaryPart& p = a.part[blockIdx.z];
  const int half = a.R / 2;
  const int turned = MODE == 0 ? half / 8 : MODE == 1 ? a.D / 8 : half;
  const int copied = MODE == 0 ? (a.D - a.R) / 8 : MODE == 1 ? 0 : a.D - a.R;
  const int chunks = turned + copied;
  const int64_t items = p.size[2] * chunks;
  const int64_t head_blocks = (p.size[1] + kHeads - 1) / kHeads;
  const int64_t outer = p.size[0] * head_blocks;
  const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (item >= items) return;
  const int64_t t = items <= 0x7fffffff ? (int64_t)((uint32_t)item / (uint32_t)chunks)
                                        : item / chunks;
  const int ch = (int)(item - t * chunks);
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
        const int at = MODE == 0 ? a.R + (ch - turned) * 8 : a.R + (ch - turned);
        if constexpr (MODE == 0) {
          Vec8<T> x;
          x.load(in + h * p.in_stride[1] + at);
          x.store(out + h * p.out_stride[1] + at);
        } else {
          out[h * p.out_stride[1] + at] = in[h * p.in_stride[1] + at];
        }
      }
      continue;
    }
    constexpr int PAIRS = MODE == 0 ? 8 : MODE == 1 ? 4 : 1;
    // all rows first, then the angles, so that the loads are under way meanwhile
    Vec8<T> lo[MODE == 2 ? 1 : kHeads], hi[MODE == 0 ? kHeads : 1];
    float l1[MODE == 2 ? kHeads : 1], h1[MODE == 2 ? kHeads : 1];
    double delta[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < nh) {
        const T* r = in + h * p.in_stride[1];
        if constexpr (MODE == 0) {
          lo[h].load(r + ch * 8);
          hi[h].load(r + half + ch * 8);
        } else if constexpr (MODE == 1) {
          lo[h].load(r + ch * 8);
        } else {
          l1[h] = load1(r + ch);
          h1[h] = load1(r + half + ch);
        }
        const int64_t q = pos[h * p.pos_stride[1]];
        delta[h] = (double)(q - (from ? (int64_t)from[h * p.from_stride[1]] : 0));
      }
    const bool shared = p.pos_stride[1] == 0 && (!from || p.from_stride[1] == 0);
    float cs[PAIRS], sn[PAIRS];
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < nh) {
        if (h == 0 || !shared) {
#pragma unroll
          for (int i = 0; i < PAIRS; ++i) {
            const int pair = ch * PAIRS + i;
            cs[i] = 1.f;
            sn[i] = 0.f;
            if (pair < half) angle(delta[h], a.freq[pair], a.amplitude, a.sign, &cs[i], &sn[i]);
          }
        }
        T* w = out + h * p.out_stride[1];
        if constexpr (MODE == 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float x = lo[h].get(i), y2 = hi[h].get(i);
            lo[h].set(i, x * cs[i] - y2 * sn[i]);
            hi[h].set(i, y2 * cs[i] + x * sn[i]);
          }
          lo[h].store(w + ch * 8);
          hi[h].store(w + half + ch * 8);
        } else if constexpr (MODE == 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (ch * 4 + i < half) {   // pairs behind the rotated ones stay as they are
              const float x = lo[h].get(2 * i), y2 = lo[h].get(2 * i + 1);
              lo[h].set(2 * i, x * cs[i] - y2 * sn[i]);
              lo[h].set(2 * i + 1, y2 * cs[i] + x * sn[i]);
            }
          }
          lo[h].store(w + ch * 8);
        } else {
          w[ch] = (T)(l1[h] * cs[0] - h1[h] * sn[0]);
          w[half + ch] = (T)(h1[h] * cs[0] + l1[h] * sn[0]);
        }
      }
  }
}

template <typename T>
void launch_mode(const RotaryArgs& a, int mode, dim3 grid, hipStream_t s) {
  if (mode == 0) rotary_kernel<T, 0><<<grid, kThreads, 0, s>>>(a);
  else if (mode == 1) rotary_kernel<T, 1><<<grid, kThreads, 0, s>>>(a);
  else rotary_kernel<T, 2><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int parts, bool interleaved, bool f32,
                         hipStream_t s) {
  const int half = a.R / 2;
  const int mode = interleaved ? 1 : half % 8 == 0 ? 0 : 2;
  const int chunks = mode == 0 ? half / 8 + (a.D - a.R) / 8 : mode == 1 ? a.D / 8
                                                                       : half + a.D - a.R;
  int64_t gx = 0, gy = 0;
  for (int i = 0; i < parts; ++i) {
    const RotaryPart& p = a.part[i];
    if (p.size[0] == 0 || p.size[1] == 0 || p.size[2] == 0) continue;
    const int64_t x = (p.size[2] * chunks + kThreads - 1) / kThreads;
    const int64_t y = p.size[0] * ((p.size[1] + kHeads - 1) / kHeads);
    gx = x > gx ? x : gx;
    gy = y > gy ? y : gy;
  }
  if (gx == 0) return hipSuccess;
  if (gy > 65535) gy = 65535;   // the kernel strides over the rest
  const dim3 grid((unsigned)gx, (unsigned)gy, (unsigned)parts);
  if (f32) launch_mode<float>(a, mode, grid, s);
  else launch_mode<__bf16>(a, mode, grid, s);
  return hipGetLastError();
}

}  // namespace cb
