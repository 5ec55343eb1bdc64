// Shared between the C ABI of the paged four-bit cache (cache_api.hip) and its
// kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cb {

constexpr int kCacheMaxEntries = 2048;     // entries of a page call: their lists lie in LDS
constexpr int kCacheMaxSeqs = 1 << 17;     // its bit set of sequences fills 16 KiB of LDS
constexpr int kCacheMaxPages = 1 << 24;
constexpr int64_t kMaxThreads = 0xffffffff;   // of a grid, along one axis

// The cache as kernels see it.
struct CacheView {
  unsigned char* pool;
  int32_t* refs;
  int32_t* table;
  int32_t* lens;
  int64_t page_bytes;
  int32_t unit_bytes;   // P * (D + D/16)
  int32_t layers, heads, D;
  int32_t page_shift;   // P = 1 << page_shift
  int32_t pages, seqs, width;
};

// Byte offsets within a unit of P positions of D values: key codes at 0, then
// value codes, key scales, value scales.
__host__ __device__ inline int unit_value_codes(int P, int D) { return P * D / 2; }
__host__ __device__ inline int unit_key_scales(int P, int D) { return P * D; }
__host__ __device__ inline int unit_value_scales(int P, int D) { return P * D + P * D / 32; }

struct RotaryPart {
  const void* in;
  void* out;
  const int32_t* pos;
  const int32_t* from;
  int64_t size[3], in_stride[3], out_stride[3], pos_stride[3], from_stride[3];
};

struct RotaryArgs {
  RotaryPart part[2];
  const double* freq;
  float amplitude, sign;
  int32_t D, R;
};

hipError_t launch_rotary(const RotaryArgs& a, int parts, bool interleaved, bool f32,
                         hipStream_t s);

struct CacheRowsArgs {
  CacheView c;
  const void* k;   // outputs of a read
  const void* v;
  const int32_t* seqs;
  const int32_t* start;
  const int32_t* counts;
  int64_t stride[4];
  int64_t max_count;
  int32_t layer0, layers, n;
};

hipError_t launch_cache_write(const CacheRowsArgs& a, bool f32, hipStream_t s);
hipError_t launch_cache_read(const CacheRowsArgs& a, bool f32, hipStream_t s);

hipError_t launch_cache_extend(const CacheView& c, const int32_t* seqs, const int32_t* add, int n,
                               int32_t* status, hipStream_t s);
hipError_t launch_cache_free(const CacheView& c, const int32_t* seqs, int n, hipStream_t s);

size_t cache_fork_ws(int64_t n, int64_t width);
hipError_t launch_cache_fork(const CacheView& c, const int32_t* parents, const int32_t* children,
                             int n, bool copy, int32_t* status, void* ws, hipStream_t s);

struct CacheCompactArgs {
  CacheView c;
  const int32_t* src;
  const int32_t* dst;
  const int32_t* idx;
  const int32_t* counts;
  int64_t idx_stride[3];
  int64_t keep;
  int32_t n;
  int32_t* status;
  int32_t* old_rows;   // [n][1 + width]: length and pages of the sources
};

size_t cache_compact_ws(int64_t n, int64_t width);
hipError_t launch_cache_compact(const CacheCompactArgs& a, hipStream_t s);

struct AttendArgs {
  CacheView c;
  const void* q;
  void* out;
  float* lse;
  const int32_t* seqs;
  const int32_t* q_lens;
  float* part_o;    // [layers][heads][slots][rows_pad][D], slot = run + sequence
  float2* part_ml;  // [layers][heads][slots][rows_pad]: reference, sum
  int64_t q_stride[4], out_stride[4];
  int64_t q_len;    // m
  int32_t layer0, layers, n, q_heads, group;
  uint32_t recip;   // floor(2^32 / group), or the most there is
  int32_t row_tiles, rows_pad;
  int32_t target;   // runs that the positions are dealt to
  int32_t whole;    // a run is a sequence
  int32_t slots;    // target + n
  int32_t room;     // no sequence is longer
  int32_t causal;
  float c2;         // scale * log2(e)
};

// Sizes of a call: row tiles, workspace.
struct AttendPlan {
  int32_t blocks;   // 16-row blocks a wave holds
  int32_t row_tiles, rows_pad, target, slots;
  int32_t room;     // positions of the longest
  bool whole;       // no sequence is cut
  bool alone;       // a workgroup is one wave
  size_t off_ml, total;
};

bool make_attend_plan(int layers, int n, int heads, int q_heads, int64_t q_len, int D, bool f32,
                      int64_t capacity, AttendPlan* p);
hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, bool f32, hipStream_t s);

}  // namespace cb
