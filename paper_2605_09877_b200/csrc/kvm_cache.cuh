// Shared by the kernels over the 8-bit cache (kvm_cache.cu, kvm_cache_decode.cu, kvm_cache_prompt.cu): what a launch is given, which keys a
// position sees, and the e4m3 conversions.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kvm.h"

namespace kvm {
namespace cache {

constexpr int kMaxBatch = 1024;   // sequences of one call
constexpr int kTile = 128;        // keys of one tile of the attention kernels

struct Params {
  const uint8_t *k, *v;
  const float *ks, *vs;
  const int32_t *pages, *start, *count;
  int32_t* status;
  int64_t n_pages, T;
  int Hkv, page, page_shift, batch, max_pages;
};

// Tokens before the call (start) and in it (n) of sequence b; false: lengths that the call does not allow.
__device__ __forceinline__ bool seq_lengths(const Params& p, int b, int& start, int& n) {
  start = p.start[b];
  n = p.count ? p.count[b] : (int)p.T;
  return start >= 0 && n >= 0 && n <= p.T && (int64_t)start + n <= (int64_t)p.max_pages * p.page;
}
__device__ __forceinline__ void report(int32_t* status, int code) {
  if (status) atomicExch(status, code);
}
// Position i sees j <= i with j > i - window, or j < sinks.  (window: INT32_MAX stands for all)
__device__ __forceinline__ bool sees(int i, int j, int window, int sinks) {
  return j <= i && (j > i - window || j < sinks);
}
// The pages that positions [first, last] see: those of the first `sinks` tokens, then the window's, without those counted twice; a key tile is
// the next kTile / page of them, whatever their numbers are (so a window with sinks costs no more tiles than its pages fill).
struct PageList {
  int n_sink, first, n, tiles;   // page i of the list is page page_at(i) of the sequence; n pages, so many tiles
};
__device__ __forceinline__ PageList pages_of(const Params& p, int first, int last, int window, int sinks) {
  PageList t;
  const int end = (last >> p.page_shift) + 1;
  const int low = first - window + 1;   // (first >= 0 and window >= 1: no overflow)
  const int w0 = low > 0 ? low >> p.page_shift : 0;
  t.n_sink = min(w0, (sinks + p.page - 1) >> p.page_shift);
  t.first = w0;
  t.n = t.n_sink + end - w0;
  const int per = kTile >> p.page_shift;
  t.tiles = (t.n + per - 1) >> (7 - p.page_shift);
  return t;
}
__device__ __forceinline__ int page_at(const PageList& t, int i) { return i < t.n_sink ? i : t.first + (i - t.n_sink); }
constexpr int kNowhere = 0x7fff0000;   // position of the keys of a page that a tile lacks: behind all others
// Whether all of positions [first, last] see all keys of a page that begins at p0.
__device__ __forceinline__ bool page_seen_by_all(const Params& p, int p0, int first, int last, int window, int sinks) {
  const int end = p0 + p.page - 1;
  return end <= first && (p0 > last - window || end < sinks);
}

// Exponent of a scale 2^e.  A NaN scale has exponent 128: exp2i(128) is NaN.
__device__ __forceinline__ int scale_exp(float s) { return (int)((__float_as_uint(s) >> 23) & 255u) - 127; }
__device__ __forceinline__ float exp2i(int e) {   // 2^e, -126 <= e <= 127; 128: NaN
  return e > 127 ? __int_as_float(0x7fc00000) : __int_as_float((e + 127) << 23);
}

// Scales of values are taken into the exponents of the weights, relative to the largest of those that are looked at together, and out of the row
// sums again: 2^90 and its inverse leave the sums within fp32.  Blocks further below contribute to the row sum only (their values are
// less than 2^-90 of the others').  Results before the division are held in units of 2^40, so that values up to bf16's largest do not overflow.
constexpr int kFoldMost = 90, kUnitExp = 40;

// two floats -> two e4m3 codes (a in the low byte), round to nearest even, saturating
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// two e4m3 codes -> two fp16 (exact)
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t c) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)c));
  return r;
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t c) {
  const uint32_t h = e4m3x2_to_f16x2(c);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Two values below 2^8 as sums of two e4m3 numbers each, hi + lo (a in the low bytes).  By way of fp16, which holds 8-bit significands exactly
// down to 2^-14 and their part above 2^-24 below: far less than the 2^-10 that e4m3 leaves.
__device__ __forceinline__ void split_e4m3x2(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __half2 y = __floats2half2_rn(a, b);
  uint16_t h, l;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(h) : "r"(*reinterpret_cast<const uint32_t*>(&y)));
  const uint32_t back = e4m3x2_to_f16x2(h);
  const __half2 d = __hsub2(y, *reinterpret_cast<const __half2*>(&back));   // (exact: a difference of neighbours)
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(l) : "r"(*reinterpret_cast<const uint32_t*>(&d)));
  hi = h;
  lo = l;
}

struct AttendArgs {
  Params p;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  int64_t sq[3], so[3];
  int Hq, G, d, window, sinks;   // window: INT32_MAX = all
  float scale_log2;              // scale * log2(e)
  float* part;                   // workspace
};
// tokens times heads of a group <= kDecodeCols; tiles: most key tiles of a sequence
constexpr int kDecodeCols = 16;
kvm_status_t launch_decode8(const AttendArgs& a, int64_t tiles, bool q_vec, cudaStream_t s);
int64_t decode_workspace(int64_t units, int64_t tiles, int d, int cols);
// more than that; rows: tokens times heads of a group
kvm_status_t launch_prompt8(const AttendArgs& a, int64_t tiles, bool q_vec, bool out_vec, cudaStream_t s);
int64_t prompt_workspace(int64_t units, int64_t rows, int64_t tiles, int d);

}  // namespace cache
}  // namespace kvm
