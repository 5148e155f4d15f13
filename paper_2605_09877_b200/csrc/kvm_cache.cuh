// Shared by the kernels over the 8-bit cache (kvm_cache.cu, kvm_cache_decode.cu, kvm_cache_prompt.cu, kvm_cache_shared.cu, kvm_front.cu): what a launch is given, which keys a
// position sees, and the e4m3 conversions.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kvm.h"

namespace kvm {
namespace cache {

constexpr int kMaxBatch = 1024;   // sequences of one call
constexpr int kTile = 128;        // keys of one tile of the attention kernels
constexpr int kLeastExp = -64;    // least exponent of a scale

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
// (skip: blocks in front that somebody else looks at)
__device__ __forceinline__ PageList pages_of(const Params& p, int first, int last, int window, int sinks, int skip = 0) {
  PageList t;
  const int end = (last >> p.page_shift) + 1;
  const int low = first - window + 1;   // (first >= 0 and window >= 1: no overflow)
  const int w0 = max(skip, low > 0 ? low >> p.page_shift : 0);
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

// n / d for 0 <= n < 2^31: with 2^(l-1) < d <= 2^l, m = floor(2^(31+l) / d) + 1, m d exceeds 2^(31+l) by at most 2^l, so n m >> (31 + l) is exact.
struct FastDiv {
  uint32_t m, s, d;
  explicit FastDiv(uint32_t x = 1) : d(x) {
    int l = 0;
    while ((1ull << l) < x) ++l;
    s = 31 + l;
    m = (uint32_t)((1ull << s) / x + 1);
  }
  __device__ __forceinline__ int div(int n) const { return (int)(((uint64_t)(uint32_t)n * m) >> s); }
};
// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t pack2(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// two floats -> two fp16 (a in the low half), round to nearest even, saturating (logits beyond 2^24 are rounded to more than 1)
__device__ __forceinline__ uint32_t to_f16x2(float a, float b) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// Groups of sequences that share their first blocks (kvm_cache_attend_shared): sequences offsets[g] .. offsets[g + 1] - 1 share shared[g] blocks.
struct Groups {
  const int32_t *offsets, *shared;
  int n;
};
// The group of sequence b: the last whose offset is not behind it (by a whole warp).
__device__ __forceinline__ int group_of(const Groups& g, int b) {
  int before = 0;
  for (int i0 = 0; i0 < g.n; i0 += 32) {
    const int i = i0 + (int)(threadIdx.x & 31);
    before += __popc(__ballot_sync(0xffffffffu, i < g.n && g.offsets[i] <= b));
  }
  return max(0, before - 1);
}
// The offsets, n + 1, to shared memory, by all NT threads of a block; whether they ascend from 0 to the batch (else nothing may be made of them).
template <int NT>
__device__ __forceinline__ bool load_groups(const Groups& g, int batch, int* offsets) {
  bool ok = true;
#pragma unroll 1
  for (int i = threadIdx.x; i <= g.n; i += NT) {
    const int x = g.offsets[i], before = i ? g.offsets[i - 1] : 0;
    offsets[i] = x;
    ok = ok && (i ? x >= before : x == 0) && (i < g.n || x == batch);
  }
  return __syncthreads_and(ok);
}
// Lengths of a sequence behind `skip` shared blocks: they have to lie in front of the call's tokens.
__device__ __forceinline__ bool shared_lengths(const Params& p, int b, int skip, int& start, int& n) {
  return seq_lengths(p, b, start, n) && skip >= 0 && skip <= p.max_pages && start >= skip << p.page_shift;
}

struct AttendArgs {
  Params p;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  int64_t sq[3], so[3];
  int Hq, G, d, window, sinks;   // window: INT32_MAX = all
  float scale_log2;              // scale * log2(e)
  float* part;                   // workspace
  // The kernels' SIDE builds: over the blocks behind the shared ones; results are left as partial ones for shared_merge_kernel.
  Groups groups;
  float* side;                   // few tokens: [unit][column][D + 2] of the units that one worker did
  int2* found;                   // few tokens: per unit its first and last worker (last -1: it is in `side`)
};
// maps of the codes of the keys and of the values (kvm_cache.cu)
bool encode_tmaps(CUtensorMap (&maps)[2], const Params& p, int d);
// tokens times heads of a group <= kDecodeCols; tiles: most key tiles of a sequence
constexpr int kDecodeCols = 16;
kvm_status_t launch_decode8(const AttendArgs& a, int64_t tiles, bool q_vec, cudaStream_t s);
int64_t decode_workspace(int64_t units, int64_t tiles, int d, int cols);
// ... SIDE: how many workers there are
kvm_status_t launch_decode8_side(const AttendArgs& a, int64_t tiles, bool q_vec, const CUtensorMap (&maps)[2], cudaStream_t s, int& workers);
// more than that; rows: tokens times heads of a group
kvm_status_t launch_prompt8(const AttendArgs& a, int64_t tiles, bool q_vec, bool out_vec, cudaStream_t s);
int64_t prompt_workspace(int64_t units, int64_t rows, int64_t tiles, int d);
// ... SIDE: row tiles of a unit and key splits, [((row tiles - 1 - row tile) * units + unit) * splits + split][D + 2][128] in a.part
struct PromptSide { int qtiles, nsplit; };
kvm_status_t launch_prompt8_side(const AttendArgs& a, int64_t tiles, bool q_vec, const CUtensorMap (&maps)[2], cudaStream_t s, PromptSide& side);
int64_t prompt_side_workspace(int64_t units, int64_t rows, int64_t tiles, int d);
constexpr int kSplitTiles = 4;    // least key tiles of a split
__host__ __device__ __forceinline__ int split_tiles(int tiles, int nsplit) {   // key tiles of a split, of a row tile that sees so many
  const int per = (tiles + nsplit - 1) / nsplit;
  return per < kSplitTiles ? kSplitTiles : per;
}

// Codes and scales that a call writes: keys, values.
struct AppendOut {
  uint8_t* codes[2];
  float* scales[2];
};

// Checks of arguments (kvm_cache.cu).  check_*: pointers too, or sizes only.
bool aligned(const void* p, uintptr_t n);
kvm_status_t check_cache(const kvm_cache_t* c, bool pointers);
kvm_status_t check_call(const kvm_cache_t* c, const kvm_cache_call_t* call, bool pointers);
Params params_of(const kvm_cache_t* c, const kvm_cache_call_t* call, int32_t* status);
// Strides of [batch, heads, tokens, d] (NULL: contiguous); false: negative ones, or rows that are written and lie on one another.
bool strides_of(const int64_t* st, int64_t B, int64_t H, int64_t T, int d, bool written, int64_t (&out)[3]);
bool rows_aligned(const void* p, const int64_t (&st)[3]);

}  // namespace cache
}  // namespace kvm
