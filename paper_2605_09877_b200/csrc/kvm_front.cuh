// Front end of an exact layer, shared by kvm_qk_norm_rope and kvm_cache_ingest (kvm_front.cu): norm of a head's row and rotary positions.
//
// A row of D channels is held by D / 8 consecutive lanes, eight channels each, as four pairs (x[j], y[j]).  Which channels these are is up to the
// rotary layout (MODE), so that both of a rotated pair are always in one lane and nothing has to be exchanged.  Pair i = 4 * lane + j, h = r / 2:
//     kSide    pairs (2i, 2i + 1): eight channels side by side, rotated for i < h
//     kHalves  pairs (i, i + h), h a multiple of 4: lanes with i < h have two runs of four, channels i .. and i + h .., the lanes behind them (not rotated)
//              eight side by side, the first four as x
//     kSingle  any h, any alignment, channel by channel: as kSide, or (i, i + h) and behind them whatever is left
// In the first two a lane loads and stores 8 bytes at a time.
//
// Angles: position * f_i in quarter turns in fp64 (off by 2^-52 of the angle: 2^-32 of a quarter turn at position 2^20), the nearest whole number taken
// off and counted as a quadrant, so that the fp32 argument of sin and cos is at most 1/8 turn and rounded to 2^-26 of a quarter turn.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kvm.h"

namespace kvm {
namespace front {

struct FrontDev {
  double quarter[64];   // quarter turns per position of each pair
  float mag, eps;
  int norm, half, h;    // half: pairs (i, i + h)
};

struct Rows {           // rows of q, k or v: element strides of (batch, head, token)
  const __nv_bfloat16* x;
  __nv_bfloat16* y;
  const float *w, *b;   // [heads, D] or NULL
  int64_t sx[3], sy[3];
  int H;
};

enum { kSide, kHalves, kSingle };

// Which channels a lane has.
template <int D, int MODE>
struct Lane {
  int i0, h;            // first pair; rotated pairs
  int c0, c1;           // runs of four (kSide, kHalves)
  bool half;            // kSingle: the half layout
  __device__ __forceinline__ Lane(const FrontDev& f, int lane) : i0(4 * lane), h(f.h), half(f.half) {
    const bool apart = MODE == kHalves && i0 < h;
    c0 = apart ? i0 : 8 * lane;   // (4 lanes' worth of pairs behind h begin at channel 2 h + 2 (i0 - h) = 8 lane)
    c1 = apart ? i0 + h : c0 + 4;
  }
  __device__ __forceinline__ bool rotated(int j) const { return MODE == kHalves ? i0 < h : i0 + j < h; }   // (kHalves: all four or none)
  // (kSingle; lanes behind the rotated ones as in kHalves, so that sums have the same order)
  __device__ __forceinline__ int ch_x(int j) const { return !half ? 2 * (i0 + j) : i0 + j < h ? i0 + j : i0 >= h ? 2 * i0 + j : 2 * (i0 + j); }
  __device__ __forceinline__ int ch_y(int j) const { return !half ? 2 * (i0 + j) + 1 : i0 + j < h ? i0 + j + h : i0 >= h ? 2 * i0 + 4 + j : 2 * (i0 + j) + 1; }
};

// A lane's share of a row as raw bf16, in the order of memory (runs) or x0 y0 x1 y1 .. (kSingle).
struct Raw { uint2 a, b; };

template <int D, int MODE>
__device__ __forceinline__ Raw load_raw(const __nv_bfloat16* row, const Lane<D, MODE>& L) {
  Raw r;
  if (MODE != kSingle) {
    r.a = __ldcs(reinterpret_cast<const uint2*>(row + L.c0));
    r.b = __ldcs(reinterpret_cast<const uint2*>(row + L.c1));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = (uint32_t)__bfloat16_as_ushort(row[L.ch_x(j)]) | ((uint32_t)__bfloat16_as_ushort(row[L.ch_y(j)]) << 16);
    r.a = make_uint2(w[0], w[1]);
    r.b = make_uint2(w[2], w[3]);
  }
  return r;
}
__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Eight values in the order of load_raw as pairs, and back.
template <int MODE>
__device__ __forceinline__ void to_pairs(const float (&v)[8], float (&x)[4], float (&y)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = MODE == kHalves ? v[j] : v[2 * j];
    y[j] = MODE == kHalves ? v[4 + j] : v[2 * j + 1];
  }
}
template <int MODE>
__device__ __forceinline__ void from_pairs(const float (&x)[4], const float (&y)[4], float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[MODE == kHalves ? j : 2 * j] = x[j];
    v[MODE == kHalves ? 4 + j : 2 * j + 1] = y[j];
  }
}
__device__ __forceinline__ void values_of(const Raw& r, float (&v)[8]) {
  v[0] = lo16(r.a.x); v[1] = hi16(r.a.x); v[2] = lo16(r.a.y); v[3] = hi16(r.a.y);
  v[4] = lo16(r.b.x); v[5] = hi16(r.b.x); v[6] = lo16(r.b.y); v[7] = hi16(r.b.y);
}
template <int D, int MODE>
__device__ __forceinline__ void store_row(__nv_bfloat16* row, const Lane<D, MODE>& L, const float (&x)[4], const float (&y)[4]) {
  if (MODE != kSingle) {
    float v[8];
    from_pairs<MODE>(x, y, v);
    __nv_bfloat162 h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<uint2*>(row + L.c0) = *reinterpret_cast<const uint2*>(&h[0]);
    *reinterpret_cast<uint2*>(row + L.c1) = *reinterpret_cast<const uint2*>(&h[2]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      row[L.ch_x(j)] = __float2bfloat16_rn(x[j]);
      row[L.ch_y(j)] = __float2bfloat16_rn(y[j]);
    }
  }
}

// Weights (or biases) of the lane's pairs; `none` where there are none.
template <int D, int MODE>
__device__ __forceinline__ void load_affine(const float* w, int head, const Lane<D, MODE>& L, float none, float (&x)[4], float (&y)[4]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = y[j] = none;
    return;
  }
  w += (int64_t)head * D;
  if (MODE != kSingle) {
    const float4 a = *reinterpret_cast<const float4*>(w + L.c0), b = *reinterpret_cast<const float4*>(w + L.c1);
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    to_pairs<MODE>(v, x, y);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[j] = w[L.ch_x(j)]; y[j] = w[L.ch_y(j)]; }
  }
}

// magnitude * (cos, sin) of the lane's pairs at a position; pairs that are not rotated: anything (rotate leaves them)
template <int D, int MODE>
__device__ __forceinline__ void angles(const FrontDev& f, const Lane<D, MODE>& L, int64_t pos, float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c[j] = 1.f;
    s[j] = 0.f;
    if (!L.rotated(j)) continue;
    const double t = (double)pos * f.quarter[L.i0 + j], n = rint(t);
    const int q = (int)((long long)n & 3);
    float sn, cs;
    sincospif((float)(t - n) * 0.5f, &sn, &cs);
    const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;   // cos(u + q pi/2), sin(u + q pi/2)
    c[j] = f.mag * (q == 1 || q == 2 ? -a : a);
    s[j] = f.mag * (q >= 2 ? -b : b);
  }
}
template <int D, int MODE>
__device__ __forceinline__ void rotate(const Lane<D, MODE>& L, const float (&c)[4], const float (&s)[4], float (&x)[4], float (&y)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = x[j], b = y[j];
    if (L.rotated(j)) {   // (a channel that is not rotated is not touched by an infinity beside it)
      x[j] = fmaf(a, c[j], -b * s[j]);
      y[j] = fmaf(b, c[j], a * s[j]);
    }
  }
}

// Norm over the D channels of the rows of a warp (every lane calls): statistics and sums in fp32, the mean taken off before the squares.
template <int D>
__device__ __forceinline__ void norm(const FrontDev& f, const float (&wx)[4], const float (&wy)[4], const float (&bx)[4], const float (&by)[4], float (&x)[4], float (&y)[4]) {
  constexpr int LPR = D / 8;
  if (f.norm == KVM_NORM_NONE) return;
  float mean = 0.f;
  if (f.norm == KVM_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) s += x[j] + y[j];
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    mean = s * (1.f / D);
  }
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] -= mean;
    y[j] -= mean;
    q = fmaf(x[j], x[j], fmaf(y[j], y[j], q));
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
  const float rstd = rsqrtf(fmaf(q, 1.f / D, f.eps));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = fmaf(x[j] * rstd, wx[j], bx[j]);
    y[j] = fmaf(y[j] * rstd, wy[j], by[j]);
  }
}

}  // namespace front
}  // namespace kvm
