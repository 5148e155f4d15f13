// Front end of an exact layer, shared by kvm_qk_norm_rope and kvm_cache_ingest (kvm_front.cu): norm of a head's row and rotary positions.
//
// A row of D channels is held by D / 8 consecutive lanes, eight channels each, as four pairs (x[j], y[j]).  Which channels are up to the
// rotary layout, so that both of a rotated pair are always in one lane and nothing has to be exchanged.  Pair i = 4 * lane + j:
//     pairs (i, i + h), h = r / 2:   i < h: channels (i, i + h); behind them (2i, 2i + 1), not rotated
//     pairs (2i, 2i + 1):            channels (2i, 2i + 1), rotated for i < h
// Where h is a multiple of 4 a lane's channels are two runs of four, loaded and stored 8 bytes at a time; else (and for rows that are not
// aligned) one by one.
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

struct Rows {           // rows of q or k: element strides of (batch, head, token)
  const __nv_bfloat16* x;
  __nv_bfloat16* y;
  const float *w, *b;   // [heads, D] or NULL
  int64_t sx[3], sy[3];
  int H;
  int vx, vy, vw;       // whether x, y, (w and b) may be accessed as runs of four
};

// Which channels a lane has.
template <int D>
struct Lane {
  int c0, c1;           // runs of four, in the order of memory: pairs (i, i + h): x = c0 .. + 3, y = c1 .. + 3; else pairs side by side from c0 on
  int i0, h;            // first pair; rotated pairs
  bool half, side;      // side: the lane's pairs lie side by side
  __device__ __forceinline__ Lane(bool half_, int h_, int lane) : i0(4 * lane), h(h_), half(half_) {
    side = !half || i0 >= h;
    c0 = half && i0 < h ? i0 : 8 * lane;   // (4 lanes' worth of pairs behind h begin at channel 2 h + 2 (i0 - h) = 8 lane)
    c1 = half && i0 < h ? i0 + h : c0 + 4;
  }
  __device__ __forceinline__ int ch_x(int j) const { return half && i0 + j < h ? i0 + j : 2 * (i0 + j); }
  __device__ __forceinline__ int ch_y(int j) const { return half && i0 + j < h ? i0 + j + h : 2 * (i0 + j) + 1; }
};

// A lane's share of a row as raw bf16, in the order of memory (runs) or x0 y0 x1 y1 .. (one by one).
struct Raw { uint2 a, b; };

template <int D>
__device__ __forceinline__ Raw load_raw(const __nv_bfloat16* row, const Lane<D>& L, bool vec) {
  Raw r;
  if (vec) {
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
// ... as pairs
__device__ __forceinline__ void to_pairs(const Raw& r, bool side, float (&x)[4], float (&y)[4]) {
  const float v[8] = {lo16(r.a.x), hi16(r.a.x), lo16(r.a.y), hi16(r.a.y), lo16(r.b.x), hi16(r.b.x), lo16(r.b.y), hi16(r.b.y)};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = side ? v[2 * j] : v[j];
    y[j] = side ? v[2 * j + 1] : v[4 + j];
  }
}
// ... and back, in the order that load_raw has
__device__ __forceinline__ void from_pairs(const float (&x)[4], const float (&y)[4], bool side, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = side ? (j & 1 ? y[j / 2] : x[j / 2]) : x[j];
    v[4 + j] = side ? (j & 1 ? y[2 + j / 2] : x[2 + j / 2]) : y[j];
  }
}
template <int D>
__device__ __forceinline__ void store_row(__nv_bfloat16* row, const Lane<D>& L, bool vec, bool side, const float (&x)[4], const float (&y)[4]) {
  float v[8];
  from_pairs(x, y, side, v);
  __nv_bfloat162 h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
  if (vec) {
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
template <int D>
__device__ __forceinline__ void load_affine(const float* w, int head, const Lane<D>& L, bool vec, bool side, float none, float (&x)[4], float (&y)[4]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = y[j] = none;
    return;
  }
  w += (int64_t)head * D;
  if (vec) {
    const float4 a = *reinterpret_cast<const float4*>(w + L.c0), b = *reinterpret_cast<const float4*>(w + L.c1);
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = side ? v[2 * j] : v[j];
      y[j] = side ? v[2 * j + 1] : v[4 + j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[j] = w[L.ch_x(j)]; y[j] = w[L.ch_y(j)]; }
  }
}

// magnitude * (cos, sin) of the lane's pairs at a position; pairs that are not rotated: anything (rotate leaves them)
template <int D>
__device__ __forceinline__ void angles(const FrontDev& f, const Lane<D>& L, int64_t pos, float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c[j] = 1.f;
    s[j] = 0.f;
    if (L.i0 + j >= L.h) continue;
    const double t = (double)pos * f.quarter[L.i0 + j], n = rint(t);
    const int q = (int)((long long)n & 3);
    float sn, cs;
    sincospif((float)(t - n) * 0.5f, &sn, &cs);
    const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;   // cos(u + q pi/2), sin(u + q pi/2)
    c[j] = f.mag * (q == 1 || q == 2 ? -a : a);
    s[j] = f.mag * (q >= 2 ? -b : b);
  }
}
template <int D>
__device__ __forceinline__ void rotate(const Lane<D>& L, const float (&c)[4], const float (&s)[4], float (&x)[4], float (&y)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = x[j], b = y[j];
    if (L.i0 + j < L.h) {   // (a channel that is not rotated is not touched by an infinity beside it)
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
