// Front end of an exact layer, shared by kvm_qk_norm_rope and kvm_cache_ingest (kvm_front.cu): norm of a head's row and rotary positions.
//
// A row of D channels is held by D / 8 consecutive lanes, eight channels each, as four pairs (x[j], y[j]).  Which channels these are is up to the
// rotary layout (MODE), so that both of a rotated pair are always in one lane and nothing has to be exchanged.  Pair i = 4 * lane + j, h = r / 2:
//     kSide    pairs (2i, 2i + 1): eight channels side by side, rotated for i < h
//     kHalves  pairs (i, i + h), h a multiple of 4: lanes with i < h have two runs of four, channels i .. and i + h .., the lanes behind them (not rotated)
//              eight side by side, the first four as x
//     kMixed   pairs (i, i + h), any h: behind them whatever is left
//     kSingle  any pairs, rows that are not aligned
// Aligned rows come by way of shared memory, 16 bytes per lane (Stage): what a kernel has on its way costs no registers, several heads ahead, and a lane
// takes its channels from there.
//
// Angles: f_i, an fp64 number (off by 2^-52 of itself, which is less than 2^-54 of a turn per position), as a fraction of a turn cut to units of 2^-64.  The product with a
// position drops whole turns and no bits of the rest: it is off by less than 2^-53 of a turn times the position, 2^-22 at 2^31.  The quadrant is its top two bits (rounded), what is
// left, of which 30 bits are taken (2^-32 of a turn, and fp32's 2^-28), is within 1/8 turn, and sin and cos of that are their Taylor polynomials (the terms left out are
// below 2e-9).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kvm_cache.cuh"

namespace kvm {
namespace front {

struct FrontDev {
  uint64_t turns[64];   // 2^64 turns per position of each pair
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

enum { kSide, kHalves, kMixed, kSingle };

// Which channels a lane has.
template <int D, int MODE>
struct Lane {
  int i0, h;            // first pair; rotated pairs
  int c0, c1;           // runs of four (kSide, kHalves); kMixed: the first of eight channels that the lane stores
  bool half;            // kMixed, kSingle: the half layout
  __device__ __forceinline__ Lane(const FrontDev& f, int lane) : i0(4 * lane), h(f.h), half(f.half) {
    const bool apart = MODE == kHalves && i0 < h;
    c0 = apart ? i0 : 8 * lane;   // (4 lanes' worth of pairs behind h begin at channel 2 h + 2 (i0 - h) = 8 lane)
    c1 = apart ? i0 + h : c0 + 4;
  }
  __device__ __forceinline__ bool rotated(int j) const { return MODE == kHalves ? i0 < h : i0 + j < h; }   // (kHalves: all four or none)
  // (kMixed, kSingle; lanes behind the rotated ones as in kHalves, so that sums have the same order)
  __device__ __forceinline__ int ch_x(int j) const { return !half ? 2 * (i0 + j) : i0 + j < h ? i0 + j : i0 >= h ? 2 * i0 + j : 2 * (i0 + j); }
  __device__ __forceinline__ int ch_y(int j) const { return !half ? 2 * (i0 + j) + 1 : i0 + j < h ? i0 + j + h : i0 >= h ? 2 * i0 + 4 + j : 2 * (i0 + j) + 1; }
};

// A lane's share of a row as raw bf16, in the order of memory (runs) or x0 y0 x1 y1 .. (channel by channel).
struct Raw { uint2 a, b; };

// From a row of 2 D bytes, in global or shared memory.
template <int D, int MODE>
__device__ __forceinline__ Raw load_raw(const __nv_bfloat16* row, const Lane<D, MODE>& L) {
  Raw r;
  if (MODE == kSide) {
    const uint4 u = *reinterpret_cast<const uint4*>(row + L.c0);
    r.a = make_uint2(u.x, u.y);
    r.b = make_uint2(u.z, u.w);
  } else if (MODE == kHalves) {
    r.a = *reinterpret_cast<const uint2*>(row + L.c0);
    r.b = *reinterpret_cast<const uint2*>(row + L.c1);
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

// Rows on their way: a block of TH threads has S stages of CH rows per lane.  D / 8 lanes of a warp write a row, 16 bytes each, and read it; nobody else does.
template <int D, int TH, int CH, int S>
struct Stage {
  static constexpr int kBytes = S * CH * TH * 16;
  uint8_t* mem;
  __device__ __forceinline__ void copy(int stage, int i, const __nv_bfloat16* row) const {   // (row: its first channel)
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(mem + ((stage * CH + i) * TH + threadIdx.x) * 16);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + threadIdx.x % (D / 8) * 8) : "memory");
  }
  __device__ __forceinline__ __nv_bfloat16* row(int stage, int i) const {
    return reinterpret_cast<__nv_bfloat16*>(mem + ((stage * CH + i) * TH + threadIdx.x / (D / 8) * (D / 8)) * 16);
  }
  __device__ __forceinline__ void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // until all but the last S - 2 groups are there, for the whole warp
  __device__ __forceinline__ void wait() const {
    asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
    __syncwarp();
  }
};

// A lane's four pairs, two to a 64-bit register (x0 x1, x2 x3; y0 y1, y2 y3): fp32 arithmetic goes two at a time.
struct Pairs { uint64_t x[2], y[2]; };

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
using cache::add2;
using cache::fma2;
using cache::pack2;
using cache::unpack2;
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Eight values in the order of load_raw as pairs, and back.
template <int MODE>
__device__ __forceinline__ Pairs to_pairs(const float (&v)[8]) {
  Pairs p;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p.x[k] = MODE == kHalves ? pack2(v[2 * k], v[2 * k + 1]) : pack2(v[4 * k], v[4 * k + 2]);
    p.y[k] = MODE == kHalves ? pack2(v[4 + 2 * k], v[5 + 2 * k]) : pack2(v[4 * k + 1], v[4 * k + 3]);
  }
  return p;
}
template <int MODE>
__device__ __forceinline__ void from_pairs(const Pairs& p, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    unpack2(p.x[k], v[MODE == kHalves ? 2 * k : 4 * k], v[MODE == kHalves ? 2 * k + 1 : 4 * k + 2]);
    unpack2(p.y[k], v[MODE == kHalves ? 4 + 2 * k : 4 * k + 1], v[MODE == kHalves ? 5 + 2 * k : 4 * k + 3]);
  }
}
__device__ __forceinline__ void values_of(const Raw& r, float (&v)[8]) {
  v[0] = lo16(r.a.x); v[1] = hi16(r.a.x); v[2] = lo16(r.a.y); v[3] = hi16(r.a.y);
  v[4] = lo16(r.b.x); v[5] = hi16(r.b.x); v[6] = lo16(r.b.y); v[7] = hi16(r.b.y);
}
// scratch (kMixed): the row in shared memory that the lanes have read.
template <int D, int MODE>
__device__ __forceinline__ void store_row(__nv_bfloat16* row, const Lane<D, MODE>& L, const Pairs& p, bool live, __nv_bfloat16* scratch) {
  float v[8];
  from_pairs<MODE>(p, v);
  __nv_bfloat162 h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
  if (MODE == kMixed) {   // (put in order there, so that what is stored are whole rows)
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      scratch[L.ch_x(j)] = h[j].x;
      scratch[L.ch_y(j)] = h[j].y;
    }
    __syncwarp();
    if (live) *reinterpret_cast<uint4*>(row + L.c0) = *reinterpret_cast<const uint4*>(scratch + L.c0);
  } else if (!live) {
  } else if (MODE == kSide) {
    *reinterpret_cast<uint4*>(row + L.c0) = *reinterpret_cast<const uint4*>(&h[0]);
  } else if (MODE == kHalves) {
    *reinterpret_cast<uint2*>(row + L.c0) = *reinterpret_cast<const uint2*>(&h[0]);
    *reinterpret_cast<uint2*>(row + L.c1) = *reinterpret_cast<const uint2*>(&h[2]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      row[L.ch_x(j)] = h[j].x;
      row[L.ch_y(j)] = h[j].y;
    }
  }
}

// Weights (or biases) of the lane's pairs; `none` where there are none.
template <int D, int MODE>
__device__ __forceinline__ Pairs load_affine(const float* w, int head, const Lane<D, MODE>& L, float none) {
  float v[8] = {none, none, none, none, none, none, none, none};
  if (w) {
    w += (int64_t)head * D;
    if (MODE <= kHalves) {
      const float4 a = *reinterpret_cast<const float4*>(w + L.c0), b = *reinterpret_cast<const float4*>(w + L.c1);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) { v[2 * j] = w[L.ch_x(j)]; v[2 * j + 1] = w[L.ch_y(j)]; }
    }
  }
  return to_pairs<MODE>(v);
}

__device__ __forceinline__ uint64_t neg2(uint64_t a) { return a ^ 0x8000000080000000ull; }

// magnitude * cos and sin of the lane's pairs at a position.
struct Turn { uint64_t c[2], s[2]; };
template <int D, int MODE>
__device__ __forceinline__ Turn angles(const FrontDev& f, const Lane<D, MODE>& L, int64_t pos) {
  float c[4], s[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c[j] = 1.f;
    s[j] = 0.f;
    if (!L.rotated(j)) continue;
    const uint64_t u = f.turns[L.i0 + j] * (uint64_t)pos + (1ull << 61);         // (modulo whole turns)
    const int q = (int)(u >> 62), rest = (int)((u >> 32) & 0x3fffffffu) - (1 << 29);   // quadrant, and 2^-32 turns within it
    const float x = (float)rest * 1.4629180792671596e-09f, xx = x * x;           // 2 pi / 2^32
    const float sn = x * fmaf(fmaf(fmaf(fmaf(1.f / 362880, xx, -1.f / 5040), xx, 1.f / 120), xx, -1.f / 6), xx, 1.f);
    const float cs = fmaf(fmaf(fmaf(fmaf(fmaf(-1.f / 3628800, xx, 1.f / 40320), xx, -1.f / 720), xx, 1.f / 24), xx, -0.5f), xx, 1.f);
    const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;   // cos(x + q pi/2), sin(x + q pi/2)
    c[j] = f.mag * (q == 1 || q == 2 ? -a : a);
    s[j] = f.mag * (q >= 2 ? -b : b);
  }
  Turn t;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    t.c[k] = pack2(c[2 * k], c[2 * k + 1]);
    t.s[k] = pack2(s[2 * k], s[2 * k + 1]);
  }
  return t;
}
template <int D, int MODE>
__device__ __forceinline__ void rotate(const Lane<D, MODE>& L, const Turn& t, Pairs& p) {
  if (!L.rotated(0)) return;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint64_t a = p.x[k], b = p.y[k];
    uint64_t x = fma2(a, t.c[k], neg2(mul2(b, t.s[k]))), y = fma2(a, t.s[k], mul2(b, t.c[k]));
    if (MODE != kHalves && !L.rotated(2 * k + 1)) {   // (a channel that is not rotated is not touched by an infinity beside it)
      float x0, x1, y0, y1, a0, a1, b0, b1;
      unpack2(x, x0, x1); unpack2(y, y0, y1); unpack2(a, a0, a1); unpack2(b, b0, b1);
      const bool first = L.rotated(2 * k);
      x = pack2(first ? x0 : a0, a1);
      y = pack2(first ? y0 : b0, b1);
    }
    p.x[k] = x;
    p.y[k] = y;
  }
}

// Sums over the lanes of a row of N values per lane (N rows: 1 or 4), to all of them.  Four rows take half of the exchanges: every lane ends up with the sum of
// one row, and they are handed round.
template <int D, int N>
__device__ __forceinline__ void sum_rows(float (&v)[N]) {
  constexpr int LPR = D / 8;
  constexpr uint32_t ALL = 0xffffffffu;
  if constexpr (N == 1) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v[0] += __shfl_xor_sync(ALL, v[0], o);
  } else {
    static_assert(N == 4, "rows");
    const int lane = threadIdx.x & 31;
    const bool up = lane & (LPR / 2), up2 = lane & (LPR / 4);
    float a = up ? v[2] : v[0], b = up ? v[3] : v[1];
    a += __shfl_xor_sync(ALL, up ? v[0] : v[2], LPR / 2);
    b += __shfl_xor_sync(ALL, up ? v[1] : v[3], LPR / 2);
    float s = (up2 ? b : a) + __shfl_xor_sync(ALL, up2 ? a : b, LPR / 4);
#pragma unroll
    for (int o = LPR / 8; o > 0; o >>= 1) s += __shfl_xor_sync(ALL, s, o);
    const int from = lane & ~(LPR / 2 + LPR / 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __shfl_sync(ALL, s, from + (k >> 1) * (LPR / 2) + (k & 1) * (LPR / 4));
  }
}

// Norm over the D channels of the rows of a warp, N of each lane (every lane calls): statistics and sums in fp32, the mean taken off before the squares.
template <int D, int N>
__device__ __forceinline__ void norm(const FrontDev& f, const Pairs& w, const Pairs& b, Pairs (&p)[N]) {
  if (f.norm == KVM_NORM_NONE) return;
  float s[N];
  if (f.norm == KVM_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s1;
      unpack2(add2(add2(p[i].x[0], p[i].y[0]), add2(p[i].x[1], p[i].y[1])), s[i], s1);
      s[i] += s1;
    }
    sum_rows<D>(s);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float mean = s[i] * (-1.f / D);
      const uint64_t m2 = pack2(mean, mean);
#pragma unroll
      for (int k = 0; k < 2; ++k) { p[i].x[k] = add2(p[i].x[k], m2); p[i].y[k] = add2(p[i].y[k], m2); }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float s1;
    unpack2(fma2(p[i].y[1], p[i].y[1], fma2(p[i].x[1], p[i].x[1], fma2(p[i].y[0], p[i].y[0], mul2(p[i].x[0], p[i].x[0])))), s[i], s1);
    s[i] += s1;
  }
  sum_rows<D>(s);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float rstd;   // (2^-22.9; a variance that is no normal number counts as 0)
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(rstd) : "f"(fmaf(s[i], 1.f / D, f.eps)));
    const uint64_t r2 = pack2(rstd, rstd);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      p[i].x[k] = fma2(mul2(p[i].x[k], r2), w.x[k], b.x[k]);
      p[i].y[k] = fma2(mul2(p[i].y[k], r2), w.y[k], b.y[k]);
    }
  }
}

}  // namespace front
}  // namespace kvm
