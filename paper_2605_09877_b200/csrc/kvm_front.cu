// Front end of an exact layer: norm of every head's queries and keys and rotary positions in one pass (kvm_qk_norm_rope), and the same on the
// way into the 8-bit cache (kvm_cache_ingest), where the keys are normalised, rotated and quantised as they are written.
//
// A row is read once and written once; what bounds the kernels over many rows is memory, and the arithmetic in between (some 30 instructions per eight channels, and as
// many for an angle) has to hide behind it.  So:
//   - a lane has eight channels of a row, chosen so that the partners of a rotation are its own: nothing but the sums of the norm crosses lanes, and those of
//     four rows at a time (sum_rows);
//   - angles are fixed-point fractions of a turn: position times frequency modulo one turn is one 64-bit product, whatever the position, and the sine and cosine of
//     the eighth of a turn that is left a short polynomial.  (With angles in fp64 and the library's sincosf the pages of 4 x 8192 tokens took 74 us, now 63.)
//     They are computed once per token and kept over the heads;
//   - rows come by way of shared memory (cp.async), three items ahead: the registers are the rows' in work.  (2 x 8192 tokens, 32 heads of 128, LayerNorm: 79 us with
//     loads into registers and 16 warps per SM, 63 by way of shared memory, 57 with equal runs of items per block, 55.5 with the angles as above; a plain copy of the same
//     268 MB takes 44.)
// Few rows are bound by latency: one row per group of lanes, no loop (one token far into a sequence: 2.6 us).
#include <algorithm>
#include <atomic>
#include <cmath>

#include "kvm_cache.cuh"
#include "kvm_front.cuh"

namespace kvm {
namespace front {

using cache::AppendOut;

constexpr int kTokens = 4;    // tokens of a lane in the kernel over many rows
constexpr int kRows = 4;      // rows of a lane in the kernel over pages
// Up to so many rows of q (and k) each is done by itself.  us, one row at a time and over tiles: LayerNorm, 128 channels, 8192 rows 3.7 and 4.9, 16384 6.1 and 6.2, 24576 8.1 and
// 7.6, 32768 10.4 and 7.7; RMS, interleaved, 16384 7.7 and 8.4, 24576 10.2 and 9.7; 64 channels meet at 32768, 6.4 and 6.5.  Ingest, where few rows go with the pages and others have
// a launch of their own: 16384 9.4 and 10.4 (64 channels 6.4 and 7.0), 32768 16.7 and 12.4 (9.6 and 10.7).
constexpr int kFewRows = 16384;
constexpr int kPagesAhead = 3;
constexpr int kAhead = 3;     // stages of rows on their way (one of them is in use)

struct QkArgs {
  FrontDev f;
  Rows r[2];            // q, k
  const int32_t *start, *count;
  int32_t* status;
  int64_t T;
  int batch;
};

// Tokens before the call and in it; false: lengths that the call does not allow.
__device__ __forceinline__ bool qk_lengths(const QkArgs& a, int b, int& start, int& n) {
  start = a.start ? a.start[b] : 0;
  n = a.count ? a.count[b] : (int)a.T;
  return start >= 0 && n >= 0 && n <= a.T;
}

// Rows of a lane through the front end.
template <int D, int MODE, int N>
__device__ __forceinline__ void rows_through(const FrontDev& f, const Lane<D, MODE>& L, const Raw (&raw)[N], const Turn (&turn)[N], const Pairs& w, const Pairs& b, Pairs (&p)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[8];
    values_of(raw[i], v);
    p[i] = to_pairs<MODE>(v);
  }
  norm<D>(f, w, b, p);
#pragma unroll
  for (int i = 0; i < N; ++i) rotate(L, turn[i], p[i]);
}

// Few rows: D / 8 lanes per row, every row by itself.
template <int D, int MODE>
__global__ void __launch_bounds__(128) qk_rows_kernel(const __grid_constant__ QkArgs a) {
  constexpr int LPR = D / 8;
  const Lane<D, MODE> L(a.f, threadIdx.x % LPR);
  const int H = a.r[0].H + a.r[1].H;
  const int64_t row = (int64_t)blockIdx.x * (128 / LPR) + threadIdx.x / LPR, rows = a.batch * a.T * H;
  const bool there = row < rows;
  int64_t rest = there ? row : 0;
  const int hh = (int)(rest % H);
  rest /= H;
  const int b = (int)(rest / a.T), t = (int)(rest - b * a.T);
  const int which = hh >= a.r[0].H, head = hh - (which ? a.r[0].H : 0);
  const Rows& r = a.r[which];
  // (a row that the lengths leave out is read all the same: it is there)
  const Raw raw[1] = {load_raw(r.x + b * r.sx[0] + head * r.sx[1] + t * r.sx[2], L)};
  int start, n;
  const bool valid = qk_lengths(a, b, start, n);
  if (!valid && there && hh == 0 && t == 0 && L.i0 == 0) cache::report(a.status, KVM_ERR_INVALID_ARG);
  const Pairs w = load_affine(r.w, head, L, 1.f), bias = load_affine(r.b, head, L, 0.f);
  const Turn turn[1] = {angles(a.f, L, (int64_t)start + t)};
  Pairs p[1];
  rows_through(a.f, L, raw, turn, w, bias, p);
  store_row(r.y + b * r.sy[0] + head * r.sy[1] + t * r.sy[2], L, p[0], there && valid && t < n, nullptr);
}

// Many rows: a tile is 256 / LPR * 4 tokens (of the whole batch, one behind the other), and an item one head of a tile, q's then k's.  Every block takes an equal
// run of items, two blocks per SM.  A lane has four tokens: their angles stay in registers over the heads, a head's weights over the tokens, and the rows of the
// items ahead are on their way.
struct Tiles {
  cache::FastDiv by_T, by_H;
  int tokens, T, H;     // tokens of the batch, of a sequence; heads of q and k
  int items, per;       // of the call; of a block
};
template <int D, int MODE, class A>
__device__ __forceinline__ void rows_tiles(const A& a, const Tiles& ts) {
  constexpr int LPR = D / 8, RP = 256 / LPR, CH = kTokens, S = kAhead;
  constexpr bool STAGED = MODE != kSingle;
  extern __shared__ __align__(16) uint8_t stage_mem[];
  const Stage<D, 256, CH, S> stages{stage_mem};
  const FrontDev& f = a.front();
  const Lane<D, MODE> L(f, threadIdx.x % LPR);
  const int begin = blockIdx.x * ts.per, end = min(ts.items, begin + ts.per), Hq = a.rows(0).H;
  // the lane's tokens of a tile: (sequence, token), whether there is one
  auto token_of = [&](int tile, int i, int& b, int& t) {
    const int token = tile * (RP * CH) + i * RP + (int)threadIdx.x / LPR;
    b = ts.by_T.div(token);
    t = token - b * ts.T;
    return token < ts.tokens;
  };
  // what is asked for: item, its head, where its rows are
  int ahead = begin, ahead_h = begin - ts.by_H.div(begin) * ts.H;
  const __nv_bfloat16* px[CH];
  uint32_t there = 0;
  auto ask = [&](int stage, bool first) {
    if (ahead < end) {
      const Rows& r = a.rows(ahead_h >= Hq);
      if (first || ahead_h == 0 || ahead_h == Hq) {
        const int tile = ts.by_H.div(ahead);
        there = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          int b, t;
          if (token_of(tile, i, b, t)) there |= 1u << i; else b = t = 0;
          px[i] = r.x + b * r.sx[0] + t * r.sx[2] + (ahead_h - (ahead_h >= Hq ? Hq : 0)) * r.sx[1];
        }
      }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        if (there >> i & 1) stages.copy(stage, i, px[i]);
        px[i] += r.sx[1];
      }
      ++ahead;
      if (++ahead_h == ts.H) ahead_h = 0;
    }
    stages.commit();
  };
  int h = ahead_h;
  if (STAGED) {
#pragma unroll
    for (int k = 0; k < S - 1; ++k) ask(k, k == 0);
  }
  __nv_bfloat16* py[CH];
  const __nv_bfloat16* pd[CH];   // kSingle: the rows themselves
  Turn turn[CH];
  uint32_t live = 0;
  int stage = 0;
#pragma unroll 1
  for (int item = begin; item < end; ++item) {
    const int which = h >= Hq, head = h - (which ? Hq : 0);
    const Rows& r = a.rows(which);
    if (item == begin || h == 0 || h == Hq) {
      const int tile = ts.by_H.div(item);
      const bool fresh = item == begin || h == 0;
      if (fresh) live = 0;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        int b, t;
        const bool in = token_of(tile, i, b, t);
        if (!in) b = t = 0;
        if (fresh) {
          int start = 0, n = 0;
          if (in && !a.lengths(b, start, n)) {
            if (t == 0 && h == 0 && L.i0 == 0) a.invalid();
            start = n = 0;
          }
          if (in && t < n) live |= 1u << i;
          turn[i] = angles(f, L, (int64_t)start + t);
        }
        py[i] = r.y + b * r.sy[0] + t * r.sy[2] + head * r.sy[1];
        if (!STAGED) pd[i] = r.x + b * r.sx[0] + t * r.sx[2] + head * r.sx[1];
      }
    }
    const Pairs w = load_affine(r.w, head, L, 1.f), bias = load_affine(r.b, head, L, 0.f);
    Raw raw[CH];
    if (STAGED) {
      stages.wait();                                  // (all lanes have read the stage that is asked for next)
      ask(stage == 0 ? S - 1 : stage - 1, false);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      raw[i] = load_raw(STAGED ? stages.row(stage, i) : pd[i], L);
      if (!STAGED) pd[i] += r.sx[1];
    }
    Pairs p[CH];
    rows_through(f, L, raw, turn, w, bias, p);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      store_row(py[i], L, p[i], live >> i & 1, STAGED ? stages.row(stage, i) : nullptr);
      py[i] += r.sy[1];
    }
    if (++stage == S) stage = 0;
    if (++h == ts.H) h = 0;
  }
}

struct QkTiles {        // what rows_tiles asks of a call without a cache
  const QkArgs& a;
  __device__ const FrontDev& front() const { return a.f; }
  __device__ const Rows& rows(int which) const { return a.r[which]; }
  __device__ bool lengths(int b, int& start, int& n) const { return qk_lengths(a, b, start, n); }
  __device__ void invalid() const { cache::report(a.status, KVM_ERR_INVALID_ARG); }
};
template <int D, int MODE>
__global__ void __launch_bounds__(256, 2) qk_tiles_kernel(const __grid_constant__ QkArgs a, const __grid_constant__ Tiles ts) {
  rows_tiles<D, MODE>(QkTiles{a}, ts);
}

// ---- into the cache ----------------------------------------------------------------------------------------------------------

struct IngestArgs {
  FrontDev f;
  cache::Params p;
  Rows q, k, v;         // (k.y, v.y and their strides are not used)
  AppendOut o;
  int chunks, heads;    // head chunks of k and v
  int tpp;              // threads per page
  int groups;           // blocks that share the pages of one sequence
  int64_t k_blocks;     // blocks of k, those of v follow, and of q where there are few rows
};
struct IngestTiles {    // what rows_tiles asks of a call over a cache
  const IngestArgs& a;
  __device__ const FrontDev& front() const { return a.f; }
  __device__ const Rows& rows(int) const { return a.q; }
  __device__ bool lengths(int b, int& start, int& n) const { return cache::seq_lengths(a.p, b, start, n); }
  __device__ void invalid() const {}   // (the blocks of k report)
};

// Least e >= -64 with x <= 448 * 2^e, from the bits of x >= 0.
__device__ __forceinline__ int least_exp(uint32_t bits) {
  return max((int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), cache::kLeastExp);
}
// max(|a|, |b|, |c|); NaN if one is
__device__ __forceinline__ float max_abs(float a, float b, float c) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// A lane's eight values as codes, in the order of memory (two runs of four channels) where the layout has runs.
__device__ __forceinline__ void codes_of(const float (&v)[8], float inv, uint32_t& a, uint32_t& b) {
  a = cache::to_e4m3x2(v[0] * inv, v[1] * inv) | (cache::to_e4m3x2(v[2] * inv, v[3] * inv) << 16);
  b = cache::to_e4m3x2(v[4] * inv, v[5] * inv) | (cache::to_e4m3x2(v[6] * inv, v[7] * inv) << 16);
}
template <int D, int MODE>
__device__ __forceinline__ void store_codes(uint8_t* row, const Lane<D, MODE>& L, uint32_t a, uint32_t b) {
  if (MODE <= kHalves) {
    *reinterpret_cast<uint32_t*>(row + L.c0) = a;
    *reinterpret_cast<uint32_t*>(row + L.c1) = b;
  } else {   // (x0 y0 x1 y1 ...)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = (j < 2 ? a : b) >> (16 * (j & 1));
      row[L.ch_x(j)] = (uint8_t)w;
      row[L.ch_y(j)] = (uint8_t)(w >> 8);
    }
  }
}
__device__ __forceinline__ uint32_t rescaled4(uint32_t w, float m) {
  const float2 a = cache::e4m3x2_to_float2(w & 0xffffu), b = cache::e4m3x2_to_float2(w >> 16);
  return cache::to_e4m3x2(a.x * m, a.y * m) | (cache::to_e4m3x2(b.x * m, b.y * m) << 16);
}

// The pages of one sequence, k or v, through a run of heads: tpp threads per page, four rows per thread; see append_kernel for the scale and
// the codes, which follow the maximum over the rows of a page.
template <int D, int TH, int MODE, bool KEYS>
__device__ __forceinline__ void pages_tile(const IngestArgs& a, int group, int chunk, int b) {
  constexpr int LPR = D / 8, CH = kRows, S = kPagesAhead;
  constexpr bool STAGED = MODE != kSingle;
  extern __shared__ __align__(16) uint8_t stage_mem[];
  __shared__ uint32_t s_top[2][TH / 32];
  const Stage<D, TH, CH, S> stages{stage_mem};
  const cache::Params& p = a.p;
  const Rows& r = KEYS ? a.k : a.v;
  const FrontDev& f = a.f;
  const int tpp = a.tpp, tt = threadIdx.x & (tpp - 1), warp = threadIdx.x >> 5, step = tpp / LPR;   // rows of a lane: tt / LPR + i * step
  int start, n;
  if (!cache::seq_lengths(p, b, start, n)) {   // (the same for the whole block)
    if (KEYS && group == 0 && chunk == 0 && threadIdx.x == 0) cache::report(p.status, KVM_ERR_INVALID_ARG);
    return;
  }
  const int per = TH / tpp, block0 = (start >> p.page_shift) + group * per, block = block0 + threadIdx.x / tpp;
  if ((int64_t)block0 << p.page_shift >= (int64_t)start + n) return;   // (so is this)
  const int64_t pos0 = (int64_t)block << p.page_shift;
  const int r0 = (int)max((int64_t)0, start - pos0);                           // rows [0, r0) are held, [r0, r1) are new
  int r1 = (int)max((int64_t)0, min((int64_t)p.page, (int64_t)start + n - pos0));
  int page = 0;
  if (r1 > r0) {
    page = p.pages[(int64_t)b * p.max_pages + block];
    if (page < 0 || page >= p.n_pages) {
      if (tt == 0) cache::report(p.status, KVM_ERR_INVALID_ARG);
      r1 = 0;
    }
  }
  const bool live = r1 > r0;
  const Lane<D, MODE> L(f, tt % LPR);
  const int h0 = chunk * a.heads, h1 = min(h0 + a.heads, p.Hkv), row0 = tt / LPR;
  const __nv_bfloat16* px = r.x + b * r.sx[0] + h0 * r.sx[1] + (pos0 + row0 - start) * r.sx[2];   // (rows in front of the call's: not looked at)
  Turn turn[CH];
  uint32_t fresh = 0;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int row = row0 + i * step;
    if (row >= r0 && row < r1) fresh |= 1u << i;
  }
  const int64_t apart = step * r.sx[2];
  int ahead = h0;   // heads that have been asked for
  auto ask = [&](int stage) {
    if (ahead < h1) {
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (fresh >> i & 1) stages.copy(stage, i, px + i * apart);
      px += r.sx[1];
      ++ahead;
    }
    stages.commit();
  };
  if (STAGED) {
#pragma unroll
    for (int k = 0; k < S - 1; ++k) ask(k);
  }
  if (KEYS) {
#pragma unroll
    for (int i = 0; i < CH; ++i) turn[i] = angles(f, L, pos0 + row0 + i * step);
  }
  int stage = 0;
#pragma unroll 1
  for (int h = h0; h < h1; ++h) {
    const int64_t unit = (int64_t)page * p.Hkv + h;
    uint8_t* codes = a.o.codes[KEYS ? 0 : 1] + (unit * p.page + row0) * D;
    float* scale = a.o.scales[KEYS ? 0 : 1] + unit;
    const float old = live && r0 > 0 ? *scale : 0.f;
    Raw raw[CH];
    if (STAGED) {
      stages.wait();                                  // (all lanes have read the stage that is asked for next)
      ask(stage == 0 ? S - 1 : stage - 1);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      raw[i].a = raw[i].b = make_uint2(0, 0);
      if (fresh >> i & 1) raw[i] = load_raw(STAGED ? stages.row(stage, i) : px + i * apart, L);
    }
    if (!STAGED) px += r.sx[1];
    if (++stage == S) stage = 0;
    float v[CH][8];
    if (KEYS) {
      const Pairs w = load_affine(r.w, h, L, 1.f), bias = load_affine(r.b, h, L, 0.f);
      Pairs x[CH];
      rows_through(f, L, raw, turn, w, bias, x);
#pragma unroll
      for (int i = 0; i < CH; ++i) from_pairs<MODE>(x[i], v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < CH; ++i) values_of(raw[i], v[i]);
    }
    float most = 0.f;   // (a NaN stays one: above all others in what follows)
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (fresh >> i & 1) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) most = max_abs(most, v[i][j], v[i][j + 1]);
      }
    uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(most) & 0x7fffffffu);
    if (tpp > 32) {   // (uniform)
      const int at = (h - h0) & 1;   // (two sets: a thread is never two heads ahead of another)
      if ((threadIdx.x & 31) == 0) s_top[at][warp] = top;
      __syncthreads();
      const int warps = tpp / 32;
      top = __reduce_max_sync(0xffffffffu, s_top[at][(warp & ~(warps - 1)) + (threadIdx.x & (warps - 1))]);
    } else {
      __syncwarp();   // (every lane has read the old scale before one writes the new one)
    }
    if (!live) continue;
    const int e_old = r0 > 0 ? max(cache::scale_exp(old), cache::kLeastExp) : cache::kLeastExp;
    const bool poisoned = top >= 0x7f800000u || e_old > 127;
    const int e = max(least_exp(top), e_old);
    if (tt == 0) *scale = poisoned ? __int_as_float(0x7fc00000) : cache::exp2i(e);
    const float inv = cache::exp2i(-e);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      uint8_t* dst = codes + i * step * D;
      if (fresh >> i & 1) {
        uint32_t ca = 0, cb = 0;
        if (!poisoned) codes_of(v[i], inv, ca, cb);
        store_codes(dst, L, ca, cb);
      } else if (row0 + i * step < r0 && e > e_old && !poisoned) {
        const float down = e - e_old > 126 ? 0.f : cache::exp2i(e_old - e);
        uint2* held = reinterpret_cast<uint2*>(dst + (tt % LPR) * 8);
        const uint2 w = *held;
        *held = make_uint2(rescaled4(w.x, down), rescaled4(w.y, down));
      }
    }
  }
}

// Rows of q one by one, D / 8 lanes each.
template <int D, int TH, int MODE>
__device__ __forceinline__ void q_rows(const IngestArgs& a, int64_t block) {
  constexpr int LPR = D / 8;
  const Lane<D, MODE> L(a.f, threadIdx.x % LPR);
  const Rows& r = a.q;
  const int64_t row = block * (TH / LPR) + threadIdx.x / LPR;
  const bool there = row < (int64_t)a.p.batch * a.p.T * r.H;
  int64_t rest = there ? row : 0;
  const int head = (int)(rest % r.H);
  rest /= r.H;
  const int b = (int)(rest / a.p.T), t = (int)(rest - b * a.p.T);
  const Raw raw[1] = {load_raw(r.x + b * r.sx[0] + head * r.sx[1] + t * r.sx[2], L)};
  int start, n;
  const bool valid = cache::seq_lengths(a.p, b, start, n);
  const Pairs w = load_affine(r.w, head, L, 1.f), bias = load_affine(r.b, head, L, 0.f);
  const Turn turn[1] = {angles(a.f, L, (int64_t)start + t)};
  Pairs p[1];
  rows_through(a.f, L, raw, turn, w, bias, p);
  store_row(r.y + b * r.sy[0] + head * r.sy[1] + t * r.sy[2], L, p[0], there && valid && t < n, nullptr);
}

template <int D, int TH, int MODE>
__global__ void __launch_bounds__(TH, 512 / TH) ingest_pages_kernel(const __grid_constant__ IngestArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (ingest_q_kernel, which has nothing to wait for before its end)
  int64_t i = blockIdx.x;
  if (i >= 2 * a.k_blocks) {   // (a call of few rows)
    q_rows<D, TH, MODE == kMixed ? kSingle : MODE>(a, i - 2 * a.k_blocks);
    return;
  }
  const bool keys = i < a.k_blocks;
  if (!keys) i -= a.k_blocks;
  const int chunk = (int)(i % a.chunks);
  i /= a.chunks;
  const int group = (int)(i % a.groups), b = (int)(i / a.groups);
  if (keys) pages_tile<D, TH, MODE, true>(a, group, chunk, b);
  else pages_tile<D, TH, MODE == kSingle ? kSingle : kSide, false>(a, group, chunk, b);   // (values: eight channels side by side)
}
template <int D, int MODE>
__global__ void __launch_bounds__(256, 2) ingest_q_kernel(const __grid_constant__ IngestArgs a, const __grid_constant__ Tiles ts) {
  rows_tiles<D, MODE>(IngestTiles{a}, ts);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // (what follows this grid counts on the end of the one before it)
}

// One token per sequence: a warp per row of k or v, D / 8 lanes per row of q.
template <int D, int MODE, bool KEYS>
__device__ __forceinline__ void token_into(const IngestArgs& a, int64_t unit_of_call) {
  constexpr int LPR = D / 8;
  const cache::Params& p = a.p;
  const FrontDev& f = a.f;
  const int lane = threadIdx.x & 31;
  const Lane<D, MODE> L(f, lane % LPR);
  const Rows& r = KEYS ? a.k : a.v;
  const int b = (int)(unit_of_call / p.Hkv), h = (int)(unit_of_call - (int64_t)b * p.Hkv);
  const Raw raw = load_raw(r.x + b * r.sx[0] + h * r.sx[1], L);   // (there whatever the lengths are)
  const Pairs w = load_affine(KEYS ? r.w : nullptr, h, L, 1.f), bias = load_affine(KEYS ? r.b : nullptr, h, L, 0.f);
  int start, n;
  if (!cache::seq_lengths(p, b, start, n)) {
    if (KEYS && h == 0 && lane == 0) cache::report(p.status, KVM_ERR_INVALID_ARG);
    return;
  }
  if (n == 0) return;
  const int page = p.pages[(int64_t)b * p.max_pages + (start >> p.page_shift)], r0 = start & (p.page - 1);
  if (page < 0 || page >= p.n_pages) {
    if (lane == 0) cache::report(p.status, KVM_ERR_INVALID_ARG);
    return;
  }
  const int64_t unit = (int64_t)page * p.Hkv + h;
  uint8_t* codes = a.o.codes[KEYS ? 0 : 1] + unit * p.page * D;
  float* scale = a.o.scales[KEYS ? 0 : 1] + unit;
  const float old = r0 > 0 ? *scale : 0.f;
  float v[8];
  values_of(raw, v);
  if (KEYS) {
    const Raw raws[1] = {raw};
    const Turn turn[1] = {angles(f, L, start)};
    Pairs x[1];
    rows_through(f, L, raws, turn, w, bias, x);
    from_pairs<MODE>(x[0], v);
  }
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = __reduce_max_sync(0xffffffffu, top);
  const int e_old = r0 > 0 ? max(cache::scale_exp(old), cache::kLeastExp) : cache::kLeastExp;
  const bool poisoned = top >= 0x7f800000u || e_old > 127;
  const int e = max(least_exp(top), e_old);
  __syncwarp();   // (every lane has read the old scale before one writes the new one)
  if (lane == 0) *scale = poisoned ? __int_as_float(0x7fc00000) : cache::exp2i(e);
  if (lane < LPR) {
    uint32_t ca = 0, cb = 0;
    if (!poisoned) codes_of(v, cache::exp2i(-e), ca, cb);
    store_codes(codes + (int64_t)r0 * D, L, ca, cb);
  }
  if (e > e_old && !poisoned) {   // (r0 = 0: nothing is held)
    const float down = e - e_old > 126 ? 0.f : cache::exp2i(e_old - e);
#pragma unroll 1
    for (int i = lane; i < r0 * (D / 16); i += 32) {
      uint4* held = reinterpret_cast<uint4*>(codes) + i;
      const uint4 w = *held;
      *held = make_uint4(rescaled4(w.x, down), rescaled4(w.y, down), rescaled4(w.z, down), rescaled4(w.w, down));
    }
  }
}
template <int D, int MODE>
__global__ void __launch_bounds__(128) ingest_token_kernel(const __grid_constant__ IngestArgs a) {
  constexpr int LPR = D / 8;
  const cache::Params& p = a.p;
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5), units = (int64_t)p.batch * p.Hkv;
  if (warp < units) {
    token_into<D, MODE, true>(a, warp);
  } else if (warp < 2 * units) {
    token_into<D, MODE == kSingle ? kSingle : kSide, false>(a, warp - units);
  } else if (a.q.H > 0) {   // (without q: a block's warps beyond the work)
    const Lane<D, MODE> L(a.f, lane % LPR);
    const Rows& r = a.q;
    int64_t row = (warp - 2 * units) * (32 / LPR) + lane / LPR;
    const bool there = row < (int64_t)p.batch * r.H;
    if (!there) row = 0;
    const int b = (int)(row / r.H), h = (int)(row - (int64_t)b * r.H);
    const Raw raw[1] = {load_raw(r.x + b * r.sx[0] + h * r.sx[1], L)};
    const Pairs w = load_affine(r.w, h, L, 1.f), bias = load_affine(r.b, h, L, 0.f);
    int start, n;
    const bool valid = cache::seq_lengths(p, b, start, n);
    const Turn turn[1] = {angles(a.f, L, start)};
    Pairs x[1];
    rows_through(a.f, L, raw, turn, w, bias, x);
    store_row(r.y + b * r.sy[0] + h * r.sy[1], L, x[0], there && valid && n > 0, nullptr);
  }
}

// ---- arguments ---------------------------------------------------------------------------------------------------------------

static bool within(double x, double lo, double hi) { return x >= lo && x <= hi; }   // (false for a NaN)

static kvm_status_t check_front(const kvm_front_t* f, int d) {
  if (!f) return KVM_ERR_INVALID_ARG;
  if (f->norm < KVM_NORM_NONE || f->norm > KVM_NORM_RMS || f->layout < KVM_ROPE_HALF || f->layout > KVM_ROPE_INTERLEAVED ||
      f->scaling < KVM_ROPE_PLAIN || f->scaling > KVM_ROPE_PARTS) return KVM_ERR_INVALID_ARG;
  if (f->rope_dims < 0 || f->rope_dims > d || f->rope_dims % 2) return KVM_ERR_INVALID_ARG;
  if (f->norm == KVM_NORM_NONE) {
    if (f->q_weight || f->q_bias || f->k_weight || f->k_bias) return KVM_ERR_INVALID_ARG;
  } else if (!within(f->eps, 0.0, 1e30)) {
    return KVM_ERR_INVALID_ARG;
  }
  if (f->rope_dims > 0) {
    if (!within(f->base, 1.0, 1e30) || !within(f->magnitude, 1e-30, 1e30)) return KVM_ERR_INVALID_ARG;
    if (f->scaling != KVM_ROPE_PLAIN && !within(f->factor, 1.0, 1e30)) return KVM_ERR_INVALID_ARG;
    if (f->scaling == KVM_ROPE_PARTS && (f->original_len < 1 || !within(f->low, 0.0, 1e30) || !within(f->high, 0.0, 1e30) || f->low >= f->high)) return KVM_ERR_INVALID_ARG;
  }
  if (f->rope_dims > 0 && f->frequencies) {
    if (!cache::aligned(f->frequencies, 8)) return KVM_ERR_INVALID_ARG;
    for (int i = 0; i < f->rope_dims / 2; ++i)
      if (!within(f->frequencies[i], 0.0, 1.0)) return KVM_ERR_INVALID_ARG;
  }
  for (const float* w : {f->q_weight, f->q_bias, f->k_weight, f->k_bias})
    if (!cache::aligned(w, 4)) return KVM_ERR_INVALID_ARG;
  return KVM_OK;
}

// Radians per position of pair i.
static double frequency(const kvm_front_t* f, int i) {
  if (f->frequencies) return f->frequencies[i];
  const double w = std::pow(f->base, -2.0 * i / f->rope_dims);
  if (f->scaling == KVM_ROPE_LINEAR) return w / f->factor;
  if (f->scaling == KVM_ROPE_PARTS) {
    const double turns = (double)f->original_len * w / 6.283185307179586476925;
    const double keep = std::min(1.0, std::max(0.0, (turns - f->low) / (f->high - f->low)));
    return keep * w + (1.0 - keep) * w / f->factor;
  }
  return w;
}

static FrontDev device_front(const kvm_front_t* f) {
  FrontDev x = {};
  x.norm = f->norm;
  x.eps = f->norm == KVM_NORM_NONE ? 0.f : f->eps;
  x.h = f->rope_dims / 2;
  x.half = f->layout == KVM_ROPE_HALF && x.h > 0;   // (without rotation kSide and kSingle have the same pairs, and sums the same order)
  x.mag = x.h ? (float)f->magnitude : 1.f;
  constexpr long double kTurns = 18446744073709551616.0L / 6.283185307179586476925286766559L;   // 2^64 / (2 pi)
  for (int i = 0; i < x.h; ++i) x.turns[i] = (uint64_t)(frequency(f, i) * kTurns);   // (f_i <= 1: below 2^62)
  return x;
}

// Rows of q, k or v with their strides; y may be NULL (nothing is written).  aligned: cleared where they cannot be accessed 16 bytes at a time.
static bool rows_of(Rows& r, bool& aligned, const kvm_front_t* f, int which, const void* x, void* y, int64_t B, int64_t H, int64_t T, int d, const int64_t* sx, const int64_t* sy) {
  if (!x || !cache::aligned(x, 2) || !cache::aligned(y, 2)) return false;
  if (!cache::strides_of(sx, B, H, T, d, false, r.sx) || !cache::strides_of(sy, B, H, T, d, true, r.sy)) return false;
  if (x == y) {   // in place: the same rows
    const int64_t n[3] = {B, H, T};
    for (int i = 0; i < 3; ++i)
      if (n[i] > 1 && r.sx[i] != r.sy[i]) return false;
  }
  r.x = (const __nv_bfloat16*)x; r.y = (__nv_bfloat16*)y;
  r.H = (int)H;
  r.w = which == 0 ? f->q_weight : which == 1 ? f->k_weight : nullptr;
  r.b = which == 0 ? f->q_bias : which == 1 ? f->k_bias : nullptr;
  aligned = aligned && cache::rows_aligned(x, r.sx) && cache::rows_aligned(y, r.sy) && cache::aligned(r.w, 16) && cache::aligned(r.b, 16);
  return true;
}

static int mode_of(const kvm_front_t* f, bool aligned) {
  if (!aligned) return kSingle;
  if (f->layout == KVM_ROPE_INTERLEAVED || f->rope_dims == 0) return kSide;
  return f->rope_dims / 2 % 4 == 0 ? kHalves : kMixed;
}

// Heads of a chunk: as many as leave `want` blocks, 16 at most (the angles of a block's tokens are computed once per chunk).
static int heads_of_chunk(int64_t blocks_per_head, int H, int64_t want) {
  const int most = (int)std::max<int64_t>(1, std::min<int64_t>({blocks_per_head * H / want, 16, H}));
  const int chunks = (H + most - 1) / most;
  return (H + chunks - 1) / chunks;
}

// Raises the limit of shared memory of a kernel on the current device (once per device).
template <auto KERNEL, int SMEM>
static bool room_for() {
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return false; }
  if (dev > 63 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) != cudaSuccess) { cudaGetLastError(); return false; }
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return true;
}

// The items of a call over its blocks; false: more than is numbered in 32 bits.
template <int D>
static bool tiles_of_call(int64_t batch, int64_t T, int H, Tiles& ts, int& blocks) {
  constexpr int TOK = 256 / (D / 8) * kTokens;
  const int64_t tokens = batch * T, items = (tokens + TOK - 1) / TOK * H;
  if (tokens > INT32_MAX - TOK || items > INT32_MAX / 2) return false;
  ts.by_T = cache::FastDiv((uint32_t)T); ts.by_H = cache::FastDiv(H);
  ts.tokens = (int)tokens; ts.T = (int)T; ts.H = H;
  ts.items = (int)items;
  ts.per = (int)((items + 2 * 148 - 1) / (2 * 148));
  blocks = (int)((items + ts.per - 1) / ts.per);
  return true;
}
template <int D, int MODE>
constexpr int kTilesSmem = MODE == kSingle ? 0 : Stage<D, 256, kTokens, kAhead>::kBytes;

template <int D, int MODE>
static kvm_status_t launch_qk(QkArgs& a, cudaStream_t s) {
  constexpr int LPR = D / 8;
  const int H = a.r[0].H + a.r[1].H;
  const int64_t tokens = a.batch * a.T;
  if (tokens * H <= kFewRows) {
    qk_rows_kernel<D, MODE == kMixed ? kSingle : MODE><<<(unsigned)((tokens * H * LPR + 127) / 128), 128, 0, s>>>(a);
  } else {
    Tiles ts;
    int blocks;
    if (!tiles_of_call<D>(a.batch, a.T, H, ts, blocks)) return KVM_ERR_UNSUPPORTED;
    if (!room_for<qk_tiles_kernel<D, MODE>, kTilesSmem<D, MODE>>()) return KVM_ERR_CUDA;
    qk_tiles_kernel<D, MODE><<<blocks, 256, kTilesSmem<D, MODE>, s>>>(a, ts);
  }
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}

template <int D, int TH, int MODE>
static kvm_status_t launch_pages(const IngestArgs& a, int64_t q_rows, cudaStream_t s) {
  constexpr int SMEM = MODE == kSingle ? 0 : Stage<D, TH, kRows, kPagesAhead>::kBytes;
  if (!room_for<ingest_pages_kernel<D, TH, MODE>, SMEM>()) return KVM_ERR_CUDA;
  ingest_pages_kernel<D, TH, MODE><<<(unsigned)(2 * a.k_blocks + (q_rows * (D / 8) + TH - 1) / TH), TH, SMEM, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}
template <int D, int MODE>
static kvm_status_t launch_ingest(IngestArgs& a, cudaStream_t s) {
  const cache::Params& p = a.p;
  if (p.T == 1) {
    const int64_t units = (int64_t)p.batch * p.Hkv, rpw = 32 / (D / 8);
    const int64_t warps = 2 * units + ((int64_t)p.batch * a.q.H + rpw - 1) / rpw;
    ingest_token_kernel<D, MODE == kMixed ? kSingle : MODE><<<(unsigned)((warps + 3) / 4), 128, 0, s>>>(a);
    return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
  }
  a.tpp = p.page * D / 8 / kRows;
  const int TH = std::max(256, a.tpp);
  const int64_t pages = (p.T + p.page - 2) / p.page + 1;   // pages that T consecutive tokens can touch
  const int64_t groups = (pages + TH / a.tpp - 1) / (TH / a.tpp);
  a.groups = (int)groups;
  a.heads = heads_of_chunk(groups * p.batch, p.Hkv, 2 * 148);
  a.chunks = (p.Hkv + a.heads - 1) / a.heads;
  a.k_blocks = groups * p.batch * a.chunks;
  Tiles ts;
  int blocks = 0;
  if (2 * a.k_blocks > INT32_MAX - kFewRows || (a.q.H > 0 && !tiles_of_call<D>(p.batch, p.T, a.q.H, ts, blocks))) return KVM_ERR_UNSUPPORTED;
  const int64_t q_rows = (int64_t)p.batch * p.T * a.q.H;
  const bool few = q_rows <= kFewRows;   // (they go with the pages: one launch)
  if (!few && !room_for<ingest_q_kernel<D, MODE>, kTilesSmem<D, MODE>>()) return KVM_ERR_CUDA;   // (before anything is written)
  const kvm_status_t rc = TH == 256 ? launch_pages<D, 256, MODE>(a, few ? q_rows : 0, s) : launch_pages<D, 512, MODE>(a, few ? q_rows : 0, s);
  if (rc != KVM_OK) return rc;
  if (!few) {
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // (as the last blocks of the pages leave room)
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at; lc.numAttrs = 1; lc.stream = s;
    lc.gridDim = dim3(blocks); lc.blockDim = dim3(256); lc.dynamicSmemBytes = kTilesSmem<D, MODE>;
    if (cudaLaunchKernelEx(&lc, ingest_q_kernel<D, MODE>, a, ts) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  }
  return KVM_OK;
}

template <int D>
static kvm_status_t launch_qk_d(QkArgs& a, int mode, cudaStream_t s) {
  switch (mode) {
    case kSide: return launch_qk<D, kSide>(a, s);
    case kHalves: return launch_qk<D, kHalves>(a, s);
    case kMixed: return launch_qk<D, kMixed>(a, s);
    default: return launch_qk<D, kSingle>(a, s);
  }
}
template <int D>
static kvm_status_t launch_ingest_d(IngestArgs& a, int mode, cudaStream_t s) {
  switch (mode) {
    case kSide: return launch_ingest<D, kSide>(a, s);
    case kHalves: return launch_ingest<D, kHalves>(a, s);
    case kMixed: return launch_ingest<D, kMixed>(a, s);
    default: return launch_ingest<D, kSingle>(a, s);
  }
}

}  // namespace front
}  // namespace kvm

using namespace kvm;
using namespace kvm::front;

#define KVM_API __attribute__((visibility("default")))

extern "C" {

KVM_API kvm_status_t kvm_rope_frequencies(const kvm_front_t* front, int32_t head_dim, double* out) {
  if (head_dim != 64 && head_dim != 128) return KVM_ERR_UNSUPPORTED;
  const kvm_status_t rc = check_front(front, head_dim);
  if (rc != KVM_OK) return rc;
  if (!out && front->rope_dims > 0) return KVM_ERR_INVALID_ARG;
  for (int i = 0; i < front->rope_dims / 2; ++i) out[i] = frequency(front, i);
  return KVM_OK;
}

KVM_API kvm_status_t kvm_qk_norm_rope(const kvm_front_t* front, const void* q, const void* k, const int32_t* start, const int32_t* count, int32_t batch,
                                      int32_t n_q_heads, int32_t n_kv_heads, int64_t n_tokens, int32_t head_dim, void* q_out, void* k_out,
                                      const int64_t* q_strides, const int64_t* k_strides, const int64_t* q_out_strides,
                                      const int64_t* k_out_strides, int32_t* status, void* cuda_stream) {
  if (head_dim != 64 && head_dim != 128) return KVM_ERR_UNSUPPORTED;
  const kvm_status_t rc = check_front(front, head_dim);
  if (rc != KVM_OK) return rc;
  if (batch < 1 || n_tokens < 1 || (!q && !k) || (q && n_q_heads < 1) || (k && n_kv_heads < 1)) return KVM_ERR_INVALID_ARG;
  if (!cache::aligned(start, 4) || !cache::aligned(count, 4) || !cache::aligned(status, 4)) return KVM_ERR_INVALID_ARG;
  if (batch > 65535 || n_tokens > (1 << 30) || (q && n_q_heads > 16384) || (k && n_kv_heads > 16384)) return KVM_ERR_UNSUPPORTED;
  QkArgs a = {};
  a.f = device_front(front);
  bool aligned = true;
  if (q && (!q_out || !rows_of(a.r[0], aligned, front, 0, q, q_out, batch, n_q_heads, n_tokens, head_dim, q_strides, q_out_strides))) return KVM_ERR_INVALID_ARG;
  if (k && (!k_out || !rows_of(a.r[1], aligned, front, 1, k, k_out, batch, n_kv_heads, n_tokens, head_dim, k_strides, k_out_strides))) return KVM_ERR_INVALID_ARG;
  a.start = start; a.count = count; a.status = status;
  a.T = n_tokens; a.batch = batch;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const int mode = mode_of(front, aligned);
  return head_dim == 128 ? launch_qk_d<128>(a, mode, s) : launch_qk_d<64>(a, mode, s);
}

KVM_API kvm_status_t kvm_cache_ingest(const kvm_cache_t* cache, const kvm_cache_call_t* call, const kvm_front_t* front, const void* q, int32_t n_q_heads,
                                      const void* k, const void* v, void* q_out, const int64_t* q_strides, const int64_t* k_strides,
                                      const int64_t* v_strides, const int64_t* q_out_strides, int32_t* status, void* cuda_stream) {
  kvm_status_t rc = cache::check_cache(cache, true);
  if (rc == KVM_OK) rc = cache::check_call(cache, call, true);
  if (rc == KVM_OK) rc = check_front(front, cache->head_dim);
  if (rc != KVM_OK) return rc;
  if (!cache::aligned(status, 4) || (q && (n_q_heads < 1 || !q_out))) return KVM_ERR_INVALID_ARG;
  if (q && n_q_heads > 16384) return KVM_ERR_UNSUPPORTED;
  IngestArgs a = {};
  a.f = device_front(front);
  a.p = cache::params_of(cache, call, status);
  const int64_t B = a.p.batch, T = a.p.T;
  const int d = cache->head_dim;
  bool aligned = true;
  if (q && !rows_of(a.q, aligned, front, 0, q, q_out, B, n_q_heads, T, d, q_strides, q_out_strides)) return KVM_ERR_INVALID_ARG;
  if (!rows_of(a.k, aligned, front, 1, k, nullptr, B, a.p.Hkv, T, d, k_strides, nullptr) || !rows_of(a.v, aligned, front, 2, v, nullptr, B, a.p.Hkv, T, d, v_strides, nullptr)) return KVM_ERR_INVALID_ARG;
  a.o.codes[0] = (uint8_t*)cache->k; a.o.codes[1] = (uint8_t*)cache->v;
  a.o.scales[0] = cache->k_scale; a.o.scales[1] = cache->v_scale;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const int mode = mode_of(front, aligned);
  return d == 128 ? launch_ingest_d<128>(a, mode, s) : launch_ingest_d<64>(a, mode, s);
}

}  // extern "C"
