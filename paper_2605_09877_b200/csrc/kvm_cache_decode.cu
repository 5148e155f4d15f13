// Attention of a few tokens per sequence (decode, speculative tokens) over the 8-bit cache.
//
// The columns of a (sequence, kv head) "unit" are its query rows, (token, head of the group) pairs, at most NC of them.  For every tile of
// 128 keys (tokens of the page table, one TMA box per page for keys and one for values):
//     S^T [128 keys x columns] = K8 (q_hi + q_lo)^T,    O^T [d x columns] = V8^T (p_hi + p_lo)^T
// on the tensor cores in kind::f8f6f4, with the codes of the cache as the A operands, as they lie in memory: nothing is converted on the
// way in.  q, scaled by a power of two per row so that its largest channel is in [128, 256), is the sum of two e4m3 numbers (4 + 4
// significant bits: all 8 of bf16; channels below 2^-10 of the largest lose what is below 2^-18 of it), and so are the weights p (2^-8 of a
// weight, 2^-18 of the tile's largest weight where it is subnormal).  hi and lo are separate columns of the same MMA, so that the codes pass
// through the tensor core once.  The scale of a block of keys multiplies the logits of its lanes; the scale of a block of values is added to
// the exponent of the weights (relative to the largest of the tile) and taken out of the row sum again.
// Every tile has a softmax reference of its own (its largest logit), so the weights use the whole range of e4m3, and the running
// result is rescaled in registers: thread = channel, one column of O per register.
//
// All tiles of all units form one list, of which every worker takes an equal, contiguous share, whatever the lengths are; a worker is a group of
// four softmax warps, and a CTA (one per SM) has NG of them, whose tiles share one ring of shared memory in turn:
//   warp 0       producer: page numbers and scales of the tiles ahead (one page per lane), TMA
//   warp 1       issues S, warp 2 issues O (one thread each)
//   warp 3       q of the units ahead: scaled, split, into shared memory
//   warps 4..    softmax, thread = key; then thread = channel
// The chain of a tile (logits, maximum over the warps, weights, products) takes a group about 3000 cycles, the tile's bytes an SM 1400: with
// one group per CTA and two CTAs per SM the kernel was bound by that chain (247 us where it takes 205 now).  A unit that spans several workers is
// merged by combine_kernel from their partial results.  The code is kept small: at 197 KB it ran from the instruction cache's misses (317 us).
//
// Bound by HBM (2 d bytes per key and kv head), a tile every 1280 cycles and SM once it runs, 8 us after its start.  Measured, d = 128: 64 sequences
// of up to 16384 tokens, 32 heads on 8: 193 to 210 us, 5.2 to 5.7 TB/s (80 to 86 % of the measured copy rate); one of 131072, 8 heads: 57 us, 4.7 TB/s; 64
// with a window of 512, 32 heads: 77 us, 3.4 TB/s (640 keys are read where 516 are seen); one of 1000: 14 us, two launches.
#include <algorithm>
#include <atomic>

#include "kvm_cache.cuh"
#include "tc_common.cuh"

namespace kvm {
namespace cache {

bool encode_tmap_codes(CUtensorMap* map, const void* base, int d, int64_t rows, int page);   // kvm_cache.cu

constexpr int kCtas = 148;
constexpr float kPShift = 8.f;   // the largest weight of a tile is 2^8 (e4m3 ends at 448)

struct alignas(16) TileInfo {
  int b, hk, flags;        // unit; kFirst ...
  int vmax, start, n;      // largest exponent of the visible blocks' value scales; lengths of the sequence
  int ze;                  // last worker that has tiles of the unit
  int pos[8];              // per page of the tile: position of its first key,
  int16_t ke[8], ve[8];    // exponents of its scales
};
// first / last tile of the worker's share of the unit; the share is all of it / begins with it; all columns see all keys of the tile
enum { kFirst = 1, kLast = 2, kWhole = 4, kBegins = 8, kAll = 16 };

template <int D, int NC>
struct DecodeCfg {
  static constexpr int NG = NC == 8 ? 4 : 3;             // groups (16 columns take 128 registers)
  static constexpr int ST = (NC == 8 ? 6 : 5) * (128 / D);   // tiles of the ring
  static constexpr int THREADS = 128 + 128 * NG;
  static constexpr int TILE = 128 * D;                   // codes of a tile of keys or values
  static constexpr int STAGE = 2 * TILE;
  static constexpr int NB = 2 * NC;                      // columns of the products: hi, then lo
  static constexpr int Q_BYTES = NB * 128, P_BYTES = NB * 128;
  static constexpr int OFF_Q = ST * STAGE;               // [group][2] (behind the last value tile: see the descriptor of V for 64 channels)
  static constexpr int OFF_P = OFF_Q + NG * 2 * Q_BYTES; // [group]
  static constexpr int OFF_INFO = OFF_P + NG * P_BYTES;
  static constexpr int OFF_CQ = OFF_INFO + ST * (int)sizeof(TileInfo);   // float [group][4][NC]
  static constexpr int OFF_MAX = OFF_CQ + NG * 4 * NC * 4;               // float4 [group][2][NC]: maxima of the four warps
  static constexpr int OFF_AB = OFF_MAX + NG * 2 * NC * 16;              // float4 [group][2][NC]
  static constexpr int OFF_L = OFF_AB + NG * 2 * NC * 16;                // float [group][4][NC]
  static constexpr int OFF_BAR = OFF_L + NG * 4 * NC * 4;
  static constexpr int OFF_PRE = OFF_BAR + 1024;         // int [batch + 1]
  static constexpr uint32_t TMEM_COLS = NC == 8 ? 256 : 512;
  static constexpr uint32_t GROUP_COLS = 3 * NB;         // two S, then O
  // barriers
  static constexpr int FULL = 0, FREE = FULL + ST, QFULL = FREE + ST, QFREE = QFULL + 4 * NG, SFULL = QFREE + 2 * NG, SFREE = SFULL + 2 * NG,
                       PFULL = SFREE + 2 * NG, ODONE = PFULL + NG, COUNT = ODONE + NG;
  static_assert(COUNT * 8 + 64 <= 1024, "barriers");
  static_assert(OFF_Q % 1024 == 0 && OFF_P % 1024 == 0 && OFF_CQ % 16 == 0 && OFF_MAX % 16 == 0 && OFF_AB % 16 == 0 && OFF_L % 16 == 0 && OFF_BAR % 8 == 0,
                "alignment");
};

// What a worker leaves for combine_kernel beside its partial results: the unit that begins in its share and goes on in the next one's (b < 0: none).
struct Cut { int b, hk, n, ze; };

struct DecodeArgs8 {
  AttendArgs a;
  Cut* cuts;     // [workers]
  int grid;      // CTAs
  int q_vec;
};

// The shares of a CTA's workers: worker g * grid + cta takes tiles [f0[g], f0[g] + n[g]) of the list; n does not grow with g.  The ring takes the
// tiles in the order of their number within the share, group by group.
template <int NG>
struct Shares {
  int f0[NG], n[NG], share;
  __device__ __forceinline__ Shares(int total, int grid, int cta) {
    share = (total + grid * NG - 1) / (grid * NG);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      f0[g] = min(total, (g * grid + cta) * share);
      n[g] = min(share, total - f0[g]);
    }
  }
  __device__ __forceinline__ int active(int i) const {   // workers that have a tile i: the first so many groups
    int a = 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) a += n[g] > i;
    return a;
  }
  __device__ __forceinline__ int tiles() const {
    int a = 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) a += n[g];
    return a;
  }
  // the (i, g) of the ring's tile jj
  __device__ __forceinline__ void at(int jj, int& i, int& g) const {
    int before = 0;
    i = g = 0;
#pragma unroll
    for (int a = NG; a > 0; --a) {   // rounds in which `a` groups are active
      const int rounds = n[a - 1] - (a < NG ? n[a < NG ? a : 0] : 0);
      const int left = jj - before;
      if (left >= 0 && left < rounds * a) { const int r = left / a; i = (a < NG ? n[a < NG ? a : 0] : 0) + r; g = left - r * a; }
      before += rounds * a;
    }
  }
  __device__ __forceinline__ int first(int g) const {   // (f0[g] for a g that is no constant)
    int x = f0[0];
#pragma unroll
    for (int k = 1; k < NG; ++k) x = g == k ? f0[k] : x;
    return x;
  }
  __device__ __forceinline__ int count(int g) const {
    int x = n[0];
#pragma unroll
    for (int k = 1; k < NG; ++k) x = g == k ? n[k] : x;
    return x;
  }
};

__device__ __forceinline__ float redux_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// Barrier of the four warps of a group that also tells whether all of them are well.
__device__ __forceinline__ bool group_barrier(int g, bool ok) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.aligned.pred q, %2, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"(ok ? 1u : 0u), "r"(1 + g) : "memory");
  return r != 0;
}
// Tiles that the call's tokens of a sequence see (0: none, or lengths that are not allowed).
__device__ __forceinline__ int seq_tiles(const AttendArgs& a, int start, int n) {
  return n > 0 ? pages_of(a.p, start, start + n - 1, a.window, a.sinks).tiles : 0;
}
// Last b with pre[b] <= f (pre ascends; f < pre[batch], so that sequence b has tiles).
__device__ __forceinline__ int seq_of(const int* pre, int batch, int f) {
  int lo = 0, hi = batch;   // pre[lo] <= f < pre[hi]
#pragma unroll 1
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= f) lo = mid; else hi = mid;
  }
  return lo;
}

// pre[0 .. batch]: tiles of the sequences before b, all heads; by all NT threads of the block
template <int NT>
__device__ __forceinline__ void list_tiles(const AttendArgs& a, int* pre, int* scratch) {
  const Params& p = a.p;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int per = (p.batch + NT - 1) / NT, b0 = tid * per;
  int sum = 0;
#pragma unroll 1
  for (int b = b0; b < min(b0 + per, p.batch); ++b) {
    int start, n;
    if (!seq_lengths(p, b, start, n)) {
      if (blockIdx.x == 0) report(p.status, KVM_ERR_INVALID_ARG);
      start = n = 0;
    }
    pre[b] = sum;
    sum += seq_tiles(a, start, n) * p.Hkv;
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) scratch[warp] = incl;
  __syncthreads();
  int add = incl - sum;
#pragma unroll 1
  for (int w = 0; w < warp; ++w) add += scratch[w];
#pragma unroll 1
  for (int b = b0; b < min(b0 + per, p.batch); ++b) pre[b] += add;
  if (tid == NT - 1) pre[p.batch] = add + sum;
  __syncthreads();
}

// Sums of v[0 .. N) over the lanes; lane l holds that of column l >> (5 - log2 N) (in all lanes with the same one).
template <int N>
__device__ __forceinline__ float sum_lanes(float (&v)[N], int lane) {
  int bit = 16;
#pragma unroll
  for (int n = N / 2; n >= 1; n >>= 1, bit >>= 1) {
    const bool up = lane & bit;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float give = up ? v[i] : v[n + i], keep = up ? v[n + i] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, bit);
    }
  }
  float s = v[0];
  for (; bit >= 1; bit >>= 1) s += __shfl_xor_sync(0xffffffffu, s, bit);
  return s;
}

template <int D, int NC>
__global__ void __launch_bounds__(DecodeCfg<D, NC>::THREADS, 1)
decode_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const __grid_constant__ DecodeArgs8 args) {
  using Cfg = DecodeCfg<D, NC>;
  constexpr int NB = Cfg::NB, NG = Cfg::NG, ST = Cfg::ST;
  const AttendArgs& a = args.a;
  const Params& p = a.p;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  TileInfo* info = reinterpret_cast<TileInfo*>(base + Cfg::OFF_INFO);
  float* s_cq = reinterpret_cast<float*>(base + Cfg::OFF_CQ);      // factors of the columns' logits, by group and unit & 3
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + Cfg::OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + Cfg::COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* pre = reinterpret_cast<int*>(base + Cfg::OFF_PRE);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (combine_kernel waits for this one before it reads what it wrote)
  if (warp == 0) {
    for (int i = lane; i < Cfg::COUNT; i += 32)   // (one after the other they would take a thousand cycles)
      tc::mbar_init(&bars[i], (i >= Cfg::SFREE && i < Cfg::PFULL) || (i >= Cfg::PFULL && i < Cfg::ODONE) ? 4 : 1);
    if (lane == 0) {
      tc::prefetch_tmap(&mapK); tc::prefetch_tmap(&mapV);
      *abort_flag = 0;
    }
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, Cfg::TMEM_COLS);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  list_tiles<Cfg::THREADS>(a, pre, reinterpret_cast<int*>(base + Cfg::OFF_AB));
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const Shares<NG> sh(pre[p.batch], args.grid, blockIdx.x);
  const int ntile = sh.tiles();
  auto fail = [&]() {
    if (!*abort_flag) report(p.status, KVM_ERR_TIMEOUT);
    *abort_flag = 1;
  };
  auto lengths = [&](int b, int& start, int& n) {   // (of a sequence that has tiles)
    start = p.start[b];
    n = p.count ? p.count[b] : (int)p.T;
  };

  if (warp == 0) {
    // ------------------------------ producer ------------------------------
    const int tshift = 7 - p.page_shift, ppt = 1 << tshift, tpb = 32 >> tshift;   // pages of a tile; tiles whose pages the warp's lanes hold at a time
    const int lt = lane >> tshift, lp = lane & (ppt - 1);
    struct Page { int row, ke, ve, pos, b, hk, flags, start, n, ze; bool all; };   // row < 0: not loaded
    // What there is to know of a batch of tiles is fetched in three steps, a few tiles apart: each waits for what the step before has asked the
    // memory for (together they take several thousand cycles when it is busy, more than the ring covers).
    Page cur{}, nxt{};
    float ks = 0.f, vs = 0.f;   // scales on their way
    auto ask_page = [&](int k) {
      Page& x = nxt;
      x = Page{-1, 0, 0, kNowhere, 0, 0, 0, 0, 0, 0, false};
      const int jj = k * tpb + lt;
      if (jj < ntile) {
        int i, g;
        sh.at(jj, i, g);
        const int F0 = sh.first(g), n = sh.count(g), f = F0 + i;
        const int b = seq_of(pre, p.batch, f);
        lengths(b, x.start, x.n);
        const int last = x.start + x.n - 1;
        const PageList t = pages_of(p, x.start, last, a.window, a.sinks);
        const int rem = f - pre[b], hk = rem / t.tiles, it = rem - hk * t.tiles, u0 = f - it;
        x.b = b; x.hk = hk;
        x.flags = (it == 0 || i == 0 ? kFirst : 0) | (it == t.tiles - 1 || i == n - 1 ? kLast : 0) | (u0 >= F0 ? kBegins : 0) |
                  (u0 >= F0 && u0 + t.tiles <= F0 + n ? kWhole : 0);
        x.ze = (u0 + t.tiles - 1) / sh.share;
        const int at = it * ppt + lp;
        if (at < t.n) {
          const int block = page_at(t, at);
          x.pos = block << p.page_shift;
          x.all = page_seen_by_all(p, x.pos, x.start, last, a.window, a.sinks);
          x.row = p.pages[(int64_t)b * p.max_pages + block];
        }
      }
    };
    auto ask_scales = [&]() {
      if (nxt.pos == kNowhere) return;   // (no page)
      if (nxt.row < 0 || nxt.row >= p.n_pages) {
        report(p.status, KVM_ERR_INVALID_ARG);
        nxt.row = -1;
        ks = vs = __int_as_float(0x7fc00000);
      } else {
        const int unit = nxt.row * p.Hkv + nxt.hk;
        nxt.row = unit * p.page;
        ks = p.ks[unit];
        vs = p.vs[unit];
      }
    };
    auto take = [&]() {
      cur = nxt;
      if (cur.pos == kNowhere) { cur.row = -1; return; }
      cur.ke = scale_exp(ks);
      cur.ve = scale_exp(vs);
    };
    bool ok = true;
    int s = 0, issued = 0;
    uint32_t par = 0;
    int ahead = 0, t = 0;   // batches asked for so far, tiles of the current one that are issued
    for (; issued < ntile; ++issued) {
      const bool none = ahead == 0;
      if (none || t == 1) ask_page(ahead++);
      if (none || t == (tpb > 4 ? 4 : 2)) ask_scales();
      if (none || t == tpb) { take(); t = 0; }
      if (lane == 0) ok = !*abort_flag && (issued < ST || tc::mbar_wait_tight(&bars[Cfg::FREE + s], par ^ 1));
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (!ok) break;
      const bool mine = lt == t;
      const uint32_t loads = __ballot_sync(0xffffffffu, mine && cur.row >= 0);
      const int v = __reduce_max_sync(0xffffffffu, mine && cur.row >= 0 && cur.ve < 128 ? cur.ve : -1000);
      const bool all = __all_sync(0xffffffffu, !mine || cur.all);
      if (mine) {
        TileInfo& ti = info[s];
        ti.pos[lp] = cur.pos;
        ti.ke[lp] = (int16_t)cur.ke;
        ti.ve[lp] = (int16_t)cur.ve;
        if (lp == 0) {
          ti.b = cur.b; ti.hk = cur.hk; ti.flags = cur.flags | (all ? kAll : 0); ti.start = cur.start; ti.n = cur.n; ti.ze = cur.ze;
          ti.vmax = v == -1000 ? 0 : v;
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_expect_tx(&bars[Cfg::FULL + s], __popc(loads) * 2 * p.page * D);
      __syncwarp();
      if (mine && cur.row >= 0) {
        uint8_t* dst = base + s * Cfg::STAGE + lp * p.page * D;
        tc::tma_load_2d(dst, &mapK, &bars[Cfg::FULL + s], 0, cur.row);
        tc::tma_load_2d(dst + Cfg::TILE, &mapV, &bars[Cfg::FULL + s], 0, cur.row);
      }
      if (++s == ST) { s = 0; par ^= 1; }
      ++t;
    }
    if (lane == 0) {
      if (!ok) fail();
      // nothing may be in flight into shared memory when the CTA ends, whatever became of the others
#pragma unroll 1
      for (int j = max(0, issued - ST); j < issued; ++j) tc::mbar_wait_tight(&bars[Cfg::FULL + j % ST], (j / ST) & 1);
    }
  } else if (warp == 1) {
    // ------------------------------ S ------------------------------
    if (lane == 0) {
      constexpr uint32_t ID = tc::idesc_f16(128, NB, false);   // (format 0: e4m3 in kind::f8f6f4)
      auto desc = [](uint32_t addr) { return D == 128 ? tc::smem_desc_sw128(addr, 16, 1024) : tc::smem_desc_sw64(addr, 16, 512); };
      const uint64_t d0 = desc(tc::smem_u32(base));
      bool ok = true;
      auto wait = [&](int bar, uint32_t parity) { ok = ok && tc::mbar_wait_tight(&bars[bar], parity); return ok; };
      uint32_t segs = 0xffffffffu;   // a byte per group: its units so far, less one
      int s = 0;
      uint32_t par = 0;
#pragma unroll 1
      for (int i = 0; i < sh.n[0] && ok; ++i) {
        const int groups = sh.active(i);
#pragma unroll 1
        for (int g = 0; g < groups; ++g) {
          if (i >= 2 && !wait(Cfg::SFREE + 2 * g + (i & 1), ((i >> 1) - 1) & 1)) break;
          if (!wait(Cfg::FULL + s, par)) break;
          const int flags = info[s].flags;
          uint32_t seg = (segs >> (8 * g)) & 255;
          if (flags & kFirst) {
            seg = (seg + 1) & 255;   // (only its last bits matter)
            segs = (segs & ~(255u << (8 * g))) | (seg << (8 * g));
            if (!wait(Cfg::QFULL + 4 * g + (seg & 3), (seg >> 2) & 1)) break;
          }
          tc::tc_fence_after();
          const uint64_t dk = d0 + s * (Cfg::STAGE >> 4), dq = d0 + ((Cfg::OFF_Q + (2 * g + (seg & 1)) * Cfg::Q_BYTES) >> 4);
          const uint32_t dS = tmem + g * Cfg::GROUP_COLS + NB * (i & 1);
#pragma unroll
          for (int ks = 0; ks < D / 32; ++ks) tc::mma_f8_ss(dS, dk + 2 * ks, dq + 2 * ks, ID, ks > 0);
          tc::mma_commit(&bars[Cfg::SFULL + 2 * g + (i & 1)]);
          if (flags & kLast) tc::mma_commit(&bars[Cfg::QFREE + 2 * g + (seg & 1)]);
          if (++s == ST) { s = 0; par ^= 1; }
        }
      }
      if (!ok) fail();
    }
  } else if (warp == 2) {
    // ------------------------------ O ------------------------------
    if (lane == 0) {
      // V8 as it lies: channels contiguous ("MN-major"), groups of 8 keys one swizzle tile apart.  A has 128 rows; with 64 channels rows 64..
      // are read from the next tile (never past OFF_P) and nobody looks at what they give.  The weights of a key are 16 bytes (MN-major, no
      // swizzle): 8 keys make one core matrix of 128 bytes.
      constexpr uint32_t ID = tc::idesc_f16(128, 16, true, true);
      const uint32_t a0 = tc::smem_u32(base);
      const uint64_t dv0 = D == 128 ? tc::smem_desc_sw128(a0 + Cfg::TILE, 1024, 1024) : tc::smem_desc_sw64(a0 + Cfg::TILE, 512, 512);
      const uint64_t dp0 = tc::smem_desc_sw128(a0 + Cfg::OFF_P, 128, 128) & ~((uint64_t)7 << 61);
      bool ok = true;
      int s = 0;
#pragma unroll 1
      for (int i = 0; i < sh.n[0] && ok; ++i) {
        const int groups = sh.active(i);
#pragma unroll 1
        for (int g = 0; g < groups; ++g) {
          if (!(ok = tc::mbar_wait_tight(&bars[Cfg::PFULL + g], i & 1))) break;
          tc::tc_fence_after();
          const uint64_t dv = dv0 + s * (Cfg::STAGE >> 4), dp = dp0 + g * (Cfg::P_BYTES >> 4);
          const uint32_t dO = tmem + g * Cfg::GROUP_COLS + 2 * NB;
#pragma unroll
          for (int c = 0; c < NB / 16; ++c)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) tc::mma_f8_ss(dO + 16 * c, dv + ks * (32 * D >> 4), dp + c * (2048 >> 4) + ks * (512 >> 4), ID, ks > 0);
          tc::mma_commit(&bars[Cfg::ODONE + g]);
          tc::mma_commit(&bars[Cfg::FREE + s]);
          if (++s == ST) s = 0;
        }
      }
      if (!ok) fail();
    }
  } else if (warp == 3) {
    // ------------------------------ q of the units ------------------------------
    // eight threads per column, D / 8 channels each
    constexpr int E = D / 8;
    const int part = lane & 7;
    bool ok = true;
    int seg[NG], next[NG];   // units so far, tile of the share with which the next one begins
#pragma unroll
    for (int g = 0; g < NG; ++g) seg[g] = next[g] = 0;
    while (ok) {
      int g = -1, i = 0x7fffffff;   // the group whose next unit comes first
#pragma unroll
      for (int k = 0; k < NG; ++k)
        if (next[k] < sh.n[k] && next[k] < i) { i = next[k]; g = k; }
      if (g < 0) break;
      const int F0 = sh.first(g), f = F0 + i, b = seq_of(pre, p.batch, f);
      int start, n, sg = 0;
      lengths(b, start, n);
      const int nt = (pre[b + 1] - pre[b]) / p.Hkv, hk = (f - pre[b]) / nt, end = pre[b] + (hk + 1) * nt - F0;
#pragma unroll
      for (int k = 0; k < NG; ++k)
        if (k == g) { sg = seg[k]++; next[k] = end; }
      uint8_t* sQ = base + Cfg::OFF_Q + (2 * g + (sg & 1)) * Cfg::Q_BYTES;
      if (sg >= 2) {
        if (lane == 0) ok = tc::mbar_wait_tight(&bars[Cfg::QFREE + 2 * g + (sg & 1)], ((sg >> 1) - 1) & 1);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
      }
#pragma unroll 1
      for (int c0 = 0; c0 < NC; c0 += 4) {
        const int c = c0 + (lane >> 3);
        float x[E];
        uint32_t top = 0;
        const bool live = c < n * a.G;
        if (live) {
          const int tok = c / a.G, hq = hk * a.G + c - tok * a.G;
          const __nv_bfloat16* src = a.q + b * a.sq[0] + hq * a.sq[1] + tok * a.sq[2] + part * E;
          if (args.q_vec) {
#pragma unroll
            for (int k = 0; k < E / 8; ++k) {
              const uint4 w4 = *reinterpret_cast<const uint4*>(src + 8 * k);
              const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
              for (int q = 0; q < 4; ++q) { x[8 * k + 2 * q] = __uint_as_float(w[q] << 16); x[8 * k + 2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u); }
            }
          } else {
#pragma unroll
            for (int k = 0; k < E; ++k) x[k] = __bfloat162float(src[k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < E; ++k) x[k] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < E; ++k) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool bad = top >= 0x7f800000u;
        const int e = max((int)(top >> 23), 10);          // largest |q| is in [2^(e-127), 2^(e-126))
        const float mul = bad ? 0.f : exp2i(134 - e);     // to [2^7, 2^8)
        uint32_t hi[E / 4], lo[E / 4];
#pragma unroll
        for (int k = 0; k < E / 4; ++k) {
          uint32_t h2[2], l2[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float y0 = bad ? 0.f : x[4 * k + 2 * q] * mul, y1 = bad ? 0.f : x[4 * k + 2 * q + 1] * mul;
            split_e4m3x2(y0, y1, h2[q], l2[q]);
          }
          hi[k] = h2[0] | (h2[1] << 16);
          lo[k] = l2[0] | (l2[1] << 16);
        }
        // swizzled as the TMA does it: 16-byte pieces of a row permuted by the row
        auto at = [&](int row, int byte) -> uint8_t* {
          const int piece = byte >> 4;
          return D == 128 ? sQ + row * 128 + ((piece ^ (row & 7)) << 4) + (byte & 15) : sQ + row * 64 + ((piece ^ ((row >> 1) & 3)) << 4) + (byte & 15);
        };
        if (E == 16) {
          *reinterpret_cast<uint4*>(at(c, part * E)) = make_uint4(hi[0], hi[1], hi[E / 4 - 2], hi[E / 4 - 1]);
          *reinterpret_cast<uint4*>(at(NC + c, part * E)) = make_uint4(lo[0], lo[1], lo[E / 4 - 2], lo[E / 4 - 1]);
        } else {
          *reinterpret_cast<uint2*>(at(c, part * E)) = make_uint2(hi[0], hi[1]);
          *reinterpret_cast<uint2*>(at(NC + c, part * E)) = make_uint2(lo[0], lo[1]);
        }
        if (part == 0) s_cq[(4 * g + (sg & 3)) * NC + c] = bad ? __int_as_float(0x7fc00000) : a.scale_log2 * exp2i(e - 134);
      }
      tc::fence_proxy_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars[Cfg::QFULL + 4 * g + (sg & 3)]);
    }
    if (!ok && lane == 0) fail();
  } else {
    // ------------------------------ softmax; results ------------------------------
    const int g = (warp - 4) >> 2, w4 = warp & 3, tok = w4 * 32 + lane;
    const int n_mine = sh.count(g), worker = g * args.grid + blockIdx.x;
    const uint32_t lanes = tmem + ((uint32_t)(w4 * 32) << 16) + g * Cfg::GROUP_COLS;
    const float* cq = s_cq + g * 4 * NC;
    float4* s_max = reinterpret_cast<float4*>(base + Cfg::OFF_MAX) + g * 2 * NC;
    float4* s_ab = reinterpret_cast<float4*>(base + Cfg::OFF_AB) + g * 2 * NC;
    float* s_l = reinterpret_cast<float*>(base + Cfg::OFF_L) + g * 4 * NC;
    uint8_t* sP = base + Cfg::OFF_P + g * Cfg::P_BYTES + tok * 16;
    float o_run[NC], l_run[NC], l_new[NC];
    float m_run = -INFINITY, m_old = -INFINITY;   // (threads below NC: running reference of column tok)
    int seg = -1;
    int pb = 0, phk = 0, pflags = 0, pn = 0, pze = 0;   // the tile before
    bool ok = true;
    auto columns = [&](uint32_t at, float (&y)[NC]) {   // hi + lo
      if (NC == 8) {
        uint32_t r[16];
        tc::tmem_ld16(at, r);
        tc::tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < NC; ++c) y[c] = __uint_as_float(r[c % 8]) + __uint_as_float(r[8 + c % 8]);
      } else {
        uint32_t r[32];
        tc::tmem_ld32(at, r);
        tc::tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < NC; ++c) y[c] = __uint_as_float(r[c]) + __uint_as_float(r[16 + c % 16]);
      }
    };
    // adds the products of tile i to the running results, and stores those of a share that ends with it
    auto gather = [&](int i) {
      if (!tc::mbar_wait_tight(&bars[Cfg::ODONE + g], i & 1)) ok = false;
      __syncwarp();
      tc::tc_fence_after();
      float o[NC];
      columns(lanes + 2 * NB, o);
      const bool first = pflags & kFirst;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float4 f = s_ab[(i & 1) * NC + c];   // factors of what there is, of the row sum, of the products
        o_run[c] = first ? o[c] * f.z : fmaf(o_run[c], f.x, o[c] * f.z);
        l_run[c] = first ? l_new[c] * f.y : fmaf(l_run[c], f.x, l_new[c] * f.y);
      }
      if (!(pflags & kLast)) return;
      const int ncol = pn * a.G;
      const float lw = sum_lanes<NC>(l_run, lane);
      if ((lane & (32 / NC - 1)) == 0) s_l[(lane / (32 / NC)) * 4 + w4] = lw;
      group_barrier(g, true);
      if (pflags & kWhole) {
        // (each thread's channel of the columns through its own bytes of the weights, which nothing reads now: the loop over the columns
        // stays small)
        uint32_t h[NC / 2];
#pragma unroll
        for (int c = 0; c < NC; c += 2) {
          float x[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float4 l4 = *reinterpret_cast<const float4*>(s_l + 4 * (c + k));
            x[k] = __fdividef(o_run[c + k], (l4.x + l4.y) + (l4.z + l4.w)) * exp2i(kUnitExp);
          }
          const __nv_bfloat162 b2 = __floats2bfloat162_rn(x[0], x[1]);
          h[c / 2] = *reinterpret_cast<const uint32_t*>(&b2);
        }
        *reinterpret_cast<uint4*>(sP) = make_uint4(h[0], h[1], h[2], h[3]);
        if (NC == 16) *reinterpret_cast<uint4*>(sP + 2048) = make_uint4(h[NC / 2 - 4], h[NC / 2 - 3], h[NC / 2 - 2], h[NC / 2 - 1]);
        __nv_bfloat16* o = a.out + pb * a.so[0] + (int64_t)phk * a.G * a.so[1] + tok;
        int hg = 0;
#pragma unroll 1
        for (int c = 0; c < ncol; ++c) {
          if (tok < D) *o = *reinterpret_cast<const __nv_bfloat16*>(sP + (c >> 3) * 2048 + (c & 7) * 2);
          o += a.so[1];
          if (++hg == a.G) { hg = 0; o += a.so[2] - a.G * a.so[1]; }
        }
      } else {
        float* part = a.part + (int64_t)(2 * worker + (pflags & kBegins ? 1 : 0)) * NC * (D + 2);
#pragma unroll
        for (int c = 0; c < NC; ++c) {   // (columns that are not in use give something that nobody reads)
          if (tok < D) part[c * (D + 2) + tok] = o_run[c];
          if (tok == c) {
            const float4 l4 = *reinterpret_cast<const float4*>(s_l + 4 * c);
            part[c * (D + 2) + D] = (i == n_mine - 1) ? m_run : m_old;
            part[c * (D + 2) + D + 1] = (l4.x + l4.y) + (l4.z + l4.w);
          }
        }
      }
      group_barrier(g, true);   // (s_l is free again)
    };
    int s = g % ST;        // the ring's tile, and the parity of its phase
    uint32_t par = (g / ST) & 1;
#pragma unroll 1
    for (int i = 0; i <= n_mine && n_mine > 0; ++i) {   // (the last time round only the products of the tile before are left)
      float y[NC];
      int flags = 0, b = 0, hk = 0, vmax = 0, n = 0, ze = 0, vr = 0;
      bool dropped = false;
      if (i < n_mine) {
        if (!tc::mbar_wait_tight(&bars[Cfg::SFULL + 2 * g + (i & 1)], (i >> 1) & 1)) ok = false;
        // (complete already: what the producer wrote about the tile and, below, the factors of the columns are acquired here)
        if (!tc::mbar_wait_tight(&bars[Cfg::FULL + s], par)) ok = false;
        __syncwarp();
        tc::tc_fence_after();
        columns(lanes + NB * (i & 1), y);
        const TileInfo& ti = info[s];
        const int start = ti.start;
        flags = ti.flags; b = ti.b; hk = ti.hk; vmax = ti.vmax; n = ti.n; ze = ti.ze;
        const int ke = ti.ke[tok >> p.page_shift], ve = ti.ve[tok >> p.page_shift];
        if (flags & kFirst) {
          // (four slots: the factors of unit seg + 4 are written after the products of seg + 2, hence after this thread's use of seg's)
          ++seg;
          if (!tc::mbar_wait_tight(&bars[Cfg::QFULL + 4 * g + (seg & 3)], (seg >> 2) & 1)) ok = false;
        }
        const int last = start + n - 1, key = ti.pos[tok >> p.page_shift] + (tok & (p.page - 1));
        const float ks = exp2i(ke);
        vr = ve > 127 ? 0 : max(ve - vmax, -kFoldMost);   // exponent that the weights take over from the values' scale
        const float vrel = ve > 127 ? __int_as_float(0x7fc00000) : (float)vr;
        dropped = ve < 128 && ve - vmax < -kFoldMost;
        const bool any = key <= last && (key > start - a.window || key < a.sinks);   // some column sees the key
#pragma unroll
        for (int c4 = 0; c4 < NC / 4; ++c4) {
          const float4 f = reinterpret_cast<const float4*>(cq + (seg & 3) * NC)[c4];
          y[4 * c4] = fmaf(y[4 * c4] * f.x, ks, vrel); y[4 * c4 + 1] = fmaf(y[4 * c4 + 1] * f.y, ks, vrel);
          y[4 * c4 + 2] = fmaf(y[4 * c4 + 2] * f.z, ks, vrel); y[4 * c4 + 3] = fmaf(y[4 * c4 + 3] * f.w, ks, vrel);
        }
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars[Cfg::SFREE + 2 * g + (i & 1)]);
        if (!(flags & kAll)) {
          if (n == 1) {
#pragma unroll
            for (int c = 0; c < NC; ++c) y[c] = any ? y[c] : -INFINITY;
          } else {
            int t = 0, gg = 0;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              if (!sees(start + t, key, a.window, a.sinks)) y[c] = -INFINITY;
              if (++gg == a.G) { gg = 0; ++t; }
            }
          }
          // whatever the ring or the page holds there must not meet the weight 0 (a block with a NaN scale may be one that was not loaded, and
          // that some columns do not see)
          if (!any || ve > 127) {
            uint4* row = reinterpret_cast<uint4*>(base + s * Cfg::STAGE + Cfg::TILE + tok * D);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) row[(k + lane) % (D / 16)] = make_uint4(0, 0, 0, 0);   // (in an order that spreads over the banks)
          }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float m = redux_max(y[c]);
          if (lane == c) reinterpret_cast<float*>(&s_max[(i & 1) * NC + c])[w4] = m;
        }
      }
      ok = group_barrier(g, ok && !*abort_flag);
      if (!ok) break;
      if (tok < NC && i < n_mine) {
        const float4 x = s_max[(i & 1) * NC + tok];
        const float m = fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w));
        m_old = m_run;
        const float from = (flags & kFirst) ? -INFINITY : m_run;
        m_run = fmaxf(from, m);
        const float alpha = from == -INFINITY ? 0.f : tc::ex2_approx(from - m_run);
        const float beta = m == -INFINITY ? 0.f : tc::ex2_approx(m - m_run);
        s_ab[(i & 1) * NC + tok] = make_float4(alpha, beta, beta * exp2i(vmax - kUnitExp), 0.f);
      }
      if (i > 0) gather(i - 1);   // (whose factors all warps have seen written)
      if (i == n_mine) break;
      // weights: 2^(y - m + 8), in two parts
      const float back = exp2i(-vr);   // (NaN weights stay NaN in either form)
      uint32_t hi[NC / 4], lo[NC / 4];
#pragma unroll
      for (int c = 0; c < NC; c += 2) {
        float w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float4 x = s_max[(i & 1) * NC + c + k];
          const float m = fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w));
          w[k] = tc::ex2_approx(y[c + k] - (m == -INFINITY ? 0.f : m - kPShift));
        }
        const uint32_t hb = to_e4m3x2(w[0], w[1]);
        const float2 h = e4m3x2_to_float2(hb);
        const uint32_t lb = to_e4m3x2(w[0] - h.x, w[1] - h.y);
        const float2 l = e4m3x2_to_float2(lb);
        // The row sum takes the weights as the products get them, so that their rounding does not shift a flat row; but where the
        // values' scale has been taken over, a weight can be too small for e4m3 and still count in the sum.
        l_new[c] = vr == 0 ? h.x + l.x : w[0] * back;
        l_new[c + 1] = vr == 0 ? h.y + l.y : w[1] * back;
        if (c % 4 == 0) { hi[c / 4] = hb; lo[c / 4] = lb; } else { hi[c / 4] |= hb << 16; lo[c / 4] |= lb << 16; }
      }
      if (dropped) {
#pragma unroll
        for (int k = 0; k < NC / 4; ++k) hi[k] = lo[k] = 0;
      }
      if (NC == 8) {
        *reinterpret_cast<uint4*>(sP) = make_uint4(hi[0], hi[1], lo[0], lo[1]);
      } else {
        *reinterpret_cast<uint4*>(sP) = make_uint4(hi[0], hi[1], hi[NC / 4 - 2], hi[NC / 4 - 1]);
        *reinterpret_cast<uint4*>(sP + 2048) = make_uint4(lo[0], lo[1], lo[NC / 4 - 2], lo[NC / 4 - 1]);
      }
      tc::fence_proxy_async();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars[Cfg::PFULL + g]);
      pb = b; phk = hk; pflags = flags; pn = n; pze = ze;
      s += sh.active(i);
      if (s >= ST) { s -= ST; par ^= 1; }
    }
    if (tok == 0) args.cuts[worker] = Cut{ok && (pflags & (kBegins | kWhole)) == kBegins ? pb : -1, phk, pn, pze};
    if (!ok) fail();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, Cfg::TMEM_COLS);
  }
}

// Units that several workers shared: out = sum_z 2^(m_z - m) O_z / sum_z 2^(m_z - m) l_z.  Block (w, c): column c of the unit that begins in worker
// w's share and goes on behind it, if there is one.  Threads: D channels, 256 / D parts of the list of workers, eight of them in flight.
template <int D, int NC>
__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ DecodeArgs8 args) {
  constexpr int ZP = 256 / D;
  const AttendArgs& a = args.a;
  __shared__ float s_o[ZP][D], s_ml[ZP][2];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Cut cut = args.cuts[blockIdx.x];
  const int c = blockIdx.y, z0 = blockIdx.x;
  if (cut.b < 0 || c >= cut.n * a.G) return;
  const int ch = threadIdx.x % D, zp = threadIdx.x / D;
  // the first worker's share begins with the unit (slot 1), those of the others in its middle (slot 0)
  const float* first = a.part + (int64_t)z0 * 2 * NC * (D + 2) + c * (D + 2);
  float m = -INFINITY, o = 0.f, l = 0.f;
  for (int z = zp; z <= cut.ze - z0; z += 8 * ZP) {
    float mz[8], lz[8], oz[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int zk = z + k * ZP;
      mz[k] = -INFINITY; lz[k] = oz[k] = 0.f;
      if (zk <= cut.ze - z0) {
        const float* r = first + (int64_t)zk * 2 * NC * (D + 2) + (zk == 0 ? NC * (D + 2) : 0);
        mz[k] = r[D]; lz[k] = r[D + 1]; oz[k] = r[ch];
      }
    }
    float mn = m;
#pragma unroll
    for (int k = 0; k < 8; ++k) mn = fmaxf(mn, mz[k]);
    const float f = m == -INFINITY ? 0.f : tc::ex2_approx(m - mn);
    o *= f;
    l *= f;
    m = mn;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float w = mz[k] == -INFINITY ? 0.f : tc::ex2_approx(mz[k] - m);
      o = fmaf(oz[k], w, o);
      l = fmaf(lz[k], w, l);
    }
  }
  s_o[zp][ch] = o;
  if (ch == 0) { s_ml[zp][0] = m; s_ml[zp][1] = l; }
  __syncthreads();
  if (zp > 0) return;
  float mm = s_ml[0][0];
#pragma unroll
  for (int z = 1; z < ZP; ++z) mm = fmaxf(mm, s_ml[z][0]);
  o = l = 0.f;
#pragma unroll
  for (int z = 0; z < ZP; ++z) {
    const float w = s_ml[z][0] == -INFINITY ? 0.f : tc::ex2_approx(s_ml[z][0] - mm);
    o = fmaf(s_o[z][ch], w, o);
    l = fmaf(s_ml[z][1], w, l);
  }
  const int t = c / a.G, hq = cut.hk * a.G + c - t * a.G;
  a.out[cut.b * a.so[0] + hq * a.so[1] + t * a.so[2] + ch] = __float2bfloat16_rn(o / l * exp2i(kUnitExp));
}

// At most so many CTAs have tiles: `units` units of at most `tiles` tiles each.
static int decode_grid(int64_t units, int64_t tiles) { return (int)std::min<int64_t>(kCtas, units * tiles); }

static int64_t decode_partials(int workers, int d, int cols) { return (int64_t)workers * 2 * (cols <= 8 ? 8 : 16) * (d + 2) * 4; }   // bytes

int64_t decode_workspace(int64_t units, int64_t tiles, int d, int cols) {
  const int workers = decode_grid(units, tiles) * (cols <= 8 ? 4 : 3);
  return decode_partials(workers, d, cols) + workers * (int64_t)sizeof(Cut);
}

template <int D, int NC>
static kvm_status_t launch_decode_nc(const DecodeArgs8& args, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t s) {
  using Cfg = DecodeCfg<D, NC>;
  static_assert(Cfg::OFF_PRE + (kMaxBatch + 1) * 4 + 1024 <= 227 * 1024, "shared memory");
  const int smem = Cfg::OFF_PRE + (args.a.p.batch + 1) * 4 + 1024;
  static std::atomic<uint64_t> ready{0};   // devices on which the limit has been raised
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  if (dev > 63 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
    constexpr int most = Cfg::OFF_PRE + (kMaxBatch + 1) * 4 + 1024;
    if (cudaFuncSetAttribute(decode_kernel<D, NC>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  decode_kernel<D, NC><<<args.grid, Cfg::THREADS, smem, s>>>(mapK, mapV, args);
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(args.grid * Cfg::NG, (unsigned)(args.a.p.T * args.a.G)); lc.blockDim = dim3(256); lc.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at; lc.numAttrs = 1;
  if (cudaLaunchKernelEx(&lc, combine_kernel<D, NC>, args) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}

kvm_status_t launch_decode8(const AttendArgs& a, int64_t tiles, bool q_vec, cudaStream_t s) {
  DecodeArgs8 args;
  args.a = a;
  args.grid = decode_grid((int64_t)a.p.batch * a.p.Hkv, tiles);
  const int cols = (int)(a.p.T * a.G);
  args.cuts = reinterpret_cast<Cut*>(reinterpret_cast<uint8_t*>(a.part) + decode_partials(args.grid * (cols <= 8 ? 4 : 3), a.d, cols));
  args.q_vec = q_vec ? 1 : 0;
  CUtensorMap mapK, mapV;
  const int64_t rows = a.p.n_pages * a.p.Hkv * a.p.page;
  if (!encode_tmap_codes(&mapK, a.p.k, a.d, rows, a.p.page) || !encode_tmap_codes(&mapV, a.p.v, a.d, rows, a.p.page)) return KVM_ERR_CUDA;
  const bool few = cols <= 8;
  if (a.d == 128) return few ? launch_decode_nc<128, 8>(args, mapK, mapV, s) : launch_decode_nc<128, 16>(args, mapK, mapV, s);
  return few ? launch_decode_nc<64, 8>(args, mapK, mapV, s) : launch_decode_nc<64, 16>(args, mapK, mapV, s);
}

}  // namespace cache
}  // namespace kvm
