// Attention of many tokens per sequence (prompts, pieces of prompts) over the 8-bit cache.
//
// The rows of a (sequence, kv head) unit are its query rows, row = token * G + head of the group, so that the heads of a group share the
// key tiles.  One CTA owns 128 rows and walks the key tiles that they see: those of the first `sinks` tokens, then the window's.
//     S = (q_hi + q_lo) K8^T   kind::f8f6f4: the codes as they lie in memory, q in two parts of e4m3 (see kvm_cache_decode.cu; exact for bf16)
//     O += P V16               kind::f16: P in fp16 from tensor memory, V16 = the codes of the values in fp16 (exact)
// Two products with e4m3 operands take the tensor core as long as one with 16-bit operands, so the keys need no conversion; the weights would
// need their two parts for every element, on the warps that already bound the kernel, so for P V it is the codes that are converted, once
// per tile, by warps of their own.
// Scales: that of a block of keys multiplies the logits of its columns, 16 columns (the smallest page) at a time.  That of a block of values is a
// power of two relative to the largest of the CTA's visible blocks, 2^vbase: it goes into the fp16 values (exact to 2^-24) unless some visible
// block lies more than kNarrow powers below.  Then a row that does not see the largest block could lose what it sees, so the scales are
// added to the exponents of the weights instead and taken out of the row sum again (625 -> 692 us where every CTA does that, two prompts of
// 8192 tokens and 16 heads).
//   warp 0       producer of keys: page numbers and scales ahead, TMA into a ring of three tiles; warp 3 the same for values, four tiles
//   warp 1       issues S into three accumulators, warp 2 issues P V (one thread each)
//   warps 4-19   softmax: tile j belongs to the eight warps of group j % 2, two threads per row, 64 columns each; S is read from tensor memory
//                twice, 32 columns at a time (maximum, then weights), and P goes over columns that have been read.  A scheduler of the SM
//                thus holds two pairs of warps that work on two different tiles of the same rows, one in its maxima while another is in its
//                exponentials; all they hand on from tile to tile is the reference of each row (with which O is scaled), decided after
//                the maximum.
//   warps 20-23  value codes -> fp16, swizzled as the MMA reads them
// A CTA that is done may go on with a block of the grid that has not begun (MORE): the warp that produces keys asks the hardware for it when it has
// three tiles left to load, works out what there is to do and tells the others, whose rings and barriers go on; keys, values and the search for
// vbase are then under way while the last tiles are still in their softmax.
// With few rows the key tiles are dealt over several CTAs (splits), whose partial results prompt_combine_kernel merges.
//
// Bound by the softmax warps and the conversion: 1600 instructions per scheduler and tile (128 x 128) against 1024 cycles of the tensor core, 2300
// cycles a tile; and by the set-up, filling and emptying per block of 128 rows (8 us, 7 where a CTA goes on), most of what short windows
// cost.  Measured: two prompts of 8192 tokens, 16 heads, d = 128: 673 to 698 us in long runs, under the power cap, 790 to 820 TFLOP/s (58 to 60 % of the
// measured sustained rate, 49 % of the burst rate), 625 us in a short one; three of 3994, 7032 and 5154, 16 heads on 4, d = 64, window 512: 164 us;
// 300 tokens behind 3000, 32 heads on 8: 42 us.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "kvm_cache.cuh"
#include "out_stage.cuh"
#include "tc_common.cuh"

namespace kvm {
namespace cache {

bool encode_tmap_codes(CUtensorMap* map, const void* base, int d, int64_t rows, int page);   // kvm_cache.cu

constexpr int kSplitTiles = 4;    // least key tiles of a split
constexpr int kMaxSplits = 32;

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
struct PromptArgs {
  AttendArgs a;
  FastDiv by_units, by_heads, by_group;
  int units, qtiles, nsplit;
  int q_vec, out_vec;
};

struct alignas(16) PromptTile {
  int flags;          // 1: some scale is NaN, or some row does not see some key
  int pos[8];         // per 16 columns: position of the first key,
  float ks[8], ve[8]; // scale of the keys, exponent of the values' scale
};
struct alignas(16) ValueTile {
  int all;            // every key is there and is seen by some row
  int pos[8];         // per page: position of the first key (kNowhere: not loaded),
  uint32_t vs[8];     // scale of the values for their fp16 form, two fp16 each
};
constexpr int kInfo = 8;   // ring of tile descriptions: that of tile j + 8 is written when S of tile j + 5 is done, hence P V of tile j + 2
constexpr int kRows = 128; // rows of a CTA
constexpr int kNarrow = 14;
// Weights are held in units of 2^-kShift of what the row's reference stands for: at most 2^(8 + kShift) (fp16 ends at 2^16), and exact or rounded
// to 2^-(24 + kShift) below.  A weight that comes to nothing there still counts in the row sum, so n such keys shift a row by up to
// n 2^-(25 + kShift): with 6, 2^-11 for a million of them (without it, 2^-5: the tail of a million keys 2^-26 below the first one was lost).
constexpr float kShift = 6.f;
constexpr int kThreads = 768;
constexpr int kValueInfo = 4;   // (as many as value tiles: written when the tile is free)

// PB_READY: P of the tile is in tensor memory (8 softmax warps) and its values are in fp16 (4 converting warps); PB_REF: the references of
// 32 rows are decided for a tile, [row quarter][tile % 3]
enum { PB_KFULL = 0, PB_KFREE = 3, PB_V8FULL = 6, PB_V8FREE = 10, PB_VFREE = 14, PB_SFULL = 16, PB_READY = 19, PB_PVDONE = 22, PB_QFULL = 25,
       PB_REF = 26, PB_LAST = 38, PB_VBASE = 39, PB_WORK = 41, PB_NEXT = 49, PB_COUNT = 50 };
// Blocks that are known: the producer of keys is at most five ahead of the slowest warp (three tiles of a block each, the next, the one to come).
constexpr int kWorks = 8;

template <int D>
struct PromptCfg {
  static constexpr int NK = 3, NV8 = 4, NV = 2, NACC = 3;
  static constexpr int T8 = 128 * D, T16 = 256 * D;
  static constexpr int OFF_Q = 0;                        // hi, lo
  static constexpr int OFF_K = OFF_Q + 2 * T8;
  static constexpr int OFF_V8 = OFF_K + NK * T8;
  static constexpr int OFF_V = OFF_V8 + NV8 * T8;
  static constexpr int OFF_INFO = OFF_V + NV * T16;
  static constexpr int OFF_VINFO = OFF_INFO + kInfo * (int)sizeof(PromptTile);
  static constexpr int OFF_M = OFF_VINFO + kValueInfo * (int)sizeof(ValueTile);    // float [128]: references of the rows
  static constexpr int OFF_XM = OFF_M + 128 * 4;                              // float [2 groups][2][2 halves][128]: maxima
  static constexpr int OFF_L = OFF_XM + 8 * 128 * 4;                          // float [4][128]: sums of the row's four threads, [4][128]: NaN marks
  static constexpr int OFF_CQ = OFF_L + 8 * 128 * 4;                          // float [128]
  static constexpr int OFF_BAR = OFF_CQ + 128 * 4;
  static constexpr int OFF_NEXT = OFF_BAR + 512;                              // what the hardware answers
  static constexpr int OFF_WORKS = OFF_NEXT + 16;
  static constexpr int END = OFF_WORKS + kWorks * 64;
  // never less than half an SM, so that one CTA with its 512 columns of tensor memory is resident
  static constexpr int SMEM = (END + 1024) > 120 * 1024 ? (END + 1024) : 120 * 1024;
  static constexpr uint32_t COL_S = 0, COL_O = 384;      // S / P accumulator i at 128 i
  static_assert(OFF_K % 1024 == 0 && OFF_V8 % 1024 == 0 && OFF_V % 1024 == 0 && OFF_M % 16 == 0 && OFF_XM % 16 == 0 && OFF_L % 16 == 0 && OFF_BAR % 8 == 0,
                "alignment");
  static_assert(OFF_NEXT % 16 == 0, "alignment");
  static_assert(PB_COUNT * 8 + 80 <= 512 && SMEM <= 227 * 1024, "shared memory");
};
// What a CTA does: its rows and its key tiles.  (Also what the merge needs to know.)
struct alignas(16) PromptWork {
  int b, hk, start, row0, rows, first, last, jb, ntiles, parts;
  PageList t;
};
__device__ __forceinline__ bool prompt_work(const PromptArgs& args, int idx, int sp, PromptWork& w) {
  const Params& p = args.a.p;
  const int turn = args.by_units.div(idx), unit = idx - turn * args.units, qt = args.qtiles - 1 - turn;   // (the last rows see the most keys: first)
  w.b = args.by_heads.div(unit); w.hk = unit - w.b * p.Hkv;
  int n;
  if (!seq_lengths(p, w.b, w.start, n)) {
    if (idx == unit && w.hk == 0 && sp == 0 && threadIdx.x == 0) report(p.status, KVM_ERR_INVALID_ARG);
    return false;
  }
  w.row0 = qt * kRows;
  const int64_t left = (int64_t)n * args.a.G - w.row0;
  if (left <= 0) return false;
  w.rows = (int)min((int64_t)kRows, left);
  w.first = w.start + args.by_group.div(w.row0);
  w.last = w.start + args.by_group.div(w.row0 + w.rows - 1);
  w.t = pages_of(p, w.first, w.last, args.a.window, args.a.sinks);
  w.parts = 1;
  w.jb = 0;
  w.ntiles = w.t.tiles;
  if (args.nsplit > 1) {
    const int per = max(kSplitTiles, (w.t.tiles + args.nsplit - 1) / args.nsplit);
    w.parts = (w.t.tiles + per - 1) / per;
    w.jb = sp * per;
    w.ntiles = min(per, w.t.tiles - w.jb);
  }
  return w.ntiles > 0;
}
static_assert(sizeof(PromptWork) == 64, "shared memory");
// Asks the hardware for a block of the grid that has not begun, to be done by this CTA (the answer's 16 bytes arrive on the barrier).
__device__ __forceinline__ void ask_next(void* answer, uint64_t* bar) {
  tc::mbar_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(tc::smem_u32(answer)),
               "r"(tc::smem_u32(bar)) : "memory");
}
// The x of that block; -1: all have begun (and nothing may be asked any more).
__device__ __forceinline__ int next_block(const void* answer) {
  uint32_t there, x;
  asm volatile(
      "{\n\t.reg .b128 h;\n\t.reg .pred p;\n\t"
      "mov.u32 %1, 0;\n\t"
      "ld.shared.b128 h, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, h;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(there), "=&r"(x) : "r"(tc::smem_u32(answer)) : "memory");
  return there ? (int)x : -1;
}
// Barrier of the two warps of a group that share 32 rows, which also tells whether both are well.
__device__ __forceinline__ bool pair_barrier(int id, bool ok) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.aligned.pred q, %2, 64, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"(ok ? 1u : 0u), "r"(id) : "memory");
  return r != 0;
}
__device__ __forceinline__ void copy16_async(void* smem, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(smem)), "l"(global) : "memory");
}
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
template <int D, bool MORE>
__global__ void __launch_bounds__(kThreads, 1)
prompt_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const __grid_constant__ PromptArgs args) {
  using Cfg = PromptCfg<D>;
  const AttendArgs& a = args.a;
  const Params& p = a.p;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  PromptTile* info = reinterpret_cast<PromptTile*>(base + Cfg::OFF_INFO);
  ValueTile* vinfo = reinterpret_cast<ValueTile*>(base + Cfg::OFF_VINFO);
  float* s_m = reinterpret_cast<float*>(base + Cfg::OFF_M);
  float* xm = reinterpret_cast<float*>(base + Cfg::OFF_XM);
  float* s_l = reinterpret_cast<float*>(base + Cfg::OFF_L);
  float* s_cq = reinterpret_cast<float*>(base + Cfg::OFF_CQ);
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + Cfg::OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + PB_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_vmax = reinterpret_cast<int*>(tmem_slot + 2);   // [work & 1]: [4] largest, [4] smallest
  PromptWork* works = reinterpret_cast<PromptWork*>(base + Cfg::OFF_WORKS);   // the CTA's blocks, a ring; ntiles 0: there are no more
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the merge waits for this kernel before it reads what it wrote)
  PromptWork first;
  if (!prompt_work(args, blockIdx.x, blockIdx.y, first)) return;
  if (MORE && tid == 0) works[0] = first;
  auto work = [&](int item) -> const PromptWork& { return MORE ? works[item % kWorks] : first; };

  // Set-up: the barriers, tensor memory, and no other barrier of the whole CTA: the producers, the queries' conversion and the search for vbase
  // (each a chain of loads) run side by side from here on.
  if (warp == 0) {
    for (int i = lane; i < PB_COUNT; i += 32) {   // (one after the other they would take a thousand cycles)
      auto in = [&](int first, int n) { return i >= first && i < first + n; };
      tc::mbar_init(&bars[i], in(PB_READY, 3) ? 8 + 4 : in(PB_V8FREE, Cfg::NV8) || in(PB_VBASE, 2) ? 4 : in(PB_REF, 12) ? 2 : in(PB_QFULL, 1) ? 16 : 1);
    }
    if (lane == 0) {
      tc::prefetch_tmap(&mapK); tc::prefetch_tmap(&mapV);
      *abort_flag = 0;
    }
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
  }
  // Page i of the CTA's tiles (ppt pages a tile): whether some row sees some key of it, and where it is.
  const int tshift = 7 - p.page_shift, ppt = 1 << tshift;
  auto page_of = [&](const PromptWork& w, int i, int& p0) -> int {   // >= 0: page; -1: there is none; -2: outside the pool
    i += w.jb * ppt;
    p0 = kNowhere;
    if (i >= w.t.n) return -1;
    const int block = page_at(w.t, i);
    p0 = block << p.page_shift;
    const int page = p.pages[(int64_t)w.b * p.max_pages + block];
    return page >= 0 && page < p.n_pages ? page : -2;
  };
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // largest exponent of the visible blocks' value scales, and whether some lie too far below, found by the converting warps (complete
  // behind PB_VBASE)
  auto vbase_found = [&](int item, bool& wide) {
    const int* x = s_vmax + 8 * (item & 1);
    const int v = max(max(x[0], x[1]), max(x[2], x[3]));
    wide = v - min(min(x[4], x[5]), min(x[6], x[7])) > kNarrow;
    return v == -1000 ? 0 : v;
  };

  // Waits for what there is to do as number `item`; false: nothing (or the wait ran out: ok is cleared).
  auto work_there = [&](int item, bool& ok) {   // (by one thread)
    if (!MORE) return item == 0;
    if (ok && item > 0 && !tc::mbar_wait_tight(&bars[PB_WORK + item % kWorks], ((item - 1) / kWorks) & 1)) ok = false;
    return ok && works[item % kWorks].ntiles > 0;
  };
  auto work_there_warp = [&](int item, bool& ok) {   // (by a warp)
    if (!MORE) return item == 0;
    const bool there = work_there(item, ok);
    ok = __all_sync(0xffffffffu, ok);
    return ok && there;
  };
  auto fail = [&]() {
    if (!*abort_flag) report(p.status, KVM_ERR_TIMEOUT);
    *abort_flag = 1;
  };
  if (warp < 4) {
    if (warp == 0 || warp == 3) {
      // ------------------------------ producers of keys (warp 0) and values (warp 3) ------------------------------
      const bool keys = warp == 0;
      const int ring = keys ? Cfg::NK : Cfg::NV8, full = keys ? PB_KFULL : PB_V8FULL, empty = keys ? PB_KFREE : PB_V8FREE;
      const CUtensorMap* map = keys ? &mapK : &mapV;
      uint8_t* tiles = base + (keys ? Cfg::OFF_K : Cfg::OFF_V8);
      const int tpb = 32 >> tshift, lt = lane >> tshift, lp = lane & (ppt - 1);   // tiles whose pages the warp's lanes hold at a time
      struct Page { int row, ke, ve, pos; };   // row < 0: not loaded
      bool ok = true;
      int s = 0, issued = 0, asked = 0;
      uint32_t par = 0;
#pragma unroll 1
      for (int item = 0; work_there_warp(item, ok); ++item) {
        bool asking = false;
        const PromptWork w = work(item);
        auto fetch = [&](int k) {
          Page g{-1, 0, 0, 0};
          const int j = k * tpb + lt;
          if (j < w.ntiles) {
            int p0;
            const int page = page_of(w, j * ppt + lp, p0);
            g.pos = p0;
            if (page == -2) {
              report(p.status, KVM_ERR_INVALID_ARG);
              g.ke = g.ve = 128;
            } else if (page >= 0) {
              const int unit = page * p.Hkv + w.hk;
              g.row = unit * p.page;
              g.ke = scale_exp(p.ks[unit]);
              g.ve = scale_exp(p.vs[unit]);
            }
          }
          return g;
        };
        int vbase = 0;
        bool wide = false;
        if (!keys) {
          tc::mbar_wait_tight(&bars[PB_VBASE + (item & 1)], (item >> 1) & 1);   // (should it run out, so do the waits for what comes after)
          vbase = vbase_found(item, wide);
        }
        Page cur{}, nxt{};
        for (int j = 0, ahead = 0, t = tpb; j < w.ntiles; ++j) {   // (ahead: batches of pages fetched; t: tiles of the current one that are issued)
          if (t == tpb) {
            t = 0;
#pragma unroll 1
            do { cur = nxt; nxt = fetch(ahead++); } while (ahead < 2);   // (one batch is always on its way)
          }
          // (late, so that a CTA does not hold what another could begin; early enough for the answer to be there when it is needed)
          if (MORE && keys && j == max(0, w.ntiles - 3)) {
            if (lane == 0) ask_next(base + Cfg::OFF_NEXT, &bars[PB_NEXT]);
            asking = true;
          }
          if (lane == 0) ok = issued < ring || tc::mbar_wait_tight(&bars[empty + s], par ^ 1);
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) break;
          const bool mine = lt == t, nan = cur.ke > 127 || cur.ve > 127;
          const uint32_t loads = __ballot_sync(0xffffffffu, mine && cur.row >= 0);
          const uint32_t nans = __ballot_sync(0xffffffffu, mine && nan);   // (pages outside the pool among them)
          // keys: all rows see all keys of the page; values: they are there, and some row sees each of them
          const bool seen = keys ? page_seen_by_all(p, cur.pos, w.first, w.last, a.window, a.sinks)
                                 : cur.row >= 0 && cur.pos + p.page - 1 <= w.last && (cur.pos > w.first - a.window || cur.pos + p.page - 1 < a.sinks);
          const bool all = __all_sync(0xffffffffu, !mine || seen);
          if (mine && keys) {
            PromptTile& ti = info[issued % kInfo];
            if (lp == 0) ti.flags = nans || !all ? 1 : 0;
            const float ks = nan ? __int_as_float(0x7fc00000) : exp2i(cur.ke);
            const float ve = nan ? 0.f : (float)cur.ve;   // (nobody looks at what is NaN or not there)
            for (int i = 0; i < p.page / 16; ++i) {
              ti.ks[lp * (p.page / 16) + i] = ks;
              ti.pos[lp * (p.page / 16) + i] = cur.pos + 16 * i;
              ti.ve[lp * (p.page / 16) + i] = ve;
            }
          } else if (mine) {
            if (lp == 0) vinfo[s].all = all;
            vinfo[s].pos[lp] = cur.row >= 0 ? cur.pos : kNowhere;
            const __half h = __float2half_rn(nan || cur.row < 0 ? 0.f : wide ? 1.f : exp2i(cur.ve - vbase));
            vinfo[s].vs[lp] = (uint32_t)__half_as_ushort(h) * 0x10001u;
          }
          __syncwarp();
          // (the arrival also hands on what was written about the tile: to the converting warps, and by the products to the softmax warps)
          if (lane == 0) tc::mbar_expect_tx(&bars[full + s], __popc(loads) * p.page * D);
          __syncwarp();
          if (mine && cur.row >= 0) tc::tma_load_2d(tiles + s * Cfg::T8 + lp * p.page * D, map, &bars[full + s], 0, cur.row);
          ++issued;
          if (++s == ring) { s = 0; par ^= 1; }
          ++t;
        }
        if (MORE && keys) {   // what comes next
          PromptWork nx;
          nx.ntiles = 0;
          while (asking) {
            ok = __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[PB_NEXT], asked & 1)) && ok;
            ++asked;
            const int block = ok ? next_block(base + Cfg::OFF_NEXT) : -1;
            tc::fence_proxy_async();
            __syncwarp();
            if (block < 0 || prompt_work(args, block, 0, nx)) { if (block < 0) nx.ntiles = 0; break; }
            if (lane == 0) ask_next(base + Cfg::OFF_NEXT, &bars[PB_NEXT]);
          }
          if (lane == 0) {
            works[(item + 1) % kWorks] = nx;
            tc::mbar_arrive(&bars[PB_WORK + (item + 1) % kWorks]);
          }
          __syncwarp();
        }
      }
      if (lane == 0) {
        if (!ok) fail();
        // nothing may be in flight into shared memory when the CTA ends, whatever became of the others
#pragma unroll 1
        for (int j = max(0, issued - ring); j < issued; ++j) tc::mbar_wait_tight(&bars[full + j % ring], (j / ring) & 1);
      }
    } else if (warp == 1) {
      // ------------------------------ S ------------------------------
      // (an issuing thread competes with the softmax warps for every instruction: descriptors are advanced, not built, and nothing but
      // barriers is looked at)
      if (lane == 0) {
        constexpr uint32_t ID = tc::idesc_f16(128, 128, false);   // (format 0: e4m3 in kind::f8f6f4)
        auto desc = [](uint32_t addr) { return D == 128 ? tc::smem_desc_sw128(addr, 16, 1024) : tc::smem_desc_sw64(addr, 16, 512); };
        const uint64_t dQ = desc(tc::smem_u32(base + Cfg::OFF_Q)), dK = desc(tc::smem_u32(base + Cfg::OFF_K));
        bool ok = true;
        int J = 0;
        uint32_t s = 0, par = 0;   // ring of three: key tiles and accumulators
#pragma unroll 1
        for (int item = 0; work_there(item, ok); ++item) {
          ok = tc::mbar_wait_tight(&bars[PB_QFULL], item & 1);
          const int ntiles = work(item).ntiles;
#pragma unroll 1
          for (int j = 0; j < ntiles && ok; ++j, ++J) {
            ok = tc::mbar_wait_tight(&bars[PB_KFULL + s], par);   // (long there, as a rule: not behind the wait that matters)
            ok = ok && (J < Cfg::NACC || tc::mbar_wait_tight(&bars[PB_PVDONE + s], par ^ 1));
            if (!ok) break;
            tc::tc_fence_after();
            const uint64_t k = dK + s * (Cfg::T8 >> 4);
            const uint32_t dS = tmem + Cfg::COL_S + 128 * s;
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) tc::mma_f8_ss(dS, dQ + 2 * ks, k + 2 * ks, ID, ks > 0);
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) tc::mma_f8_ss(dS, dQ + (Cfg::T8 >> 4) + 2 * ks, k + 2 * ks, ID, 1u);
            tc::mma_commit(&bars[PB_SFULL + s]);
            tc::mma_commit(&bars[PB_KFREE + s]);
            if (++s == 3) { s = 0; par ^= 1; }
          }
        }
        if (!ok) fail();
      }
    } else if (warp == 2) {
      // ------------------------------ P V ------------------------------
      if (lane == 0) {
        constexpr uint32_t ID = tc::idesc_f16(128, D, true);
        const uint64_t dV = tc::smem_desc_sw128(tc::smem_u32(base + Cfg::OFF_V), 128 * 128, 1024);
        uint32_t s = 0, par = 0, J = 0;
        bool ok = true;
#pragma unroll 1
        for (int item = 0; work_there(item, ok); ++item) {
          const int ntiles = work(item).ntiles;
#pragma unroll 1
          for (int j = 0; j < ntiles; ++j, ++J) {
            ok = tc::mbar_wait_tight(&bars[PB_READY + s], par);
            if (!ok) break;
            tc::tc_fence_after();
            const uint64_t v = dV + (J & 1) * (Cfg::T16 >> 4);
            const uint32_t aP = tmem + Cfg::COL_S + 128 * s;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)   // 16 keys: 8 columns of P, 16 rows of 128 bytes of every 64-channel half of V
              tc::mma_f16_ts(tmem + Cfg::COL_O, aP + 64 * (kk >> 2) + 8 * (kk & 3), v + kk * (2048 >> 4), ID, (j > 0 || kk > 0) ? 1u : 0u);
            tc::mma_commit(&bars[PB_PVDONE + s]);
            tc::mma_commit(&bars[PB_VFREE + (J & 1)]);
            if (++s == 3) { s = 0; par ^= 1; }
          }
          if (ok) tc::mma_commit(&bars[PB_LAST]);   // (a barrier of its own: a group whose tiles are done may be more than a phase ahead of PB_PVDONE)
        }
        if (!ok) fail();
      }
    }
  } else if (warp >= 20) {
    // ------------------------------ values to fp16 ------------------------------
    constexpr int PIECES = D / 16;             // 16-byte pieces of a row of codes
    constexpr int N = PIECES / 4;              // a warp's lanes take eight rows and four pieces at a time: no two share a bank
    const int r8 = lane & 7, pc0 = lane >> 3, rows0 = (warp - 20) * 32;
    bool ok = true;
    uint32_t s3 = 0;
    int J = 0;
#pragma unroll 1
    for (int item = 0; work_there_warp(item, ok); ++item) {
      const PromptWork w = work(item);
      {
        int v = -1000, low = 1000;
#pragma unroll 1
        for (int i = tid - 640; i < w.ntiles * ppt; i += 128) {
          int p0;
          const int page = page_of(w, i, p0);
          if (page < 0) continue;
          const int e = scale_exp(p.vs[page * p.Hkv + w.hk]);
          if (e < 128) { v = max(v, e); low = min(low, e); }
        }
        v = __reduce_max_sync(0xffffffffu, v);
        low = __reduce_min_sync(0xffffffffu, low);
        if (lane == 0) {
          // (two sets: the next work's is sought while this one's softmax may not have looked yet, the one after that when it is done)
          s_vmax[8 * (item & 1) + warp - 20] = v;
          s_vmax[8 * (item & 1) + 4 + warp - 20] = low;
          tc::mbar_arrive(&bars[PB_VBASE + (item & 1)]);
        }
      }
      ok = tc::mbar_wait_tight(&bars[PB_QFULL], item & 1);   // (the queries lay where the first tiles go)
#pragma unroll 1
      for (int j = 0; j < w.ntiles; ++j, ++J) {
        const int sv = J & 1, s8 = J % Cfg::NV8;
        bool good = ok && tc::mbar_wait_tight(&bars[PB_V8FULL + s8], (J / Cfg::NV8) & 1);
        if (good && J >= Cfg::NV) good = tc::mbar_wait_tight(&bars[PB_VFREE + sv], ((J >> 1) - 1) & 1);
        ok = __all_sync(0xffffffffu, good);
        if (!ok) break;
        const ValueTile& vt = vinfo[s8];
        const bool all = vt.all;
        const uint8_t* src = base + Cfg::OFF_V8 + s8 * Cfg::T8;
        uint8_t* dst = base + Cfg::OFF_V + sv * Cfg::T16;
        uint4 c[4 * N];
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) {
          const int r = rows0 + 8 * (i / N) + r8, pc = pc0 + 4 * (i % N);
          c[i] = *reinterpret_cast<const uint4*>(src + r * D + (D == 128 ? (pc ^ r8) : (pc ^ ((r8 >> 1) & 3))) * 16);
        }
        if (!all) {   // whatever the ring or the page holds there must not meet the weight 0
#pragma unroll
          for (int i = 0; i < 4 * N; ++i) {
            const int row = rows0 + 8 * (i / N) + r8, key = vt.pos[row >> p.page_shift] + (row & (p.page - 1));
            if (!(key <= w.last && (key > w.first - a.window || key < a.sinks))) c[i] = make_uint4(0, 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) {
          const int r = rows0 + 8 * (i / N) + r8, pc = pc0 + 4 * (i % N);
          const uint32_t f2 = vt.vs[(rows0 + 8 * (i / N)) >> p.page_shift];
          auto scaled = [&](uint32_t code2) {
            const uint32_t h = e4m3x2_to_f16x2(code2);
            const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&h), *reinterpret_cast<const __half2*>(&f2));
            return *reinterpret_cast<const uint32_t*>(&x);
          };
          uint4 lo, hi;
          lo.x = scaled(c[i].x & 0xffff); lo.y = scaled(c[i].x >> 16); lo.z = scaled(c[i].y & 0xffff); lo.w = scaled(c[i].y >> 16);
          hi.x = scaled(c[i].z & 0xffff); hi.y = scaled(c[i].z >> 16); hi.z = scaled(c[i].w & 0xffff); hi.w = scaled(c[i].w >> 16);
          uint8_t* at = dst + (pc >> 2) * (128 * 128) + r * 128;
          *reinterpret_cast<uint4*>(at + (((2 * (pc & 3)) ^ r8) << 4)) = lo;
          *reinterpret_cast<uint4*>(at + (((2 * (pc & 3) + 1) ^ r8) << 4)) = hi;
        }
        tc::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          tc::mbar_arrive(&bars[PB_READY + s3]);
          tc::mbar_arrive(&bars[PB_V8FREE + s8]);
        }
        if (++s3 == 3) s3 = 0;
      }
      ok = __all_sync(0xffffffffu, ok);
    }
    if (!ok && lane == 0) fail();
  } else {
    // ------------------------------ q; softmax; results ------------------------------
    const int group = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, quarter = warp & 3, row = quarter * 32 + lane;
    auto all_barrier = []() { asm volatile("bar.sync 1, 512;" ::: "memory"); };
    bool ok = true;
    // the queries as they are, to where the fp16 values will be (the converting warps wait for them to be used up)
    auto load_q = [&](const PromptWork& w) {
      uint8_t* raw = base + Cfg::OFF_V;
      constexpr int CPR = D / 8;   // 16-byte pieces of a row
#pragma unroll 1
      for (int i = tid - 128; i < 128 * CPR; i += 512) {
        const int r = i / CPR, c = i % CPR, rg = w.row0 + r, tok = args.by_group.div(rg), hq = w.hk * a.G + rg - tok * a.G;
        uint4* dst = reinterpret_cast<uint4*>(raw + r * (2 * D) + ((c ^ (r & 7)) << 4));
        const __nv_bfloat16* src = a.q + w.b * a.sq[0] + hq * a.sq[1] + tok * a.sq[2] + 8 * c;
        if (r >= w.rows) {
          *dst = make_uint4(0, 0, 0, 0);
        } else if (args.q_vec) {
          copy16_async(dst, src);
        } else {
#pragma unroll 1
          for (int e = 0; e < 8; ++e) reinterpret_cast<__nv_bfloat16*>(dst)[e] = src[e];
        }
      }
    };
    int J0 = 0;   // tiles of the works before
#pragma unroll 1
    for (int item = 0; ok; ++item) {
      const PromptWork& w = work(item);
      if (item == 0) load_q(w);
      {
        // power-of-two scale of the row's largest channel to [2^7, 2^8), two parts of e4m3, swizzled like the keys; D / 16 threads per row
        constexpr int TPR = D / 16;
        const uint8_t* raw = base + Cfg::OFF_V;
        asm volatile("cp.async.wait_all;" ::: "memory");
        all_barrier();
#pragma unroll 1
        for (int i = tid - 128; i < 128 * TPR; i += 512) {
          const int r = i / TPR, piece = i % TPR;
          uint32_t x[8];
          {
            const uint4 u = *reinterpret_cast<const uint4*>(raw + r * (2 * D) + (((2 * piece) ^ (r & 7)) << 4));
            const uint4 v = *reinterpret_cast<const uint4*>(raw + r * (2 * D) + (((2 * piece + 1) ^ (r & 7)) << 4));
            x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
          }
          uint32_t top2 = 0;
#pragma unroll
          for (int q = 0; q < 8; ++q) top2 = __vmaxu2(top2, x[q] & 0x7fff7fffu);
          uint32_t top = max(top2 & 0xffffu, top2 >> 16);
#pragma unroll
          for (int o = 1; o < TPR; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
          const bool nan = top >= 0x7f80u;
          const int e = max((int)(top >> 7), 10);
          const float mul = nan ? 0.f : exp2i(134 - e);
          uint32_t hi[4] = {0, 0, 0, 0}, lo[4] = {0, 0, 0, 0};
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const uint32_t v = nan ? 0u : x[q];
            const float y0 = __uint_as_float(v << 16) * mul, y1 = __uint_as_float(v & 0xffff0000u) * mul;
            uint32_t h, l;
            split_e4m3x2(y0, y1, h, l);
            hi[q >> 1] |= h << (16 * (q & 1));
            lo[q >> 1] |= l << (16 * (q & 1));
          }
          uint8_t* at = base + Cfg::OFF_Q + r * D + ((D == 128 ? piece ^ (r & 7) : piece ^ ((r >> 1) & 3)) << 4);
          *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(at + Cfg::T8) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          if (piece == 0) s_cq[r] = nan ? __int_as_float(0x7fc00000) : a.scale_log2 * exp2i(e - 134);
        }
        tc::fence_proxy_async();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars[PB_QFULL]);
        all_barrier();
      }
      const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), to = lanes + Cfg::COL_O;
      const int pos_row = row < w.rows ? w.start + args.by_group.div(w.row0 + row) : w.last;
      float cq = s_cq[row];
      bool bad = !(cq == cq);   // NaN rows are marked, not computed with
      if (bad) cq = 0.f;
      float m_ref = -INFINITY, l_run = 0.f;   // l_run is relative to 2^(m_ref - kShift)
      if (!tc::mbar_wait_tight(&bars[PB_VBASE + (item & 1)], (item >> 1) & 1)) ok = false;
      bool wide;   // (uniform)
      const float vbase = (float)vbase_found(item, wide);
      const int ntiles = w.ntiles;
      float* my_xm = xm + group * 512;   // [tile parity of the group][half][row]
      // (one of two builds of the loop: with the values' scales in the exponents, and without)
      auto walk = [&](auto in_exponents) {
        constexpr bool wide = decltype(in_exponents)::value;
        const int j0 = (group ^ J0) & 1;   // (tile J0 + j of the CTA belongs to group (J0 + j) % 2,)
        uint32_t s = (J0 + j0) % 3, par = ((J0 + j0) / 3) & 1, flip = 0;   // (accumulator (J0 + j) % 3, its phase (J0 + j) / 3)
#pragma unroll 1
        for (int j = j0; j < ntiles; j += 2, flip ^= 1) {
          const uint32_t ts = lanes + Cfg::COL_S + 128 * s, sb = s == 0 ? 2 : s - 1, parb = s == 0 ? par ^ 1 : par;   // (sb, parb: of the tile before)
          if (!tc::mbar_wait_tight(&bars[PB_SFULL + s], par)) ok = false;
          __syncwarp();
          tc::tc_fence_after();
          const PromptTile& ti = info[(J0 + j) % kInfo];
          const bool slow = ti.flags;   // (uniform) masks, or NaN scales
          // S of columns 64 half + 32 c .. + 31; what the row does not see as -inf
          auto load = [&](int c, uint32_t (&x)[32]) {
            tc::tmem_ld32(ts + 64 * half + 32 * c, x);
            tc::tmem_wait_ld();
            if (slow) {
              // bit i: the row sees column i.  j <= pos_row, and j > pos_row - window or j < sinks
              auto below = [&](int n) { return n <= 0 ? 0u : n >= 16 ? 0xffffu : (1u << n) - 1u; };   // columns i < n of 16
              const int low = pos_row - a.window;   // (window <= 2^31 - 1 and pos_row >= 0: no overflow)
              uint32_t see = 0;
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                const int key0 = ti.pos[4 * half + 2 * c + g];
                const float ks = ti.ks[4 * half + 2 * c + g];
                uint32_t cols = below(pos_row - key0 + 1) & (~below(low < key0 ? 0 : low - key0 + 1) | below(a.sinks - key0));
                if (!(ks == ks)) {
                  bad = bad || cols;
                  cols = 0;
                }
                see |= cols << (16 * g);
              }
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = (see >> i) & 1 ? x[i] : 0xff800000u;
            }
          };
          float mx = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            uint32_t x[32];
            load(c, x);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              float m = __uint_as_float(x[16 * g]), m2 = __uint_as_float(x[16 * g + 1]);
#pragma unroll
              for (int i = 2; i < 14; i += 4) {
                m = tc::fmax3(m, __uint_as_float(x[16 * g + i]), __uint_as_float(x[16 * g + i + 1]));
                m2 = tc::fmax3(m2, __uint_as_float(x[16 * g + i + 2]), __uint_as_float(x[16 * g + i + 3]));
              }
              m = tc::fmax3(m, __uint_as_float(x[16 * g + 14]), __uint_as_float(x[16 * g + 15]));
              // (the factor is never 0 or NaN: a masked column is -inf)
              float y = fmaxf(m, m2) * fmaxf(cq * ti.ks[4 * half + 2 * c + g], 1.17549435e-38f);
              if constexpr (wide) y += fmaxf(ti.ve[4 * half + 2 * c + g] - vbase, -(float)kFoldMost);
              mx = fmaxf(mx, y);
            }
          }
          // the maximum of the row's other half, and the reference of the tile before
          float* x2 = my_xm + flip * 256;
          x2[half * 128 + row] = mx;
          if (j > 0 && !tc::mbar_wait_tight(&bars[PB_REF + quarter * 3 + sb], parb)) ok = false;
          ok = pair_barrier(2 + 1 + group * 4 + quarter, ok);
          if (!ok) break;
          mx = fmaxf(mx, x2[(1 - half) * 128 + row]);
          // the reference of the row: that of the tile before, unless this tile's maximum is more than 2^8 above it
          float m = j > 0 ? s_m[row] : -INFINITY;
          if (__any_sync(0xffffffffu, mx > m + 8.0f || j == 0)) {   // (the same decision in both warps)
            const float mnew = fmaxf(m, mx);
            if (j > 0) {
              // all earlier P V products must have landed before O is touched; each warp takes half of the channels
              if (!tc::mbar_wait_tight(&bars[PB_PVDONE + sb], parb)) ok = false;
              __syncwarp();
              tc::tc_fence_after();
              const float corr = (m == -INFINITY) ? 0.f : tc::ex2_approx(m - mnew);
#pragma unroll 1
              for (int c = half * (D / 64); c < (half + 1) * (D / 64); ++c) {
                uint32_t r[32];
                tc::tmem_ld32(to + c * 32, r);
                tc::tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * corr);
                tc::tmem_st32(to + c * 32, r);
              }
              tc::tmem_wait_st();
              ok = pair_barrier(2 + 1 + group * 4 + quarter, ok);   // (both have read the reference)
            }
            m = mnew;
            if (half == 0) s_m[row] = m;
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&bars[PB_REF + quarter * 3 + s]);
          // (a wait that ran out is acted on at the next barrier of the pair, by both warps)
          l_run = m_ref == -INFINITY ? 0.f : l_run * tc::ex2_approx(m_ref - m);
          m_ref = m;
          const float neg_m = (m == -INFINITY) ? 0.f : kShift - m;
          const uint64_t neg_m2 = pack2(neg_m, neg_m);
          uint64_t s0 = 0, s1 = 0;   // sums of the tile's weights
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            uint32_t x[32], wd[16];
            load(c, x);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const float f = fmaxf(cq * ti.ks[4 * half + 2 * c + g], 1.17549435e-38f);
              const uint64_t f2 = pack2(f, f);
              float vr = 0.f, fold = 0.f;
              uint64_t a2 = neg_m2;
              if constexpr (wide) {
                vr = ti.ve[4 * half + 2 * c + g] - vbase;
                fold = fmaxf(vr, -(float)kFoldMost);
                a2 = pack2(neg_m + fold, neg_m + fold);
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint64_t y = fma2(pack2(__uint_as_float(x[16 * g + 2 * i]), __uint_as_float(x[16 * g + 2 * i + 1])), f2, a2);
                float p0, p1;
                unpack2(y, p0, p1);
                p0 = tc::ex2_approx(p0);
                p1 = tc::ex2_approx(p1);
                const uint64_t p2 = pack2(p0, p1);
                if (i & 1) s1 = add2(s1, p2); else s0 = add2(s0, p2);
                wd[8 * g + i] = to_f16x2(p0, p1);
              }
              if constexpr (wide) {
                float l0, l1;
                unpack2(add2(s0, s1), l0, l1);
                l_run = fmaf(l0 + l1, exp2i(-(int)fold), l_run);
                s0 = s1 = 0;
                if (vr < fold) {
#pragma unroll
                  for (int i = 0; i < 8; ++i) wd[8 * g + i] = 0;
                }
              }
            }
            tc::tmem_st16(ts + 64 * half + 16 * c, wd);   // (columns that this thread has read)
          }
          tc::tmem_wait_st();
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&bars[PB_READY + s]);
          float l0, l1;
          unpack2(add2(s0, s1), l0, l1);
          l_run += l0 + l1;
          if (s == 0) s = 2; else { --s; par ^= 1; }
        }
      };
      if (wide) walk(std::true_type{}); else walk(std::false_type{});
      if (ok) ok = tc::mbar_wait_tight(&bars[PB_LAST], item & 1);
      if (!ok) fail();
      const bool more = work_there_warp(item + 1, ok);
      tc::tc_fence_after();
      if (MORE && more) load_q(work(item + 1));   // (on its way while this one's results are written)
      // (the last P V is done: every reference has been decided) the row sum is the sum of its four threads' sums
      const float m_end = s_m[row];
      const int part4 = group * 2 + half;
      s_l[part4 * 128 + row] = m_ref == -INFINITY ? 0.f : l_run * tc::ex2_approx(m_ref - m_end);
      s_l[(4 + part4) * 128 + row] = bad ? 1.f : 0.f;
      {
        uint32_t r;   // (also whether all are well, and so whether there is a next time: the same for all)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t"
            "setp.ne.u32 p, %1, 0;\n\t"
            "barrier.cta.red.and.aligned.pred q, 1, 512, p;\n\t"
            "selp.u32 %0, 1, 0, q;\n\t}"
            : "=r"(r) : "r"(ok && !*abort_flag ? 1u : 0u) : "memory");
        ok = r != 0;
      }
      const bool good = ok;
      const float l = (s_l[row] + s_l[128 + row]) + (s_l[256 + row] + s_l[384 + row]), nan = __int_as_float(0x7fc00000);
      bad = s_l[512 + row] + s_l[640 + row] + s_l[768 + row] + s_l[896 + row] != 0.f;
      uint8_t* stage = base + Cfg::OFF_Q;   // (the queries are not needed any more)
      const int rg = w.row0 + row, tokr = args.by_group.div(rg), hqr = w.hk * a.G + rg - tokr * a.G;
      const float vunit = exp2i((int)vbase - kUnitExp), unit = bad ? nan : w.parts == 1 ? vunit / l : vunit;
      if (good && part4 < D / 32) {
        const int c = part4;   // 32 channels
        uint32_t r[32];
        __syncwarp();
        tc::tmem_ld32(to + c * 32, r);
        tc::tmem_wait_ld();
        if (w.parts > 1) {   // partial result: O (in units of 2^(m_end - kShift), as the sum), m_end and the sum, [channel][row]
          float* mine = a.part + ((int64_t)blockIdx.x * args.nsplit + blockIdx.y) * (D + 2) * 128;
#pragma unroll
          for (int i = 0; i < 32; ++i) mine[(c * 32 + i) * 128 + row] = __uint_as_float(r[i]) * unit;
          if (c == 0) {
            mine[D * 128 + row] = m_end;
            mine[(D + 1) * 128 + row] = bad ? nan : l;
          }
        } else if (args.out_vec) {   // rows go through shared memory, so that the global stores are whole rows of 16-byte pieces
          stage_row32<D>(stage, row, c, r, unit * exp2i(kUnitExp));
        } else if (row < w.rows) {
          __nv_bfloat16* orow = a.out + w.b * a.so[0] + hqr * a.so[1] + tokr * a.so[2] + c * 32;
#pragma unroll
          for (int i = 0; i < 32; ++i) orow[i] = __float2bfloat16_rn(__uint_as_float(r[i]) * unit * exp2i(kUnitExp));
        }
      }
      tc::tc_fence_before();   // (O has been read: the next product may be issued behind the barriers to come)
      if (w.parts == 1 && args.out_vec) {
        all_barrier();
        if (good) {
          constexpr int CPR = D / 8, RPI = 32 / CPR;
          const int k = lane % CPR;
#pragma unroll 1
          for (int i = (warp - 4) * RPI + lane / CPR; i < w.rows; i += 16 * RPI) {
            const int ri = w.row0 + i, tok = args.by_group.div(ri), hq = w.hk * a.G + ri - tok * a.G;
            *reinterpret_cast<uint4*>(a.out + w.b * a.so[0] + hq * a.so[1] + tok * a.so[2] + k * 8) = *stage_chunk<D>(stage, i, k);
          }
        }
      }
      J0 += ntiles;
      if (!MORE || !more) break;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");   // (queries of a work that is not begun, should a wait have run out)
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, 512);
  }
}

// Rows whose key tiles were split: thread = row, block (row tile, 16 channels).
template <int D>
__global__ void __launch_bounds__(128) prompt_combine_kernel(const __grid_constant__ PromptArgs args) {
  const AttendArgs& a = args.a;
  PromptWork w;
  const bool split = prompt_work(args, blockIdx.x, 0, w) && w.parts > 1;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // (by every block: what follows this grid counts on the end of the one before it)
  if (!split) return;
  const int row = threadIdx.x, c0 = blockIdx.y * 16;
  constexpr int ST = (D + 2) * 128;
  const float* part = a.part + (int64_t)blockIdx.x * args.nsplit * ST + row;
  float m = -INFINITY;
#pragma unroll 8
  for (int z = 0; z < w.parts; ++z) m = fmaxf(m, part[z * ST + D * 128]);
  float o[16], l = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll 2
  for (int z = 0; z < w.parts; ++z) {
    const float mz = part[z * ST + D * 128], lz = part[z * ST + (D + 1) * 128];
    const float wz = mz == -INFINITY ? 0.f : tc::ex2_approx(mz - m);
    l += lz == lz ? lz * wz : lz;   // (a NaN row stays one where its weight is 0)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = fmaf(part[z * ST + (c0 + i) * 128], wz, o[i]);
  }
  if (row >= w.rows) return;
  const int rg = w.row0 + row, tok = args.by_group.div(rg), hq = w.hk * a.G + rg - tok * a.G;
  __nv_bfloat16* out = a.out + w.b * a.so[0] + hq * a.so[1] + tok * a.so[2] + c0;
  const float inv = 1.f / l;
  __nv_bfloat162 h[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = __floats2bfloat162_rn(o[2 * i] * inv * exp2i(kUnitExp), o[2 * i + 1] * inv * exp2i(kUnitExp));
  if (args.out_vec) {
    reinterpret_cast<uint4*>(out)[0] = reinterpret_cast<uint4*>(h)[0];
    reinterpret_cast<uint4*>(out)[1] = reinterpret_cast<uint4*>(h)[1];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) { out[2 * i] = h[i].x; out[2 * i + 1] = h[i].y; }
  }
}

// (row tiles of 128, key splits) of a call: the number of splits that the launch is done with first, if every row tile saw `tiles` key tiles, a CTA's
// set-up and end took as long as five of them (8 us and 1.3 us a tile, when the rule was made) and the merge as three.  Row tiles that see fewer take
// fewer (prompt_work).  Lengths are on the device, so without a window `tiles` is what the page table has room for: a table wider than the sequences
// costs splits, and a merge, that they do not ask for (300 tokens behind 3000, 32 heads on 8: 40 us, 66 with a table for 32768).
static void prompt_plan(int64_t units, int64_t rows, int64_t tiles, int& qtiles, int& nsplit) {
  qtiles = (int)((rows + kRows - 1) / kRows);
  const int64_t ctas = units * qtiles;
  nsplit = 1;
  int64_t best = INT64_MAX;
  for (int ns = 1; ns <= kMaxSplits && ns <= (tiles + kSplitTiles - 1) / kSplitTiles && (ns == 1 || ctas * ns <= 4 * 148); ++ns) {
    const int64_t cost = (ctas * ns + 147) / 148 * ((tiles + ns - 1) / ns + 5) + (ns > 1 ? 3 : 0);
    if (cost < best) { best = cost; nsplit = ns; }
  }
}

int64_t prompt_workspace(int64_t units, int64_t rows, int64_t tiles, int d) {
  int qt, ns;
  prompt_plan(units, rows, tiles, qt, ns);
  return ns == 1 ? 0 : units * qt * ns * (d + 2) * 128 * 4;
}

template <int D, bool MORE>
static kvm_status_t launch_prompt_d(const PromptArgs& args, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};   // devices on which the limit has been raised
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  if (dev > 63 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(prompt_kernel<D, MORE>, cudaFuncAttributeMaxDynamicSharedMemorySize, PromptCfg<D>::SMEM) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  prompt_kernel<D, MORE><<<dim3((unsigned)(args.units * args.qtiles), args.nsplit), kThreads, PromptCfg<D>::SMEM, s>>>(mapK, mapV, args);
  if (args.nsplit > 1) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)(args.units * args.qtiles), D / 16); lc.blockDim = dim3(128); lc.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at; lc.numAttrs = 1;
    if (cudaLaunchKernelEx(&lc, prompt_combine_kernel<D>, args) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  }
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}

kvm_status_t launch_prompt8(const AttendArgs& a, int64_t tiles, bool q_vec, bool out_vec, cudaStream_t s) {
  PromptArgs args;
  args.a = a;
  args.units = a.p.batch * a.p.Hkv;
  // Key tiles that 128 rows see: of a window layer far fewer than its table has, whose entries behind the window are only numbers.  Planned by the
  // table's width and by what is seen, behind 30000 tokens, 32 heads on 8: 300 tokens with a window of 128 22 and 18 us, 512 28 and 21, 2048 52 and 34,
  // 4096 72 and 54; 20 tokens 23 and 18, 23 and 20, 22 and 23, 25 and 23.  (Never more splits than the workspace is for, which is counted
  // without the window.)
  const int64_t seen = std::min<int64_t>(tiles, ((int64_t)a.window + a.sinks + 128 / a.G) / kTile + 2);
  int most;
  prompt_plan(args.units, a.p.T * a.G, tiles, args.qtiles, most);
  prompt_plan(args.units, a.p.T * a.G, seen, args.qtiles, args.nsplit);
  args.nsplit = std::min(args.nsplit, most);
  args.by_units = FastDiv(args.units); args.by_heads = FastDiv(a.p.Hkv); args.by_group = FastDiv(a.G);
  args.q_vec = q_vec ? 1 : 0; args.out_vec = out_vec ? 1 : 0;
  CUtensorMap mapK, mapV;
  const int64_t rows = a.p.n_pages * a.p.Hkv * a.p.page;
  if (!encode_tmap_codes(&mapK, a.p.k, a.d, rows, a.p.page) || !encode_tmap_codes(&mapV, a.p.v, a.d, rows, a.p.page)) return KVM_ERR_CUDA;
  // Going on saves the start of a CTA, and costs registers in the loop over the tiles: it pays where rows see few of them (two prompts of 8192, 16 heads,
  // d = 128, without and with: window 128 193 -> 177 us, 512 239 -> 224, 2048 387 -> 384, 4096 524 -> 534, all 622 -> 641; d = 64 on 4 heads:
  // 144 -> 128, 192 -> 179, 326 -> 317, 453 -> 451, 548 -> 554).  Not where a merge waits for the grid.
  constexpr int kMoreTiles = 18;
  const bool more = args.nsplit == 1 && seen <= kMoreTiles && (int64_t)args.units * args.qtiles > 148;
  if (a.d == 128) return more ? launch_prompt_d<128, true>(args, mapK, mapV, s) : launch_prompt_d<128, false>(args, mapK, mapV, s);
  return more ? launch_prompt_d<64, true>(args, mapK, mapV, s) : launch_prompt_d<64, false>(args, mapK, mapV, s);
}

}  // namespace cache
}  // namespace kvm
