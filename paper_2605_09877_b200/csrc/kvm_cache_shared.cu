// Attention for a batch whose sequences share their first blocks in groups (a system prompt, a document, the samples or beams of one prompt):
// every shared block is multiplied with the queries of its whole group, and read once per 128 rows of them.
//
// Three launches.  shared_kernel: the rows of a group, (sequence, token, head of a kv head's group), over the group's shared blocks, all of which
// all of them see.  The kernels of kvm_cache_attend in their SIDE builds: every sequence's rows over its own blocks.  shared_merge_kernel: partial
// results (O, reference m and sum l of a row, over some of its keys) to out = sum_z 2^(m_z - m) O_z / sum_z 2^(m_z - m) l_z.
//
// shared_kernel.  A unit is a (group, kv head) and 128 of the group's rows, or what is left of them.  The key tiles (128 tokens) of all units form one list; every CTA
// takes an equal, contiguous share of it, whatever the lengths and the sizes of the groups are, and leaves one partial result per unit that it has tiles of.
//     S = (q_hi + q_lo) K8^T   kind::f8f6f4: the codes as they lie in memory, q in two parts of e4m3
//     O += P V16               kind::f16: P in fp16 from tensor memory, V16 = the codes of the values as fp16 numbers (exact)
// S goes into three buffers in turn, P takes the place of its S; two groups of softmax warps take the tiles alternately, so that S of a tile and P V of another are
// under way beside the softmax of a third.  A row's reference, common to both groups, is the maximum of the unit's first tile, and hardly ever has to be changed: later, S is
// read once, no maximum is taken, and the two threads of a row, 64 columns each, need not meet.  What leaves the range shows in the sums of weights: then the products wait, the
// group takes new references and shifts O to them, and weights of the other group that are in units of older ones are shifted before they are used (a version tells).
// Scales of values go into the exponents of the weights, relative to the largest of the share's blocks, and out of the row sums again.
//   warp 0       producer of keys (TMA, page numbers and scales ahead), warp 3 of values
//   warp 1       issues the products, warp 2 finds the CTA's segments and writes down what the merge has to know
//   warps 4-19   queries (scaled, split); softmax, eight warps per group, two threads per row, 64 columns each; results
//   warps 20-23  value codes -> fp16, swizzled as the MMA reads them
//
// What bounds it: per 128 rows and 128 keys the products take 1024 cycles of the tensor core (q is there twice, so that S costs as much as in bf16), the powers 1024
// of the special-function unit, operands and tiles some 1400 of shared memory; the chain from S to S of a buffer makes 2300 of it.  64 sequences of 32 heads on a document of
// 32768 tokens: 58 us, of which 7 are start (the list, the queries) and 2 the results; the tensor core is active for a third of it.  (Without powers, stores of widened values and most
// of the products the whole call would take 70 us instead of 85: what is left is start, end, the keys' way and the two kernels behind.)  Half of the powers by a polynomial were
// slower (+9%: instructions).  Two row tiles on the same keys, each with its own O and one S, widened the values once for both, 88 us: more partial results, and nothing
// under way while a stream's weights are computed.  Code is read from memory by every CTA that begins: 93 -> 75 KB of it saved 2.5 us.
// Weights in bf16 need no maximum at all (2 us less), but add as much error again as the result's own rounding has.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "kvm_cache.cuh"
#include "kvm_internal.h"
#include "tc_common.cuh"

namespace kvm {
namespace cache {

kvm_status_t attend_args(const kvm_cache_t* cache, const kvm_cache_call_t* call, const void* q, int32_t n_q_heads, float scale, int32_t window, int32_t sinks, void* out,
                         const int64_t* q_strides, const int64_t* out_strides, int32_t* status, AttendArgs& a);

namespace {

constexpr int kCtas = 148;
constexpr int kThreads = 768;
constexpr int kInfo = 16;
// Weights of a row, 2^(y - m), y = logit + exponent of the value's scale relative to the largest (2^-kFoldMost at least), go into the products as fp16 numbers in units of
// 2^-kBias, and the codes of the values as fp16 numbers of 2^-kCode of what they stand for (their bits, shifted: nothing is multiplied).  The reference m need not be the
// row's maximum: anything will do between the largest y so far, rounded up, and where 16 weights sum up to more than kMost (fp16 ends at 65504, 2^9 of the reference).
// It is the largest y of the first tile to begin with; the largest weight is then at least 2^6, and half a step of fp16's least number 2^-31 of it.  Row sums take
// the weights before they are rounded, in fp32 and without the values' scales: at most 2^(9 + kFoldMost).
constexpr int kBias = 7, kCode = 8;
constexpr float kMost = 60000.f;
constexpr int kLowValues = 24;   // where the values are small their sums are held in units smaller by that, so that all bits stay above 2^-126
constexpr float kShift = 6.f;    // what the kernels for few and for many tokens count their weights in (of 2^-8 and 2^-6 of the reference)
constexpr float kDecodeShift = 8.f;
constexpr int kStartTiles = 4;   // key tiles that take as long as a unit's start and end

// A sequence, as shared_kernel leaves it for the merge: lengths (n = 0: no rows), its group's shared blocks and rows, its first row among them, the group's
// place in the list, and how the list is dealt.
struct alignas(16) SeqInfo { int start, n, blocks, rows, row0, pre, at, deal; };

struct SharedArgs {
  AttendArgs a;
  FastDiv by_seq, by_group;      // rows of a sequence, heads of a group
  int seq_rows, grid, q_vec, out_vec;
  float* part;                   // partial results of shared_kernel
  struct SeqInfo* seqs;          // [batch]: what the merge has to know
  // what the kernels over the other blocks leave: of few tokens (cols columns), of many (cols = 0)
  const float* own;
  int cols, workers;
  PromptSide many;
};

// What there is to do: prefix sums over the groups, in shared memory.
struct Plan {
  const int *offsets, *pre, *rows;   // sequences, positions of the list, rows of the partial results before each group
  int total, share;                  // positions; of a CTA
  bool whole;                        // every unit begins with a share: its positions are rounded up to whole ones
  __device__ __forceinline__ int length(int tiles) const { return whole ? (tiles + share - 1u) / (uint32_t)share * share : tiles; }   // of a unit
};
// One unit, as a CTA sees it that begins at position f of the list and ends at most at `end`.
struct Unit {
  int b0, hk, blocks, tiles;     // the group's first sequence, kv head; shared blocks, key tiles of the unit
  int row0, n;                   // the unit's rows among the group's
  int begin;                     // position of the first tile
  int at;                        // rows of partial results before the unit's first
  int pitch;                     // rows that a channel of a partial result takes
  // tiles [jb, je) of the CTA whose share begins at w0
  __device__ __forceinline__ void of(int w0, int share, int& jb, int& je) const {
    jb = max(0, w0 - begin);
    je = min(tiles, max(0, w0 + share - begin));
  }
  // where the partial result of that CTA (its number: cta) is: one step further in the list is one unit or one CTA further
  __device__ __forceinline__ int64_t slot(int cta) const { return at + (int64_t)cta * 128; }
};
__device__ __forceinline__ int rows_of_group(const SharedArgs& s, const int* offsets, int g) { return (offsets[g + 1] - offsets[g]) * s.seq_rows; }
// The shared blocks of a group (out of range: none, and the call is reported).
__device__ __forceinline__ int blocks_of_group(const SharedArgs& s, int g) {
  const int x = s.a.groups.shared[g];
  return x >= 0 && x <= s.a.p.max_pages ? x : -1;
}
__device__ __forceinline__ int tiles_of(const Params& p, int blocks) { return (blocks + (kTile >> p.page_shift) - 1) >> (7 - p.page_shift); }
__device__ __forceinline__ int pad8(int x) { return (x + 7) & ~7; }
// units of n rows of a group, per kv head; rows of their partial results
__device__ __forceinline__ int units_of(int n) { return (n + 127) >> 7; }
__device__ __forceinline__ int space_of(int n) { return (n & ~127) + pad8(n & 127); }

// The plan, by one warp; mem: 3 (n_groups + 1) ints.  false: groups that are none.
// Where there are no more units than CTAs, a share is the least of 32 lengths with which every CTA has tiles of one unit only: a unit that begins in the middle of a share
// costs its CTA a start and an end more, 6 us (kStartTiles), and the others wait for it.  Where none of them does (many short units beside long ones), either the longest unit is
// a share, or the list is dealt in equal ones whatever begins in them: what takes less for the CTA with the most to do.  Units of 128 channels, us as a list and with the
// longest as a share: 8 of 256 tiles and 112 of 2 (8 heads) 108 and 382; 16 of 150 and 130 of 1 144 and 234; 24 of 100 and 120 of 1 144 and 169; 38 of 60 and 110 of 2 103 and
// 118; and 38 of 60, 90 and 120 and 110 of 1 139, 183, 230 and 118, 158, 197.
__device__ __forceinline__ bool make_plan(const SharedArgs& s, int* mem, Plan& plan) {
  const Groups& gr = s.a.groups;
  const Params& p = s.a.p;
  int *offsets = mem, *pre = offsets + gr.n + 1, *rows = pre + gr.n + 1;
  plan.offsets = offsets; plan.pre = pre; plan.rows = rows;
  plan.total = 0;
  plan.share = 2;
  plan.whole = false;
  constexpr uint32_t kAll = 0xffffffffu;
  const int lane = threadIdx.x & 31;
  bool ok = true;
  int tiles_sum = 0, units = 0, most = 0, least = INT32_MAX;   // tiles of all units, units, tiles of the longest and of the shortest
#pragma unroll 1
  for (int g0 = 0; g0 <= gr.n; g0 += 32) {
    // sequences before a group; its key tiles (in `pre` for now)
    const int g = g0 + lane;
    if (g <= gr.n) {
      const int at = gr.offsets[g], end = g < gr.n ? gr.offsets[g + 1] : at, blocks = g < gr.n ? blocks_of_group(s, g) : 0;
      offsets[g] = at;
      ok = ok && end >= at && (g > 0 || at == 0) && (g < gr.n || at == p.batch);
      if (blocks < 0 && blockIdx.x == 0) report(p.status, KVM_ERR_INVALID_ARG);
      const int n = (end - at) * s.seq_rows, tiles = n > 0 && blocks > 0 ? tiles_of(p, blocks) : 0;
      pre[g] = tiles;
      if (tiles > 0) {
        tiles_sum += p.Hkv * tiles * units_of(n);
        units += p.Hkv * units_of(n);
        most = max(most, tiles);
        least = min(least, tiles);
      }
    }
  }
  if (!__all_sync(kAll, ok)) {
    if (blockIdx.x == 0 && lane == 0) report(p.status, KVM_ERR_INVALID_ARG);
    return false;
  }
  __syncwarp();
  units = __reduce_add_sync(kAll, units);
  plan.share = max(2, (__reduce_add_sync(kAll, tiles_sum) + s.grid - 1) / s.grid);   // (both groups of softmax warps have something to do)
  if (units <= s.grid && units > 0) {
    // every lane: how many CTAs the length share * (1 + lane / 16) takes
    const uint32_t length = plan.share + plan.share * lane / 16;
    int ctas = 0;
#pragma unroll 1
    for (int g0 = 0; g0 < gr.n; g0 += 32) {
      const int g = g0 + lane, t = g < gr.n ? pre[g] : 0, n = t > 0 ? rows_of_group(s, offsets, g) : 0;
#pragma unroll 1
      for (uint32_t there = __ballot_sync(kAll, t > 0); there; there &= there - 1) {
        const int i = __ffs(there) - 1, rows_i = __shfl_sync(kAll, n, i);
        const uint32_t tiles = __shfl_sync(kAll, t, i);
        ctas += units_of(rows_i) * ((tiles + length - 1) / length);
      }
    }
    const uint32_t fits = __ballot_sync(kAll, ctas * p.Hkv <= s.grid);
    most = __reduce_max_sync(kAll, most);
    least = __reduce_min_sync(kAll, least);
    if (fits) {
      plan.share = __shfl_sync(kAll, length, __ffs(fits) - 1);
      plan.whole = true;
    } else if (most <= plan.share + kStartTiles * ((plan.share - 2) / least + 1)) {   // (a run of so many tiles lies in that many units more than one, at most)
      plan.share = max(2, most);
      plan.whole = true;
    }
  }
  int at_pre = 0, at_rows = 0;   // before the next 32 groups
#pragma unroll 1
  for (int g0 = 0; g0 <= gr.n; g0 += 32) {
    const int g = g0 + lane, tiles = g < gr.n ? pre[g] : 0;
    int x = 0, y = 0;
    if (tiles > 0) {
      const int n = rows_of_group(s, offsets, g);
      x = p.Hkv * units_of(n) * plan.length(tiles);
      y = p.Hkv * space_of(n);
    }
    const int x0 = x, y0 = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int dx = __shfl_up_sync(kAll, x, o), dy = __shfl_up_sync(kAll, y, o);
      if (lane >= o) { x += dx; y += dy; }
    }
    if (g <= gr.n) {
      pre[g] = at_pre + x - x0;
      rows[g] = at_rows + y - y0;
    }
    at_pre += __shfl_sync(kAll, x, 31);
    at_rows += __shfl_sync(kAll, y, 31);
  }
  plan.total = at_pre;
  __syncwarp();
  return true;
}
// Last g with pre[g] <= f < pre[n].
__device__ __forceinline__ int last_before(const int* pre, int n, int f) {
  int lo = 0, hi = n;
#pragma unroll 1
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= f) lo = mid; else hi = mid;
  }
  return lo;
}
// The unit of rows 128 rb .. of kv head hk of a group: n rows behind `blocks` shared blocks, at position pre of the list, rows `at` of the partial results.
__device__ __forceinline__ Unit unit_of(const Params& p, const Plan& plan, int n, int blocks, int pre, int at, int hk, int rb) {
  Unit u;
  u.hk = hk; u.blocks = blocks;
  u.tiles = tiles_of(p, blocks);
  u.row0 = rb * 128;
  u.n = min(128, n - u.row0);
  u.pitch = pad8(u.n);
  u.begin = pre + (hk * units_of(n) + rb) * plan.length(u.tiles);
  u.at = at + hk * space_of(n) + u.row0;
  return u;
}
__device__ __forceinline__ Unit unit_at(const SharedArgs& s, const Plan& plan, int f) {
  const int g = last_before(plan.pre, s.a.groups.n, f), blocks = blocks_of_group(s, g), n = rows_of_group(s, plan.offsets, g);
  const uint32_t which = (uint32_t)(f - plan.pre[g]) / (uint32_t)plan.length(tiles_of(s.a.p, blocks)), hk = which / (uint32_t)units_of(n);
  Unit u = unit_of(s.a.p, plan, n, blocks, plan.pre[g], plan.rows[g], hk, which - hk * units_of(n));
  u.b0 = plan.offsets[g];
  return u;
}
// The CTA's next unit with tiles behind position f of the list; its share is [w0, w1).
template <class Segment>
__device__ __forceinline__ bool segment_at(const SharedArgs& s, const Plan& plan, int w0, int w1, int& f, Segment& g) {
  while (f < w1) {
    g.u = unit_at(s, plan, f);
    int je;
    g.u.of(w0, plan.share, g.jb, je);
    g.n = je - g.jb;
    f = g.u.begin + plan.length(g.u.tiles);
    if (g.n > 0) return true;
  }
  return false;
}
// A row of a group: its sequence, token and head (of the kv head's group).
struct Row { int b, t, h; };
__device__ __forceinline__ Row row_of(const SharedArgs& s, int b0, int r) {
  Row x;
  const int q = s.by_seq.div(r);
  r -= q * s.seq_rows;
  x.b = b0 + q;
  x.t = s.by_group.div(r);
  x.h = r - x.t * s.a.G;
  return x;
}

struct alignas(16) KeyTile {
  int flags;          // 1: some scale is NaN (or some page outside the pool)
  int n;              // keys that are there
  float ks[8], ve[8]; // per 16 keys: scale of the keys, exponent of the values' scale
};

// SB_SFULL: [group][number of its tile & 1]; SB_PREADY, SB_VERDICT: per group of softmax warps
enum { SB_KFULL = 0, SB_KFREE = 6, SB_V8FULL = 12, SB_V8FREE = 16, SB_VFULL = 20, SB_VFREE = 22, SB_SFULL = 24, SB_PREADY = 28, SB_VERDICT = 30, SB_PVDONE = 32,
       SB_END = 33, SB_REF = 34, SB_QFULL = 35, SB_VBASE = 36, SB_SEGFULL = 40, SB_SEGFREE = 44, SB_COUNT = 48 };

struct Segment { Unit u; int jb, n; };   // tiles [jb, jb + n) of the unit; n = 0: there are no more
template <int D>
struct SharedCfg {
  static constexpr int NK = D == 128 ? 5 : 6, NV8 = 2 * (128 / D), NV = 2;   // (3 of each with 128 channels: 84.4 us instead of 84.0 on a document)
  static constexpr int T8 = 128 * D, T16 = 256 * D;
  static constexpr int OFF_Q = 0;                        // hi, lo
  static constexpr int OFF_K = OFF_Q + 2 * T8;
  static constexpr int OFF_V8 = OFF_K + NK * T8;
  static constexpr int OFF_V = OFF_V8 + NV8 * T8;
  static constexpr int OFF_INFO = OFF_V + NV * T16;
  static constexpr int OFF_CQ = OFF_INFO + kInfo * (int)sizeof(KeyTile);   // float [128]
  static constexpr int OFF_REF = OFF_CQ + 128 * 4;                         // float [128]: references of the rows
  static constexpr int OFF_X = OFF_REF + 128 * 4;                          // float [group][half][128]: maxima, sums
  static constexpr int OFF_BAR = OFF_X + 4 * 128 * 4;
  static constexpr int OFF_SEG = OFF_BAR + 640;          // Segment [4]
  static constexpr int OFF_PLAN = OFF_SEG + 256;         // int [3][n_groups + 1]
  // never less than half an SM, so that one CTA with its 512 columns of tensor memory is resident
  static int smem(int n_groups) { return std::max(OFF_PLAN + 12 * (n_groups + 1) + 1024, 120 * 1024); }
  static constexpr uint32_t COL_S = 0, COL_O = 384;      // S of buffer b: + 128 b
  static_assert(NK <= 6 && NV8 <= 4 && NK + 3 <= kInfo, "rings");   // (S is at most three tiles ahead of the softmax)
  static_assert(OFF_K % 1024 == 0 && OFF_V8 % 1024 == 0 && OFF_V % 1024 == 0 && OFF_INFO % 16 == 0 && OFF_CQ % 16 == 0 && OFF_BAR % 8 == 0 && OFF_PLAN % 8 == 0, "alignment");
  static_assert(4 * sizeof(Segment) <= 256, "shared memory");
  static_assert(SB_COUNT * 8 + 192 <= 640 && OFF_PLAN + 12 * (kMaxBatch + 1) + 1024 <= 227 * 1024, "shared memory");
};

// Four e4m3 codes (channels 0 .. 3) as fp16 numbers of 2^-kCode of what they stand for, channels 0 and 2, then 1 and 3: sign, four bits of exponent and three
// of mantissa where they belong (a subnormal code is a subnormal number).  The results' channels are put in order when they are read.
__device__ __forceinline__ void widen4(uint32_t c, uint32_t& even, uint32_t& odd) {
  even = ((c & 0x007f007fu) << 7) | ((c << 8) & 0x80008000u);
  odd = ((c & 0x7f007f00u) >> 1) | (c & 0x80008000u);
}
__device__ __forceinline__ int channel_of(int i) { return (i & ~3) | ((i & 1) << 1) | ((i >> 1) & 1); }
// Barrier of the two warps of a group that share 32 rows.
__device__ __forceinline__ void pair_barrier(int id) {
  __syncwarp();
  asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
}
// A warp that gives up does not keep the other one waiting.
__device__ __forceinline__ void pair_leave(int id) {
  __syncwarp();
  asm volatile("bar.arrive %0, 64;" ::"r"(id) : "memory");
}
// One thread of a warp (the same one every time).
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
template <int D>
__global__ void __launch_bounds__(kThreads, 1)
shared_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const __grid_constant__ SharedArgs args) {
  using Cfg = SharedCfg<D>;
  const AttendArgs& a = args.a;
  const Params& p = a.p;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  KeyTile* info = reinterpret_cast<KeyTile*>(base + Cfg::OFF_INFO);
  float* s_cq = reinterpret_cast<float*>(base + Cfg::OFF_CQ);
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + Cfg::OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + SB_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_vmax = reinterpret_cast<int*>(tmem_slot + 2);                  // [segment % 4][4]
  volatile uint32_t* s_there = reinterpret_cast<uint32_t*>(s_vmax + 16); // [value tile of the ring]: pages that were loaded
  volatile int* s_flag = reinterpret_cast<int*>(s_vmax + 20);           // [group]: the tile whose weights leave the range
  volatile int* s_redo = s_flag + 2;                                    // [group]: the tile that is done again
  volatile int* s_used = s_redo + 2;                                    // [group][warp]: the version of the references that its weights are in
  volatile int* s_version = s_used + 16;                                // (written by the warp that issues the products alone)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (who waits for this kernel does so before reading what it wrote)
  if (warp == 0) {
    for (int i = lane; i < SB_COUNT; i += 32) {
      auto in = [&](int first, int n) { return i >= first && i < first + n; };
      tc::mbar_init(&bars[i], in(SB_V8FREE, 4) || in(SB_VFULL, 2) || in(SB_VBASE, 4) || i == SB_REF ? 4 : in(SB_PREADY, 2) || in(SB_SEGFREE, 4) ? 8 : i == SB_QFULL ? 16 : 1);
    }
    if (lane == 0) {
      tc::prefetch_tmap(&mapK); tc::prefetch_tmap(&mapV);
      *abort_flag = 0;
      s_flag[0] = s_flag[1] = s_redo[0] = s_redo[1] = -1;
      *s_version = 0;
    }
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  // The CTA's segments, as warp 2 finds them: a ring of four, for the three other single warps, the four that widen values and the softmax.
  Segment* segs = reinterpret_cast<Segment*>(base + Cfg::OFF_SEG);
  Plan plan;
  bool planned = false;
  int f = 0, w0 = 0, w1 = 0;   // where the next segment may begin; the share
  if (warp == 2) {
    planned = make_plan(args, reinterpret_cast<int*>(base + Cfg::OFF_PLAN), plan);
    if (planned) {
      f = w0 = (int)min((int64_t)plan.total, (int64_t)blockIdx.x * plan.share);
      w1 = min(plan.total, w0 + plan.share);
    }
    Segment first;
    if (!segment_at(args, plan, w0, w1, f, first)) first.n = 0;
    if (lane == 0) segs[0] = first;
  }
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto fail = [&]() {
    if (!*abort_flag) report(p.status, KVM_ERR_TIMEOUT);
    *abort_flag = 1;
  };
  auto next_segment = [&](int seg, Segment& g, bool& ok) {   // (by a whole warp)
    if (seg > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[SB_SEGFULL + (seg & 3)], (seg >> 2) & 1));
    if (!ok) return false;
    g = segs[seg & 3];
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(&bars[SB_SEGFREE + (seg & 3)]);
    return g.n > 0;
  };
  const int tshift = 7 - p.page_shift, ppt = 1 << tshift;
  Segment g;
  if (warp < 4) {
    if (warp == 2) {
      // ------------------------------ segments; what the merge has to know ------------------------------
      bool ok = true;
#pragma unroll 1
      for (int seg = 0; ok; ++seg) {
        if (seg >= 4) ok = __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[SB_SEGFREE + (seg & 3)], ((seg >> 2) - 1) & 1));
        if (!ok) break;
        if (seg == 0) g.n = segs[0].n;   // (it has been there since the block's barrier)
        else if (!segment_at(args, plan, w0, w1, f, g)) g.n = 0;
        if (lane == 0) {
          if (seg > 0) segs[seg & 3] = g;
          tc::mbar_arrive(&bars[SB_SEGFULL + (seg & 3)]);
        }
        if (seg == 0) {
#pragma unroll 1
          for (int b = blockIdx.x * 32 + lane; b < p.batch; b += args.grid * 32) {
            SeqInfo x{0, 0, 0, 0, 0, 0, 0, plan.share * 2 + (plan.whole ? 1 : 0)};
            if (planned) {
              const int g = last_before(plan.offsets, a.groups.n, b);
              x.blocks = blocks_of_group(args, g);
              x.rows = rows_of_group(args, plan.offsets, g);
              x.row0 = (b - plan.offsets[g]) * args.seq_rows;
              x.pre = plan.pre[g];
              x.at = plan.rows[g];
              if (!shared_lengths(p, b, x.blocks, x.start, x.n)) x.n = 0;
            }
            args.seqs[b] = x;
          }
          __syncwarp();
        }
        if (g.n == 0) break;
      }
      if (!ok && lane == 0) fail();
    } else if (warp == 0 || warp == 3) {
      // ------------------------------ producers of keys (warp 0) and values (warp 3) ------------------------------
      const bool keys = warp == 0;
      const int ring = keys ? Cfg::NK : Cfg::NV8, full = keys ? SB_KFULL : SB_V8FULL, empty = keys ? SB_KFREE : SB_V8FREE;
      const CUtensorMap* map = keys ? &mapK : &mapV;
      uint8_t* tiles = base + (keys ? Cfg::OFF_K : Cfg::OFF_V8);
      const int tpb = 32 >> tshift, lt = lane >> tshift, lp = lane & (ppt - 1);   // tiles whose pages the warp's lanes hold at a time
      struct Page { int row, ke, ve; };   // row < 0: not loaded
      bool ok = true;
      int s = 0, issued = 0;
      uint32_t par = 0;
#pragma unroll 1
      for (int seg = 0; ok && next_segment(seg, g, ok); ++seg) {
        const int32_t* table = p.pages + (int64_t)g.u.b0 * p.max_pages;
        auto fetch = [&](int k) {
          Page x{-1, 0, 0};
          const int j = k * tpb + lt, block = (g.jb + j) * ppt + lp;
          if (j < g.n && block < g.u.blocks) {
            const int page = table[block];
            if (page < 0 || page >= p.n_pages) {
              report(p.status, KVM_ERR_INVALID_ARG);
              x.ke = x.ve = 128;
            } else {
              const int unit = page * p.Hkv + g.u.hk;
              x.row = unit * p.page;
              x.ke = scale_exp(p.ks[unit]);
              x.ve = scale_exp(p.vs[unit]);
            }
          }
          return x;
        };
        Page cur{}, nxt{};
        for (int j = 0, ahead = 0, t = tpb; j < g.n; ++j) {   // (ahead: batches of pages fetched; t: tiles of the current one that are issued)
          if (t == tpb) {
            t = 0;
#pragma unroll 1
            do { cur = nxt; nxt = fetch(ahead++); } while (ahead < 2);   // (one batch is always on its way)
          }
          if (lane == 0) ok = issued < ring || tc::mbar_wait_tight(&bars[empty + s], par ^ 1);
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) break;
          const bool mine = lt == t, nan = cur.ke > 127 || cur.ve > 127;
          const uint32_t loads = __ballot_sync(0xffffffffu, mine && cur.row >= 0);
          const uint32_t nans = __ballot_sync(0xffffffffu, mine && nan);
          if (mine && keys) {
            KeyTile& ti = info[issued % kInfo];
            if (lp == 0) {
              ti.flags = nans ? 1 : 0;
              ti.n = min(kTile, (g.u.blocks - (g.jb + j) * ppt) << p.page_shift);
            }
            for (int i = 0; i < p.page / 16; ++i) {
              ti.ks[lp * (p.page / 16) + i] = nan ? 1.f : exp2i(cur.ke);   // (rows of a NaN are marked, not computed with)
              ti.ve[lp * (p.page / 16) + i] = nan || cur.row < 0 ? -1000.f : (float)cur.ve;   // (below all others: what is not there has no weight)
            }
          } else if (mine && lp == 0) {
            s_there[s] = loads >> lane;
          }
          __syncwarp();
          if (lane == 0) tc::mbar_expect_tx(&bars[full + s], __popc(loads) * p.page * D);
          __syncwarp();
          if (mine && cur.row >= 0) tc::tma_load_2d(tiles + s * Cfg::T8 + lp * p.page * D, map, &bars[full + s], 0, cur.row);
          ++issued;
          if (++s == ring) { s = 0; par ^= 1; }
          ++t;
        }
      }
      if (lane == 0) {
        if (!ok) fail();
        // nothing may be in flight into shared memory when the CTA ends, whatever became of the others
#pragma unroll 1
        for (int j = max(0, issued - ring); j < issued; ++j) tc::mbar_wait_tight(&bars[full + j % ring], (j / ring) & 1);
      }
    } else if (warp == 1) {
      // ------------------------------ products ------------------------------
      // S of a segment's tiles goes into three buffers in turn, up to three tiles ahead; P V of tile i waits for its weights, and what is behind it in the
      // buffer's place, S of tile i + 3, for P V.  Weights that leave the range, or are in units of references that have moved since, are done again before their P V, when
      // all products before it have landed: verdict.  The whole warp walks through this and one thread issues, so that addresses and descriptors are uniform.
      constexpr uint32_t ID_S = tc::idesc_f16(128, 128, false);   // (format 0: e4m3 in kind::f8f6f4)
      constexpr uint32_t ID_O = tc::idesc_f16(128, D, true);
      auto desc = [](uint32_t addr) { return D == 128 ? tc::smem_desc_sw128(addr, 16, 1024) : tc::smem_desc_sw64(addr, 16, 512); };
      const uint64_t dQ = desc(tc::smem_u32(base + Cfg::OFF_Q)), dK = desc(tc::smem_u32(base + Cfg::OFF_K));
      const uint64_t dV = tc::smem_desc_sw128(tc::smem_u32(base + Cfg::OFF_V), 128 * 128, 1024);
      const bool leader = elect_one();
      bool ok = true;
      uint32_t odd = 0, back = 0;            // per group: which of its two barriers S is next for; phase of the weights
      int J = 0, version = 0;                // tiles so far
      uint32_t s = 0, par = 0, v = 0, vpar = 0;   // rings of keys, of values
      auto wait = [&](int bar, uint32_t parity) {   // the same answer in every lane
        ok = ok && __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[bar], parity));
        return ok;
      };
#pragma unroll 1
      for (int seg = 0; ok && next_segment(seg, g, ok); ++seg) {
        if (!wait(SB_QFULL, seg & 1)) break;
        int j = 0;                           // next S, and its buffer
        uint32_t buf = 0, at = 0;            // (columns); at: buffer of the next P V
#pragma unroll 1
        for (int i = -3; i < g.n && ok; ++i) {
          // (what is there as a rule is asked for first, so that nothing but the products lies between the weights, P V and S)
          if (j < g.n && !wait(SB_KFULL + s, par)) break;
          if (i >= 0) {
            const uint32_t grp = i & 1;
            auto weights = [&]() {
              wait(SB_PREADY + grp, (back >> grp) & 1);
              back ^= 1u << grp;
            };
            if (!wait(SB_VFULL + v, vpar)) break;
            weights();
            if (!ok) break;
            const int said = lane < 8 ? s_used[8 * grp + lane] : s_flag[grp];
            const uint32_t again = __ballot_sync(0xffffffffu, lane < 8 ? said != version : said == J);
            const bool moved = again >> 8;
            if (again) {   // (at most once)
              tc::tc_fence_after();
              tc::tc_fence_before();
              if (leader) {
                s_redo[grp] = J;
                tc::mbar_arrive(&bars[SB_VERDICT + grp]);
              }
              __syncwarp();
              weights();
              if (!ok) break;
              if (moved) {
                ++version;
                if (leader) *s_version = version;   // (read behind a verdict to come)
              }
            }
            tc::tc_fence_after();
            const uint64_t b = dV + v * (Cfg::T16 >> 4);
            const uint32_t dO = tmem + Cfg::COL_O, aP = tmem + Cfg::COL_S + at, more = i > 0 ? 1u : 0u;
            if (leader) {
              tc::mbar_arrive(&bars[SB_VERDICT + grp]);
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)   // 16 keys: 8 columns of P, 16 rows of 128 bytes of every 64-channel half of V
                tc::mma_f16_ts(dO, aP + 64 * (kk >> 2) + 8 * (kk & 3), b + kk * (2048 >> 4), ID_O, kk > 0 ? 1u : more);
              tc::mma_commit(&bars[SB_PVDONE]);
              tc::mma_commit(&bars[SB_VFREE + v]);
            }
            __syncwarp();
            at = at == 256 ? 0 : at + 128;
            if (++v == Cfg::NV) { v = 0; vpar ^= 1; }
            if (!wait(SB_PVDONE, J & 1)) break;
            ++J;
          }
          if (j < g.n) {
            tc::tc_fence_after();
            const uint64_t k = dK + s * (Cfg::T8 >> 4);
            const uint32_t dS = tmem + Cfg::COL_S + buf, grp = j & 1;
            if (leader) {
#pragma unroll
              for (int ks = 0; ks < D / 32; ++ks) tc::mma_f8_ss(dS, dQ + 2 * ks, k + 2 * ks, ID_S, ks > 0);
#pragma unroll
              for (int ks = 0; ks < D / 32; ++ks) tc::mma_f8_ss(dS, dQ + (Cfg::T8 >> 4) + 2 * ks, k + 2 * ks, ID_S, 1u);
              tc::mma_commit(&bars[SB_SFULL + 2 * grp + ((odd >> grp) & 1)]);
              tc::mma_commit(&bars[SB_KFREE + s]);
            }
            __syncwarp();
            odd ^= 1u << grp;
            buf = buf == 256 ? 0 : buf + 128;
            if (++s == Cfg::NK) { s = 0; par ^= 1; }
            ++j;
          }
        }
        if (!ok) break;
        tc::tc_fence_after();
        tc::tc_fence_before();
        if (leader) tc::mbar_arrive(&bars[SB_END]);   // (all products have landed)
        __syncwarp();
      }
      if (!ok && leader) fail();
    }
  } else if (warp >= 20) {
    // ------------------------------ values to fp16 ------------------------------
    constexpr int PIECES = D / 16, N = PIECES / 4;   // 16-byte pieces of a row of codes; a warp's lanes take eight rows and four pieces at a time
    const int r8 = lane & 7, pc0 = lane >> 3, rows0 = (warp - 20) * 32;
    bool ok = true;
    int J = 0;
#pragma unroll 1
    for (int seg = 0; ok && next_segment(seg, g, ok); ++seg) {
      {   // largest exponent of the values' scales
        const int32_t* table = p.pages + (int64_t)g.u.b0 * p.max_pages;
        int v = -1000;
#pragma unroll 1
        for (int i = g.jb * ppt + tid - 640; i < min((g.jb + g.n) * ppt, g.u.blocks); i += 128) {
          const int page = table[i];
          if (page < 0 || page >= p.n_pages) continue;
          const int e = scale_exp(p.vs[page * p.Hkv + g.u.hk]);
          if (e < 128) v = max(v, e);
        }
        v = __reduce_max_sync(0xffffffffu, v);
        if (lane == 0) {
          // (four sets: with a tile of segment X to come, that of X - 3 has at least been used)
          s_vmax[4 * (seg & 3) + warp - 20] = v;
          tc::mbar_arrive(&bars[SB_VBASE + (seg & 3)]);
        }
      }
#pragma unroll 1
      for (int j = 0; j < g.n; ++j, ++J) {
        const int sv = J % Cfg::NV, s8 = J % Cfg::NV8;
        bool good = ok && tc::mbar_wait_tight(&bars[SB_V8FULL + s8], (J / Cfg::NV8) & 1);
        if (good && J >= Cfg::NV) good = tc::mbar_wait_tight(&bars[SB_VFREE + sv], (J / Cfg::NV - 1) & 1);
        ok = __all_sync(0xffffffffu, good);
        if (!ok) break;
        const uint32_t there = s_there[s8];
        const uint8_t* src = base + Cfg::OFF_V8 + s8 * Cfg::T8;
        uint8_t* dst = base + Cfg::OFF_V + sv * Cfg::T16;
        uint4 c[4 * N];
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) {
          const int r = rows0 + 8 * (i / N) + r8, pc = pc0 + 4 * (i % N);
          c[i] = *reinterpret_cast<const uint4*>(src + r * D + (D == 128 ? (pc ^ r8) : (pc ^ ((r8 >> 1) & 3))) * 16);
        }
        if (there != (1u << ppt) - 1) {   // whatever the ring holds there must not meet the weight 0
#pragma unroll
          for (int i = 0; i < 4 * N; ++i)
            if (!(there >> ((rows0 + 8 * (i / N) + r8) >> p.page_shift) & 1)) c[i] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) {
          const int r = rows0 + 8 * (i / N) + r8, pc = pc0 + 4 * (i % N);
          uint4 lo, hi;
          widen4(c[i].x, lo.x, lo.y); widen4(c[i].y, lo.z, lo.w);
          widen4(c[i].z, hi.x, hi.y); widen4(c[i].w, hi.z, hi.w);
          uint8_t* at = dst + (pc >> 2) * (128 * 128) + r * 128;
          *reinterpret_cast<uint4*>(at + (((2 * (pc & 3)) ^ r8) << 4)) = lo;
          *reinterpret_cast<uint4*>(at + (((2 * (pc & 3) + 1) ^ r8) << 4)) = hi;
        }
        tc::fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          tc::mbar_arrive(&bars[SB_VFULL + sv]);
          tc::mbar_arrive(&bars[SB_V8FREE + s8]);
        }
      }
    }
    if (!ok && lane == 0) fail();
  } else {
    // ------------------------------ q; softmax; results ------------------------------
    const int grp = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, quarter = warp & 3, row = quarter * 32 + lane, pair = 2 + 4 * grp + quarter;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), tO = lanes + Cfg::COL_O;
    float* s_x = reinterpret_cast<float*>(base + Cfg::OFF_X);                // [group][half][128]
    volatile float* s_ref = reinterpret_cast<float*>(base + Cfg::OFF_REF);
    auto rows_barrier = []() { asm volatile("bar.sync 1, 512;" ::: "memory"); };
    bool ok = true;
    int turn = 0, verdicts = 0, J0 = 0;   // tiles of this group, verdicts on them; tiles of the CTA
#pragma unroll 1
    for (int seg = 0;; ++seg) {
      const Segment& g = segs[seg & 3];   // (free again behind the results)
      if (g.n == 0) break;
      // The queries: every thread takes 32 bytes of a few rows, all on their way before the first is split (those of any alignment one after the other).  Rows behind a
      // sequence's count are taken as 0: whatever they hold must not move references that its warp shares (the results of other rows would be rounded otherwise).
      constexpr int TPR = D / 16, ITER = 128 * TPR / 512;   // threads per row; rows of a thread
      const int piece = tid % TPR, row0 = (tid - 128) / TPR;
      auto row_at = [&](const Row& rw) { return a.q + rw.b * a.sq[0] + (int64_t)(g.u.hk * a.G + rw.h) * a.sq[1] + rw.t * a.sq[2] + 16 * piece; };
      uint4 raw[2 * ITER];
      uint32_t there = 0;   // of the thread's rows: those in front of the count
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
        const int r = row0 + 512 / TPR * i;
        raw[2 * i] = raw[2 * i + 1] = make_uint4(0, 0, 0, 0);
        if (r < g.u.n) {
          const Row rw = row_of(args, g.u.b0, g.u.row0 + r);
          if (args.q_vec) {   // (on its way beside the count)
            const uint4* src = reinterpret_cast<const uint4*>(row_at(rw));
            raw[2 * i] = src[0];
            raw[2 * i + 1] = src[1];
          }
          if (!p.count || rw.t < p.count[rw.b]) there |= 1u << i;
        }
      }
#pragma unroll 1
      for (int i = 0; i < ITER; ++i) {
        // power-of-two scale of the row's largest channel to [2^7, 2^8), two parts of e4m3, swizzled like the keys
        const int r = row0 + 512 / TPR * i;
        uint32_t x[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
        for (int j = 0; j < 2 * ITER - 2; ++j) raw[j] = raw[j + 2];
        if (!(there >> i & 1)) {
#pragma unroll
          for (int q = 0; q < 8; ++q) x[q] = 0;
        } else if (!args.q_vec) {
          const uint16_t* src = reinterpret_cast<const uint16_t*>(row_at(row_of(args, g.u.b0, g.u.row0 + r)));
#pragma unroll
          for (int q = 0; q < 8; ++q) x[q] = src[2 * q] | (uint32_t)src[2 * q + 1] << 16;
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
          uint32_t h, l;
          split_e4m3x2(__uint_as_float(v << 16) * mul, __uint_as_float(v & 0xffff0000u) * mul, h, l);
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
      if (lane == 0) tc::mbar_arrive(&bars[SB_QFULL]);
      int version = *s_version;   // of the references that the group knows (nobody moves any before the first weights, which are given away behind this barrier)
      rows_barrier();
      float cq = s_cq[row];
      bool bad = !(cq == cq);   // NaN rows are marked, not computed with
      if (bad) cq = 0.f;
      ok = __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[SB_VBASE + (seg & 3)], (seg >> 2) & 1));
      const int* vm = s_vmax + 4 * (seg & 3);
      const int vb = max(max(vm[0], vm[1]), max(vm[2], vm[3]));
      const float vbase = vb == -1000 ? 0.f : (float)vb;
      float m = 0.f, l = 0.f;   // reference of the thread's weights (a whole number), their sum
      if (ok && grp == 1 && g.n > 1) {
        ok = __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[SB_REF], seg & 1));
        m = s_ref[row];
      }
      uint32_t tS = lanes + Cfg::COL_S + 128 * grp + 64 * half;
#pragma unroll 1
      for (int i = grp; i < g.n && ok; i += 2) {
        ok = __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[SB_SFULL + 2 * grp + (turn & 1)], (turn >> 1) & 1));
        ++turn;
        if (!ok) break;
        tc::tc_fence_after();
        const KeyTile& ti = info[(J0 + i) % kInfo];
        const int n = ti.n - 64 * half;         // the half's columns that are there: pages are whole, 16 columns are there or not
        if (ti.flags) bad = true;
        float sum = 0.f;
        bool held = false, redo = false;        // weights that are not given away: some leave the range
#pragma unroll 1
        for (;;) {
          if (i == 0 || redo) {
            // The row's reference in the first tile: its largest y.  Or some row has weights beyond the range, or references have moved for the tile before: the largest y of the
            // halves whose weights are held back, or what it is by now; weights that are not held back are shifted to it where they lie.  (References that the other
            // group has moved are taken over here only, however early they are there: results do not depend on who is faster.)
            const float now = redo ? s_ref[row] : -INFINITY;
            if (redo) version = *s_version + (s_flag[grp] == J0 + i ? 1 : 0);   // (once this is done)
            float mx = -INFINITY;
            if (!redo || held) {
#pragma unroll 1
              for (int c = 0; c < 4; ++c) {
                uint32_t x[16];
                tc::tmem_ld16(tS + 16 * c, x);
                tc::tmem_wait_ld();
                float m0 = -INFINITY;
#pragma unroll
                for (int k = 0; k < 16; ++k) m0 = fmaxf(m0, __uint_as_float(x[k]));
                const float fac = fmaxf(cq * ti.ks[4 * half + c], 1.17549435e-38f), fold = fmaxf(ti.ve[4 * half + c] - vbase, -(float)kFoldMost);
                if (16 * c < n) mx = fmaxf(mx, m0 * fac + fold);
              }
            }
            float* mine = s_x + 256 * grp + row;
            mine[128 * half] = mx;
            pair_barrier(pair);
            mx = ceilf(fmaxf(mx, mine[128 * (1 - half)]));
            const float next = redo ? fmaxf(now, mx) : mx;
            if (half == 0) s_ref[row] = next;
            if (redo) {
              if (i > 0 && __any_sync(0xffffffffu, next != now)) {
                const float corr = tc::ex2_approx(now - next);
#pragma unroll 1
                for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 16) {
                  uint32_t r[16];
                  tc::tmem_ld16(tO + c, r);
                  tc::tmem_wait_ld();
#pragma unroll
                  for (int k = 0; k < 16; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * corr);
                  tc::tmem_st16(tO + c, r);
                }
              }
              const float corr = tc::ex2_approx(m - next);
              if (i > 1) l *= corr;
              if (!held) {
#pragma unroll 1
                for (int c = 0; c < 32; c += 16) {
                  uint32_t r[16];
                  tc::tmem_ld16(tS + c, r);
                  tc::tmem_wait_ld();
#pragma unroll
                  for (int k = 0; k < 16; ++k) {
                    const float2 w = __half22float2(*reinterpret_cast<const __half2*>(&r[k]));
                    r[k] = to_f16x2(w.x * corr, w.y * corr);
                  }
                  tc::tmem_st16(tS + c, r);
                }
                sum *= corr;
              }
            } else if (half == 0) {
              __syncwarp();
              if (lane == 0) tc::mbar_arrive(&bars[SB_REF]);
            }
            m = next;
          }
          if (!redo || held) {
            uint32_t pr[32];   // weights of columns 64 half .. + 63, two to a word
            const float neg_m = (float)kBias - m;
            float top = 0.f;   // largest sum of 16 weights
            sum = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              uint32_t x[16];
              tc::tmem_ld16(tS + 16 * c, x);
              const float fac = fmaxf(cq * ti.ks[4 * half + c], 1.17549435e-38f);   // (never 0: what is not there is -inf)
              const float vr = ti.ve[4 * half + c] - vbase, fold = fmaxf(vr, -(float)kFoldMost);
              const uint64_t f2 = pack2(fac, fac), a2 = pack2(neg_m + fold, neg_m + fold);
              tc::tmem_wait_ld();
              if (n <= 16 * c) {
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = 0xff800000u;
              }
              uint64_t s0 = 0, s1 = 0;
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                float p0, p1;
                unpack2(fma2(pack2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), f2, a2), p0, p1);
                p0 = tc::ex2_approx(p0);
                p1 = tc::ex2_approx(p1);
                if (k & 1) s1 = add2(s1, pack2(p0, p1)); else s0 = add2(s0, pack2(p0, p1));
                pr[8 * c + k] = to_f16x2(p0, p1);
              }
              if (vr < fold) {
#pragma unroll
                for (int k = 0; k < 8; ++k) pr[8 * c + k] = 0;
              }
              float l0, l1;
              unpack2(add2(s0, s1), l0, l1);
              l0 += l1;
              sum += l0 * exp2i(-(int)fold - kBias);
              top = fmaxf(top, l0);
            }
            held = !redo && i > 0 && __any_sync(0xffffffffu, top > kMost);   // (the first tile has its own maximum)
            if (!held) tc::tmem_st32(tS, pr);   // (columns that the warp has read)
            else if (lane == 0) s_flag[grp] = J0 + i;
          }
          tc::tmem_wait_st();
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (!redo) s_used[8 * grp + ((warp - 4) & 7)] = version;
            tc::mbar_arrive(&bars[SB_PREADY + grp]);
          }
          ok = __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[SB_VERDICT + grp], verdicts & 1));
          ++verdicts;
          if (!ok || redo || s_redo[grp] != J0 + i) break;
          redo = true;
          tc::tc_fence_after();
        }
        l += sum;
        tS = tS >= lanes + Cfg::COL_S + 128 + 64 * half ? tS - 128 : tS + 256;   // (two buffers further of three)
      }
      if (!ok) pair_leave(pair);
      // (the next segment is waited for here, so that all warps begin it or none)
      ok = ok && __all_sync(0xffffffffu, tc::mbar_wait_tight(&bars[SB_END], seg & 1) && tc::mbar_wait_tight(&bars[SB_SEGFULL + ((seg + 1) & 3)], ((seg + 1) >> 2) & 1));
      tc::tc_fence_after();
      // the four threads' sums; whether all are well, and so whether there is a next time: the same for all
      const float nan = __int_as_float(0x7fc00000), ref = s_ref[row];
      s_x[256 * grp + 128 * half + row] = bad ? nan : g.n > grp ? l * tc::ex2_approx(m - ref) : 0.f;
      {
        uint32_t r;
        __syncwarp();
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t"
            "setp.ne.u32 p, %1, 0;\n\t"
            "barrier.cta.red.and.aligned.pred q, 1, 512, p;\n\t"
            "selp.u32 %0, 1, 0, q;\n\t}"
            : "=r"(r) : "r"(ok && !*abort_flag ? 1u : 0u) : "memory");
        ok = r != 0;
      }
      if (!ok) break;
      float* mine = args.part + g.u.slot(blockIdx.x) * (D + 2) + row;
      const float total = (s_x[row] + s_x[128 + row]) + (s_x[256 + row] + s_x[384 + row]);
      const float low_values = vbase > 0.f ? 0.f : (float)kLowValues;   // (so that neither the largest nor the smallest leave fp32's range)
      const float unit = total == total ? exp2i((int)vbase - kUnitExp + (int)low_values) : nan;
      const bool live = row < g.u.n;
#pragma unroll 1
      for (int c = (2 * grp + half) * (D / 4); c < (2 * grp + half + 1) * (D / 4); c += 16) {
        uint32_t r[16];
        tc::tmem_ld16(tO + c, r);
        tc::tmem_wait_ld();
        if (live) {
#pragma unroll
          for (int k = 0; k < 16; ++k) mine[(c + channel_of(k)) * g.u.pitch] = __uint_as_float(r[k]) * unit;
        }
      }
      if (live && grp == 0 && half == 0) {
        const float shift = (float)(kCode - kBias) - low_values;
        mine[D * g.u.pitch] = ref + shift;
        mine[(D + 1) * g.u.pitch] = total * exp2i(-(int)shift);
      }
      tc::tc_fence_before();   // (O has been read: the next product may be issued behind the barriers to come)
      J0 += g.n;
      rows_barrier();
      if (tid == 128) tc::mbar_arrive(&bars[SB_SEGFREE + (seg & 3)]);
    }
    if (!ok) fail();
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, 512);
  }
}

// Merge.  Block: 128 rows (b, t, head of the kv head's group), CH channels, one kv head; kLists threads per row, which take the row's partial results in turn.
// Bound by the latency of what it reads (10 MB, mostly out of L2).  Two lists, four partial results on their way, eight channels: 84.6 us for the whole call on 64 samples of a
// document, 50.9 for 24 x 4 tokens of 64 channels; four lists 87.5 and 50.3 (of two results 87.2 and 49.4), two results 85.9 and 52.9, six 84.8 and 51.0.
constexpr int kLists = 2;
template <int D, int CH>
__global__ void __launch_bounds__(128 * kLists) shared_merge_kernel(const __grid_constant__ SharedArgs s) {
  __shared__ float s_part[kLists - 1][CH + 2][128];
  const AttendArgs& a = s.a;
  const Params& p = a.p;
  const int lane = threadIdx.x & 127, list = threadIdx.x >> 7;
  const int r = blockIdx.x * 128 + lane, c0 = blockIdx.y * CH, hk = blockIdx.z;
  const Row rw = row_of(s, 0, r);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  SeqInfo x{};
  if (rw.b < p.batch) x = s.seqs[rw.b];
  const bool live = rw.t < x.n;
  const int start = x.start, n = x.n, blocks = x.blocks;
  float m = -INFINITY, l = 0.f, o[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) o[i] = 0.f;
  int turn = 0, seen = 0;   // this thread's next partial result; those of the lists before
  // Partial results z = 0 .. n - 1 at x + z * next (z = 0: at x0): channel i at [i * step], m, l; FOUR of them on their way at a time.
  auto add = [&](const float* x0, const float* x, int64_t next, int count, int64_t step, float below) {
    constexpr int FOUR = 4;
    const int64_t at_m = (D - c0) * step, at_l = at_m + step;
    for (; turn < count; turn += FOUR * kLists) {
      float mz[FOUR], lz[FOUR], v[FOUR][CH];
#pragma unroll
      for (int k = 0; k < FOUR; ++k) {
        const int z = turn + k * kLists;
        const float* y = z == 0 ? x0 : x + z * next;
        mz[k] = -INFINITY;
        lz[k] = 0.f;
        if (z < count) {
          mz[k] = y[at_m] - below;
          lz[k] = y[at_l];
#pragma unroll
          for (int i = 0; i < CH; ++i) v[k][i] = y[i * step];
        }
      }
      float mn = m;
#pragma unroll
      for (int k = 0; k < FOUR; ++k) mn = fmaxf(mn, mz[k]);
      const float f0 = m == -INFINITY ? 0.f : tc::ex2_approx(m - mn);
      l *= f0;
#pragma unroll
      for (int i = 0; i < CH; ++i) o[i] *= f0;
      m = mn;
#pragma unroll
      for (int k = 0; k < FOUR; ++k) {
        l = lz[k] == lz[k] ? l : lz[k];   // (a NaN row stays one where its weight is 0)
        if (mz[k] == -INFINITY) continue;   // (nothing was looked at there)
        const float f1 = tc::ex2_approx(mz[k] - mn);
        l = fmaf(lz[k], f1, l);
#pragma unroll
        for (int i = 0; i < CH; ++i) o[i] = fmaf(v[k][i], f1, o[i]);
      }
    }
  };
  auto add_after = [&](const float* x0, const float* x, int64_t next, int count, int64_t step, float below) {
    turn = (list - seen) & (kLists - 1);
    add(x0, x, next, count, step, below);
    seen += count;
  };
  // the shared blocks: the CTAs that had tiles of the unit
  if (live && blocks > 0) {
    Plan plan;
    plan.share = x.deal >> 1;
    plan.whole = x.deal & 1;
    int row = x.row0 + r - rw.b * s.seq_rows;
    const Unit u = unit_of(p, plan, x.rows, blocks, x.pre, x.at, hk, row >> 7);
    const int first = u.begin / plan.share, last = (u.begin + u.tiles - 1) / plan.share;
    const float* x0 = s.part + u.slot(first) * (D + 2) + (row & 127) + (int64_t)c0 * u.pitch;
    add_after(x0, x0, 128 * (D + 2), last - first + 1, u.pitch, 0.f);
  }
  // the sequence's own
  if (live) {
    const int64_t unit = (int64_t)rw.b * p.Hkv + hk;
    const int col = rw.t * a.G + rw.h;
    if (s.cols == 0) {
      const int qt = col >> 7, row0 = qt * 128, last = min(n * a.G, row0 + 128) - 1;   // (as prompt_work has it)
      const int tiles = pages_of(p, start + s.by_group.div(row0), start + s.by_group.div(last), INT32_MAX, 0, blocks).tiles, per = split_tiles(tiles, s.many.nsplit);
      const float* x = s.own + ((int64_t)(s.many.qtiles - 1 - qt) * p.batch * p.Hkv + unit) * s.many.nsplit * (D + 2) * 128 + (col & 127) + c0 * 128;
      add_after(x, x, (D + 2) * 128, (tiles + per - 1) / per, 128, kShift);
    } else {
      const int2 from = a.found[unit];
      const float* whole = a.side + (unit * s.cols + col) * (D + 2) + c0;
      const int z0 = max(0, min(from.x, s.workers - 1)), z1 = min(from.y, s.workers - 1);   // (what a call leaves whose waits ran out may be anything)
      const float* x = s.own + ((int64_t)2 * z0 * s.cols + col) * (D + 2) + c0;
      const int64_t slot = (int64_t)s.cols * (D + 2);
      if (from.y < 0) add_after(whole, whole, 0, 1, 1, kDecodeShift);
      else add_after(x + slot, x, 2 * slot, z1 - z0 + 1, 1, kDecodeShift);   // (the first worker's share begins with the unit)
    }
  }
  if (list > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) s_part[list - 1][i][lane] = o[i];
    s_part[list - 1][CH][lane] = m;
    s_part[list - 1][CH + 1][lane] = l;
  }
  __syncthreads();
  if (list > 0 || !live) return;
  float mn = m;
#pragma unroll
  for (int k = 0; k < kLists - 1; ++k) mn = fmaxf(mn, s_part[k][CH][lane]);
  float f = m == -INFINITY ? 0.f : tc::ex2_approx(m - mn);
  l *= f;
#pragma unroll
  for (int i = 0; i < CH; ++i) o[i] *= f;
#pragma unroll
  for (int k = 0; k < kLists - 1; ++k) {
    const float mz = s_part[k][CH][lane], lz = s_part[k][CH + 1][lane];
    f = mz == -INFINITY ? 0.f : tc::ex2_approx(mz - mn);
    l = lz == lz ? fmaf(lz, f, l) : lz;
#pragma unroll
    for (int i = 0; i < CH; ++i) o[i] = fmaf(s_part[k][i][lane], f, o[i]);
  }
  __nv_bfloat16* out = a.out + rw.b * a.so[0] + (int64_t)(hk * a.G + rw.h) * a.so[1] + rw.t * a.so[2] + c0;
  const float inv = 1.f / l;
  __nv_bfloat162 h[CH / 2];
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) h[i] = __floats2bfloat162_rn(o[2 * i] * inv * exp2i(kUnitExp), o[2 * i + 1] * inv * exp2i(kUnitExp));
  if (s.out_vec) {
#pragma unroll
    for (int i = 0; i < CH / 8; ++i) reinterpret_cast<uint4*>(out)[i] = reinterpret_cast<const uint4*>(h)[i];
  } else {
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) { out[2 * i] = h[i].x; out[2 * i + 1] = h[i].y; }
  }
}

// ---- arguments ----

struct Space {
  int64_t part, own, side, found, seqs, all;   // bytes
};
int64_t align16(int64_t x) { return (x + 15) & ~(int64_t)15; }
// Sizes of what a call leaves; false: beyond what is numbered in 32 bits.
bool space_of_call(const kvm_cache_t* c, const kvm_cache_call_t* call, int32_t n_groups, int32_t n_q_heads, Space& x) {
  const int64_t Hkv = c->n_kv_heads, G = n_q_heads / Hkv, B = call->batch, units = B * Hkv, cols = call->n_tokens * G, d = c->head_dim;
  const int64_t tiles = ((int64_t)call->max_pages * c->page_tokens + kTile - 1) / kTile;
  const int64_t rows = B * cols;
  if (rows > INT32_MAX / 4 || (rows / 128 + n_groups) * Hkv * tiles > INT32_MAX / 2) return false;
  const int64_t slots = Hkv * (rows + 8 * (int64_t)n_groups) + 128 * (kCtas + 1);
  if (slots > INT32_MAX / 2) return false;
  x.part = align16(slots * (d + 2) * 4);
  const bool few = cols <= kDecodeCols;
  x.own = align16(few ? decode_workspace(units, tiles, (int)d, (int)cols) : prompt_side_workspace(units, cols, tiles, (int)d));
  x.side = few ? align16(units * (cols <= 8 ? 8 : 16) * (d + 2) * 4) : 0;
  x.found = few ? align16(units * 8) : 0;
  x.seqs = B * (int64_t)sizeof(SeqInfo);
  x.all = x.part + x.own + x.side + x.found + x.seqs;
  return true;
}

template <int D>
kvm_status_t launch_shared(const SharedArgs& args, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};   // devices on which the limit has been raised
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  if (dev > 63 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(shared_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SharedCfg<D>::smem(kMaxBatch)) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  shared_kernel<D><<<args.grid, kThreads, SharedCfg<D>::smem(args.a.groups.n), s>>>(mapK, mapV, args);
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}
template <int D>
kvm_status_t launch_merge(const SharedArgs& args, cudaStream_t s) {
  constexpr int CH = 8;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at; lc.numAttrs = 1; lc.stream = s;
  lc.gridDim = dim3((unsigned)((args.a.p.batch * (int64_t)args.seq_rows + 127) / 128), D / CH, args.a.p.Hkv); lc.blockDim = dim3(128 * kLists);
  if (cudaLaunchKernelEx(&lc, shared_merge_kernel<D, CH>, args) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  return KVM_OK;
}

}  // namespace
}  // namespace cache
}  // namespace kvm

using namespace kvm;
using namespace kvm::cache;

#define KVM_API __attribute__((visibility("default")))

extern "C" {

KVM_API int64_t kvm_cache_shared_workspace(const kvm_cache_t* cache, const kvm_cache_call_t* call, int32_t n_groups, int32_t n_q_heads) {
  if (kvm_cache_workspace(cache, call, n_q_heads) < 0 || n_groups < 1 || n_groups > call->batch) return -1;
  Space x;
  return space_of_call(cache, call, n_groups, n_q_heads, x) ? x.all : -1;
}

KVM_API kvm_status_t kvm_cache_attend_shared(const kvm_cache_t* cache, const kvm_cache_call_t* call, const int32_t* groups, const int32_t* shared, int32_t n_groups,
                                             const void* q, int32_t n_q_heads, float scale, void* out, const int64_t* q_strides, const int64_t* out_strides,
                                             void* workspace, int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  SharedArgs args = {};
  const kvm_status_t rc = attend_args(cache, call, q, n_q_heads, scale, 0, 0, out, q_strides, out_strides, status, args.a);
  if (rc != KVM_OK) return rc;
  if (!groups || !shared || !aligned(groups, 4) || !aligned(shared, 4) || n_groups < 1 || n_groups > call->batch) return KVM_ERR_INVALID_ARG;
  AttendArgs& a = args.a;
  Space x;
  if (!space_of_call(cache, call, n_groups, n_q_heads, x)) return KVM_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 16)) return KVM_ERR_INVALID_ARG;
  if (workspace_bytes < x.all) return KVM_ERR_CAPACITY;
  uint8_t* ws = (uint8_t*)workspace;
  args.part = (float*)ws;
  args.own = a.part = (float*)(ws + x.part);
  a.side = (float*)(ws + x.part + x.own);
  a.found = (int2*)(ws + x.part + x.own + x.side);
  args.seqs = (SeqInfo*)(ws + x.part + x.own + x.side + x.found);
  a.groups = Groups{groups, shared, n_groups};
  args.seq_rows = (int)(a.p.T * a.G);
  args.cols = args.seq_rows <= 8 ? 8 : args.seq_rows <= kDecodeCols ? 16 : 0;
  args.by_seq = FastDiv(args.seq_rows); args.by_group = FastDiv(a.G);
  args.q_vec = rows_aligned(q, a.sq); args.out_vec = rows_aligned(out, a.so);
  const int64_t tiles = ((int64_t)a.p.max_pages * a.p.page + kTile - 1) / kTile, rows = (int64_t)a.p.batch * args.seq_rows;
  args.grid = (int)std::min<int64_t>(kCtas, (rows / 128 + n_groups) * a.p.Hkv * tiles);
  CUtensorMap maps[2];
  if (!encode_tmaps(maps, a.p, a.d)) return KVM_ERR_CUDA;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  kvm_status_t r = a.d == 128 ? launch_shared<128>(args, maps[0], maps[1], s) : launch_shared<64>(args, maps[0], maps[1], s);
  if (r == KVM_OK) r = args.cols ? launch_decode8_side(a, tiles, args.q_vec, maps, s, args.workers) : launch_prompt8_side(a, tiles, args.q_vec, maps, s, args.many);
  if (r == KVM_OK) r = a.d == 128 ? launch_merge<128>(args, s) : launch_merge<64>(args, s);
  return r;
}

}  // extern "C"
