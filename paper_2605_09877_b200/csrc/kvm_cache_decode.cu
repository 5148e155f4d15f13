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
// All tiles of all units form one list, of which every CTA takes an equal share, whatever the lengths are (2 CTAs per SM):
//   warp 0      producer: page numbers and scales of the tiles ahead (one page per lane), TMA into a ring of three tiles
//   warp 1      issues the MMAs (one thread)
//   warps 2, 3  q of the next unit: scaled, split, into shared memory
//   warps 4-7   softmax, thread = key; then thread = channel
// A unit that spans several CTAs is merged by combine_kernel from their partial results.
//
// Bound by HBM (2 d bytes per key and kv head): 
#include <algorithm>
#include <atomic>

#include "kvm_cache.cuh"
#include "tc_common.cuh"

namespace kvm {
namespace cache {

bool encode_tmap_codes(CUtensorMap* map, const void* base, int d, int64_t rows, int page);   // kvm_cache.cu

constexpr int kStages = 3;
constexpr int kCtas = 2 * 148;
constexpr float kPShift = 8.f;   // the largest weight of a tile is 2^8 (e4m3 ends at 448)

struct TileInfo {
  int pos, b, hk, flags;   // first key position; unit; 1: first tile of the CTA's share of the unit, 2: last
  int vmax;                // largest exponent of the visible blocks' value scales
  int pad[3];
  int16_t ke[8], ve[8];    // exponents of the scales per page of the tile
};

template <int D, int NC>
struct DecodeCfg {
  static constexpr int TILE = 128 * D;                   // codes of a tile of keys or values
  static constexpr int STAGE = 2 * TILE;
  static constexpr int NB = 2 * NC;                      // columns of the MMAs: hi, then lo
  static constexpr int Q_BYTES = NB * 128, P_BYTES = NB * 128;
  static constexpr int OFF_Q = kStages * STAGE;          // (behind the last value tile: see the descriptor of V for 64 channels)
  static constexpr int OFF_P = OFF_Q + 2 * Q_BYTES;
  static constexpr int OFF_INFO = OFF_P + P_BYTES;
  static constexpr int OFF_CQ = OFF_INFO + kStages * (int)sizeof(TileInfo);
  static constexpr int OFF_MAX = OFF_CQ + 4 * NC * 4;    // float [2][4][NC]
  static constexpr int OFF_AB = OFF_MAX + 2 * 4 * NC * 4;   // float4 [2][NC]
  static constexpr int OFF_L = OFF_AB + 2 * NC * 16;     // float [4][NC]
  static constexpr int OFF_BAR = OFF_L + 4 * NC * 4;
  static constexpr int OFF_SEQ = OFF_BAR + 256;          // int2 [batch], int [batch + 1]
  static constexpr uint32_t TMEM_COLS = 128;
  static constexpr uint32_t COL_S = 0, COL_O = 64;       // S of tile j at 32 (j & 1)
};
enum { DB_FULL = 0, DB_FREE = 3, DB_QFULL = 6, DB_QFREE = 10, DB_SFULL = 12, DB_SFREE = 14, DB_PFULL = 16, DB_ODONE = 17, DB_COUNT = 18 };

struct DecodeArgs8 {
  AttendArgs a;
  int grid;
  int q_vec;
};

__device__ __forceinline__ float redux_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// Barrier of the four softmax warps that also tells whether all of them are well.
__device__ __forceinline__ bool softmax_barrier(bool ok) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.aligned.pred q, 1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"(ok ? 1u : 0u) : "memory");
  return r != 0;
}

// Tiles that the call's tokens of a sequence see (0: none, or lengths that are not allowed).
__device__ __forceinline__ int seq_tiles(const AttendArgs& a, int start, int n) {
  return n > 0 ? tiles_of(start, start + n - 1, a.window, a.sinks).n : 0;
}
// Last b with pre[b] <= f (pre ascends; f < pre[batch], so that sequence b has tiles).
__device__ __forceinline__ int seq_of(const int* pre, int batch, int f) {
  int lo = 0, hi = batch;   // pre[lo] <= f < pre[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= f) lo = mid; else hi = mid;
  }
  return lo;
}

template <int D, int NC>
__global__ void __launch_bounds__(256, 2)
decode_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const __grid_constant__ DecodeArgs8 args) {
  using Cfg = DecodeCfg<D, NC>;
  constexpr int NB = Cfg::NB;
  const AttendArgs& a = args.a;
  const Params& p = a.p;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sP = base + Cfg::OFF_P;
  TileInfo* info = reinterpret_cast<TileInfo*>(base + Cfg::OFF_INFO);
  float* s_cq = reinterpret_cast<float*>(base + Cfg::OFF_CQ);      // [4][NC] factors of the columns' logits, by unit & 3
  float* s_max = reinterpret_cast<float*>(base + Cfg::OFF_MAX);
  float4* s_ab = reinterpret_cast<float4*>(base + Cfg::OFF_AB);
  float* s_l = reinterpret_cast<float*>(base + Cfg::OFF_L);
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + Cfg::OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + DB_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_scan = reinterpret_cast<int*>(tmem_slot + 2);             // [8]
  int2* s_len = reinterpret_cast<int2*>(base + Cfg::OFF_SEQ);
  int* pre = reinterpret_cast<int*>(s_len + p.batch);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    tc::prefetch_tmap(&mapK); tc::prefetch_tmap(&mapV);
    for (int s = 0; s < kStages; ++s) { tc::mbar_init(&bars[DB_FULL + s], 1); tc::mbar_init(&bars[DB_FREE + s], 1); }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&bars[DB_QFULL + 2 * s], 64);
      tc::mbar_init(&bars[DB_QFULL + 2 * s + 1], 64);
      tc::mbar_init(&bars[DB_QFREE + s], 1);
      tc::mbar_init(&bars[DB_SFULL + s], 1);
      tc::mbar_init(&bars[DB_SFREE + s], 4);
    }
    tc::mbar_init(&bars[DB_PFULL], 4);
    tc::mbar_init(&bars[DB_ODONE], 1);
    *abort_flag = 0;
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, Cfg::TMEM_COLS);
    tc::tmem_relinquish();
  }
  // the list of tiles: pre[b] = tiles of the sequences before b, all heads
  {
    const int per = (p.batch + 255) / 256, b0 = tid * per;
    int sum = 0;
    for (int b = b0; b < min(b0 + per, p.batch); ++b) {
      int start, n;
      if (!seq_lengths(p, b, start, n)) {
        if (blockIdx.x == 0) report(p.status, KVM_ERR_INVALID_ARG);
        start = n = 0;
      }
      s_len[b] = make_int2(start, n);
      pre[b] = sum;
      sum += seq_tiles(a, start, n) * p.Hkv;
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    int add = incl - sum;
    for (int w = 0; w < warp; ++w) add += s_scan[w];
    for (int b = b0; b < min(b0 + per, p.batch); ++b) pre[b] += add;
    if (tid == 255) pre[p.batch] = add + sum;
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int total = pre[p.batch];
  const int share = (total + args.grid - 1) / args.grid;
  const int F0 = min(total, (int)blockIdx.x * share), F1 = min(total, F0 + share), ntile = F1 - F0;

  if (warp == 0) {
    // ------------------------------ producer ------------------------------
    const int ppt = kTile / p.page, tpb = 32 / ppt;   // pages of a tile; tiles whose pages the warp's lanes hold at a time
    const int lt = lane / ppt, lp = lane % ppt;
    struct Page { int row, ke, ve, pos, b, hk, flags; };   // row < 0: not loaded
    auto fetch = [&](int k) {
      Page g{-1, 0, 0, 0, 0, 0, 0};
      const int f = F0 + k * tpb + lt;
      if (f < F1) {
        const int b = seq_of(pre, p.batch, f);
        const int2 len = s_len[b];
        const Tiles t = tiles_of(len.x, len.x + len.y - 1, a.window, a.sinks);
        const int rem = f - pre[b], hk = rem / t.n, i = rem - hk * t.n;
        const int last = len.x + len.y - 1;
        g.b = b; g.hk = hk; g.pos = tile_at(t, i) * kTile;
        g.flags = (i == 0 || f == F0 ? 1 : 0) | (i == t.n - 1 || f == F1 - 1 ? 2 : 0);
        const int p0 = g.pos + lp * p.page;   // the page is needed if any token of the call sees any of its positions
        if (p0 <= last && (p0 + p.page > len.x - a.window + 1 || p0 < a.sinks)) {
          const int page = p.pages[(int64_t)b * p.max_pages + (p0 >> p.page_shift)];
          if (page < 0 || page >= p.n_pages) {
            report(p.status, KVM_ERR_INVALID_ARG);
            g.ke = g.ve = 128;
          } else {
            const int unit = page * p.Hkv + hk;
            g.row = unit * p.page;
            g.ke = scale_exp(p.ks[unit]);
            g.ve = scale_exp(p.vs[unit]);
          }
        }
      }
      return g;
    };
    Page cur = fetch(0), nxt = fetch(1);
    int issued = 0;
    bool ok = true;
    for (int j = 0, k = 0, t = 0; j < ntile && ok; ++j) {
      const int s = j % kStages;
      if (lane == 0) ok = !*abort_flag && (j < kStages || tc::mbar_wait(&bars[DB_FREE + s], ((j / kStages) - 1) & 1));
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (!ok) break;
      const bool mine = lt == t;
      const uint32_t loads = __ballot_sync(0xffffffffu, mine && cur.row >= 0);
      int v = mine && cur.row >= 0 && cur.ve < 128 ? cur.ve : -1000;
      v = __reduce_max_sync(0xffffffffu, v);
      if (mine) {
        info[s].ke[lp] = (int16_t)cur.ke;
        info[s].ve[lp] = (int16_t)cur.ve;
        if (lp == 0) {
          info[s].pos = cur.pos; info[s].b = cur.b; info[s].hk = cur.hk; info[s].flags = cur.flags;
          info[s].vmax = v == -1000 ? 0 : v;
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_expect_tx(&bars[DB_FULL + s], __popc(loads) * 2 * p.page * D);
      __syncwarp();
      if (mine && cur.row >= 0) {
        uint8_t* dst = base + s * Cfg::STAGE + lp * p.page * D;
        tc::tma_load_2d(dst, &mapK, &bars[DB_FULL + s], 0, cur.row);
        tc::tma_load_2d(dst + Cfg::TILE, &mapV, &bars[DB_FULL + s], 0, cur.row);
      }
      issued = j + 1;
      if (++t == tpb) { t = 0; ++k; cur = nxt; nxt = fetch(k + 1); }
    }
    if (lane == 0) {
      if (!ok) {
        if (!*abort_flag) report(p.status, KVM_ERR_TIMEOUT);
        *abort_flag = 1;
      }
      // nothing may be in flight into shared memory when the CTA ends, whatever became of the others
      for (int j = max(0, issued - kStages); j < issued; ++j) tc::mbar_wait(&bars[DB_FULL + j % kStages], (j / kStages) & 1);
    }
  } else if (warp == 1) {
    // ------------------------------ MMA issuer ------------------------------
    if (lane == 0 && ntile > 0) {
      constexpr uint32_t ID_S = tc::idesc_f16(128, NB, false), ID_O = tc::idesc_f16(128, NB, false, true);
      const uint32_t a0 = tc::smem_u32(base);
      auto desc = [](uint32_t addr) { return D == 128 ? tc::smem_desc_sw128(addr, 16, 1024) : tc::smem_desc_sw64(addr, 16, 512); };
      bool ok = true;
      auto wait = [&](int bar, uint32_t parity) { ok = ok && !*abort_flag && tc::mbar_wait(&bars[bar], parity); return ok; };
      int seg = -1;
      auto product_pv = [&](int j) {
        const int s = j % kStages;
        if (!wait(DB_PFULL, j & 1)) return;
        tc::tc_fence_after();
        const uint32_t aV = a0 + s * Cfg::STAGE + Cfg::TILE, aP = a0 + Cfg::OFF_P;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          // V8 as it lies: channels contiguous ("MN-major"), 8-key groups one swizzle tile apart.  128 rows of A are needed; with 64 channels
          // rows 64.. are read from the next tile (never past OFF_P) and their results from nowhere.
          const uint64_t dv = D == 128 ? tc::smem_desc_sw128(aV + ks * 4096, 1024, 1024) : tc::smem_desc_sw64(aV + ks * 2048, 512, 512);
          tc::mma_f8_ss(tmem + Cfg::COL_O, dv, tc::smem_desc_sw128(aP + ks * 32, 16, 1024), ID_O, ks > 0);
        }
        tc::mma_commit(&bars[DB_ODONE]);
        tc::mma_commit(&bars[DB_FREE + s]);
      };
      for (int j = 0; j < ntile && ok; ++j) {
        const int s = j % kStages;
        if (!wait(DB_FULL + s, (j / kStages) & 1)) break;
        const int flags = info[s].flags;
        if (flags & 1) {
          ++seg;
          if (!wait(DB_QFULL + (seg & 3), (seg >> 2) & 1)) break;
        }
        if (j >= 2 && !wait(DB_SFREE + (j & 1), ((j >> 1) - 1) & 1)) break;
        tc::tc_fence_after();
        const uint32_t aK = a0 + s * Cfg::STAGE, aQ = a0 + Cfg::OFF_Q + (seg & 1) * Cfg::Q_BYTES;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
          tc::mma_f8_ss(tmem + Cfg::COL_S + 32 * (j & 1), desc(aK + ks * 32), desc(aQ + ks * 32), ID_S, ks > 0);
        tc::mma_commit(&bars[DB_SFULL + (j & 1)]);
        if (flags & 2) tc::mma_commit(&bars[DB_QFREE + (seg & 1)]);
        if (j > 0) product_pv(j - 1);
      }
      if (ok) product_pv(ntile - 1);
      if (!ok) {
        if (!*abort_flag) report(p.status, KVM_ERR_TIMEOUT);
        *abort_flag = 1;
      }
    }
  } else if (warp < 4) {
    // ------------------------------ q of the units ------------------------------
    // eight threads per column, D / 8 channels each
    constexpr int E = D / 8;
    const int t = tid - 64, part = t & 7;
    bool ok = true;
    for (int f = F0, seg = 0; f < F1 && ok; ++seg) {
      const int b = seq_of(pre, p.batch, f);
      const int2 len = s_len[b];
      const int nt = (pre[b + 1] - pre[b]) / p.Hkv, hk = (f - pre[b]) / nt;
      f = pre[b] + (hk + 1) * nt;
      uint8_t* sQ = base + Cfg::OFF_Q + (seg & 1) * Cfg::Q_BYTES;
      if (seg >= 2) {
        if (lane == 0) ok = !*abort_flag && tc::mbar_wait(&bars[DB_QFREE + (seg & 1)], ((seg >> 1) - 1) & 1);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
      }
#pragma unroll
      for (int c0 = 0; c0 < NC; c0 += 8) {
        const int c = c0 + (t >> 3);
        float x[E];
        uint32_t top = 0;
        const bool live = c < len.y * a.G;
        if (live) {
          const int tok = c / a.G, hq = hk * a.G + c - tok * a.G;
          const __nv_bfloat16* src = a.q + b * a.sq[0] + hq * a.sq[1] + tok * a.sq[2] + part * E;
          if (args.q_vec) {
#pragma unroll
            for (int i = 0; i < E / 8; ++i) {
              const uint4 w4 = *reinterpret_cast<const uint4*>(src + 8 * i);
              const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
              for (int q = 0; q < 4; ++q) { x[8 * i + 2 * q] = __uint_as_float(w[q] << 16); x[8 * i + 2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u); }
            }
          } else {
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = __bfloat162float(src[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i) x[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < E; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool bad = top >= 0x7f800000u;
        const int e = max((int)(top >> 23), 10);          // largest |q| is in [2^(e-127), 2^(e-126))
        const float mul = bad ? 0.f : exp2i(134 - e);     // to [2^7, 2^8)
        uint32_t hi[E / 4], lo[E / 4];
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
          uint32_t h2[2], l2[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float y0 = bad ? 0.f : x[4 * i + 2 * q] * mul, y1 = bad ? 0.f : x[4 * i + 2 * q + 1] * mul;
            h2[q] = to_e4m3x2(y0, y1);
            const float2 back = e4m3x2_to_float2(h2[q]);
            l2[q] = to_e4m3x2(y0 - back.x, y1 - back.y);
          }
          hi[i] = h2[0] | (h2[1] << 16);
          lo[i] = l2[0] | (l2[1] << 16);
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
        if (part == 0) s_cq[(seg & 3) * NC + c] = bad ? __int_as_float(0x7fc00000) : a.scale_log2 * exp2i(e - 134);
      }
      tc::fence_proxy_async();
      tc::mbar_arrive(&bars[DB_QFULL + (seg & 3)]);
    }
    if (!ok) {
      if (!*abort_flag) report(p.status, KVM_ERR_TIMEOUT);
      *abort_flag = 1;
    }
  } else {
    // ------------------------------ softmax; results ------------------------------
    const int tok = tid - 128, w4 = warp - 4;
    const uint32_t lanes = tmem + ((uint32_t)(w4 * 32) << 16);
    float o_run[NC], l_run[NC], l_new[NC];
    float m_run = -INFINITY, m_old = -INFINITY;   // (threads below NC: running reference of column tid)
    int seg = -1;
    int pb = 0, phk = 0, pflags = 0;              // the tile before
    bool ok = true;
    // adds the products of tile j to the running results, and stores those of a share that ends with it
    auto gather = [&](int j) {
      if (!tc::mbar_wait(&bars[DB_ODONE], j & 1)) ok = false;
      __syncwarp();
      tc::tc_fence_after();
      float o[NC];
      if (NC == 8) {
        uint32_t r[16];
        tc::tmem_ld16(lanes + Cfg::COL_O, r);
        tc::tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] = __uint_as_float(r[c % 8]) + __uint_as_float(r[8 + c % 8]);
      } else {
        uint32_t r[32];
        tc::tmem_ld32(lanes + Cfg::COL_O, r);
        tc::tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] = __uint_as_float(r[c]) + __uint_as_float(r[16 + c % 16]);
      }
      const bool first = pflags & 1;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float4 f = s_ab[(j & 1) * NC + c];   // factors of what there is, of the row sum, of the products
        o_run[c] = first ? o[c] * f.z : fmaf(o_run[c], f.x, o[c] * f.z);
        l_run[c] = first ? l_new[c] * f.y : fmaf(l_run[c], f.x, l_new[c] * f.y);
      }
      if (!(pflags & 2)) return;
      const int2 len = s_len[pb];
      const int ncol = len.y * a.G;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float l = l_run[c];
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
        if (lane == 0) s_l[w4 * NC + c] = l;
      }
      softmax_barrier(true);
      const int nt = (pre[pb + 1] - pre[pb]) / p.Hkv, u0 = pre[pb] + phk * nt;
      const bool whole = u0 >= F0 && u0 + nt <= F1;
      float* part = a.part + (int64_t)(2 * blockIdx.x + (u0 >= F0 ? 1 : 0)) * NC * (D + 2);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (c >= ncol) continue;
        const float l = s_l[c] + s_l[NC + c] + s_l[2 * NC + c] + s_l[3 * NC + c];
        if (whole) {
          const int t = c / a.G, hq = phk * a.G + c - t * a.G;
          if (tok < D) a.out[pb * a.so[0] + hq * a.so[1] + t * a.so[2] + tok] = __float2bfloat16_rn(o_run[c] / l);
        } else {
          if (tok < D) part[c * (D + 2) + tok] = o_run[c];
          if (tok == c) { part[c * (D + 2) + D] = (j == ntile - 1) ? m_run : m_old; part[c * (D + 2) + D + 1] = l; }
        }
      }
      softmax_barrier(true);   // (s_l is free again)
    };
    for (int j = 0; j < ntile; ++j) {
      const int s = j % kStages;
      if (!tc::mbar_wait(&bars[DB_SFULL + (j & 1)], (j >> 1) & 1)) ok = false;
      // (complete already: what the producer wrote about the tile and, below, the factors of the columns are acquired here)
      if (!tc::mbar_wait(&bars[DB_FULL + s], (j / kStages) & 1)) ok = false;
      __syncwarp();
      tc::tc_fence_after();
      float y[NC];
      if (NC == 8) {
        uint32_t r[16];
        tc::tmem_ld16(lanes + Cfg::COL_S + 32 * (j & 1), r);
        tc::tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < NC; ++c) y[c] = __uint_as_float(r[c % 8]) + __uint_as_float(r[8 + c % 8]);
      } else {
        uint32_t r[32];
        tc::tmem_ld32(lanes + Cfg::COL_S + 32 * (j & 1), r);
        tc::tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < NC; ++c) y[c] = __uint_as_float(r[c]) + __uint_as_float(r[16 + c % 16]);
      }
      const int flags = info[s].flags, b = info[s].b, hk = info[s].hk, vmax = info[s].vmax, pos = info[s].pos;
      const int ke = info[s].ke[tok >> p.page_shift], ve = info[s].ve[tok >> p.page_shift];
      if (flags & 1) {
        // (four slots: the factors of unit seg + 4 are written after the products of seg + 2, hence after this thread's use of seg's)
        ++seg;
        if (!tc::mbar_wait(&bars[DB_QFULL + (seg & 3)], (seg >> 2) & 1)) ok = false;
      }
      const int2 len = s_len[b];
      const int last = len.x + len.y - 1, key = pos + tok;
      const float ks = exp2i(ke);
      const int vr = ve > 127 ? 0 : max(ve - vmax, -60);              // exponent that the weights take over from the values' scale
      const float vrel = ve > 127 ? __int_as_float(0x7fc00000) : (float)vr;
      const bool any = key <= last && (key > len.x - a.window || key < a.sinks);   // some column sees the key
      const bool all = pos + 127 <= len.x && (pos > last - a.window || pos + 127 < a.sinks);   // (uniform) all columns see all keys
#pragma unroll
      for (int c = 0; c < NC; ++c) y[c] = fmaf(y[c] * s_cq[(seg & 3) * NC + c], ks, vrel);
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars[DB_SFREE + (j & 1)]);
      if (!all) {
        int t = 0, g = 0;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (!sees(len.x + t, key, a.window, a.sinks)) y[c] = -INFINITY;
          if (++g == a.G) { g = 0; ++t; }
        }
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float m = redux_max(y[c]);
        if (lane == c) s_max[((j & 1) * 4 + w4) * NC + c] = m;
      }
      ok = softmax_barrier(ok && !*abort_flag);
      if (!ok) break;
      if (tid - 128 < NC) {
        const float* x = s_max + (j & 1) * 4 * NC + tok;
        const float m = fmaxf(fmaxf(x[0], x[NC]), fmaxf(x[2 * NC], x[3 * NC]));
        m_old = m_run;
        const float from = (flags & 1) ? -INFINITY : m_run;
        m_run = fmaxf(from, m);
        const float alpha = from == -INFINITY ? 0.f : exp2f(from - m_run);
        const float beta = m == -INFINITY ? 0.f : exp2f(m - m_run);
        s_ab[(j & 1) * NC + tok] = make_float4(alpha, beta, beta * exp2i(vmax), 0.f);
      }
      if (j > 0) gather(j - 1);
      // weights: 2^(y - m + 8), in two parts
      const float back = exp2i(-vr);   // (NaN weights stay NaN in either form)
      const bool dropped = ve < 128 && ve - vmax < -60;   // its values are below 2^-60 of the tile's largest
#pragma unroll
      for (int c = 0; c < NC; c += 2) {
        float w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float* x = s_max + (j & 1) * 4 * NC + c + i;
          const float m = fmaxf(fmaxf(x[0], x[NC]), fmaxf(x[2 * NC], x[3 * NC]));
          w[i] = tc::ex2_approx(y[c + i] - (m == -INFINITY ? 0.f : m - kPShift));
        }
        const uint32_t hi = to_e4m3x2(w[0], w[1]);
        const float2 h = e4m3x2_to_float2(hi);
        const uint32_t lo = to_e4m3x2(w[0] - h.x, w[1] - h.y);
        const float2 l = e4m3x2_to_float2(lo);
        // The row sum takes the weights as the products get them, so that their rounding does not shift a flat row; but where the
        // values' scale has been taken over, a weight can be too small for e4m3 and still count in the sum.
        l_new[c] = vr == 0 ? h.x + l.x : w[0] * back;
        l_new[c + 1] = vr == 0 ? h.y + l.y : w[1] * back;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = c + i;
          uint8_t* at = sP + row * 128 + (((tok >> 4) ^ (row & 7)) << 4) + (tok & 15);
          at[0] = dropped ? 0 : (uint8_t)(hi >> (8 * i));
          at[NC * 128] = dropped ? 0 : (uint8_t)(lo >> (8 * i));
        }
      }
      if (!any) {   // whatever the ring or the page holds there must not meet the weight 0
        uint4* row = reinterpret_cast<uint4*>(base + s * Cfg::STAGE + Cfg::TILE + tok * D);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) row[i] = make_uint4(0, 0, 0, 0);
      }
      tc::fence_proxy_async();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars[DB_PFULL]);
      pb = b; phk = hk; pflags = flags;
    }
    if (ntile > 0) ok = softmax_barrier(ok) && ok;   // (the factors of the last tile)
    if (ok && ntile > 0) gather(ntile - 1);
    if (!ok) {
      if (!*abort_flag) report(p.status, KVM_ERR_TIMEOUT);
      *abort_flag = 1;
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, Cfg::TMEM_COLS);
  }
}

// Units that several CTAs shared: out = sum_z 2^(m_z - m) O_z / sum_z 2^(m_z - m) l_z.  One block per unit; thread = channel.
template <int D, int NC>
__global__ void __launch_bounds__(128) combine_kernel(const __grid_constant__ DecodeArgs8 args) {
  const AttendArgs& a = args.a;
  const Params& p = a.p;
  __shared__ int s_sum[2][4];
  const int b = blockIdx.x / p.Hkv, hk = blockIdx.x % p.Hkv, tid = threadIdx.x;
  int total = 0, before = 0, nt = 0, start = 0, n = 0;
  for (int i = tid; i < p.batch; i += 128) {
    int st, cn;
    const int x = seq_lengths(p, i, st, cn) ? seq_tiles(a, st, cn) * p.Hkv : 0;
    total += x;
    if (i < b) before += x;
  }
  total = __reduce_add_sync(0xffffffffu, total);
  before = __reduce_add_sync(0xffffffffu, before);
  if ((tid & 31) == 0) { s_sum[0][tid >> 5] = total; s_sum[1][tid >> 5] = before; }
  if (seq_lengths(p, b, start, n)) nt = seq_tiles(a, start, n);
  __syncthreads();
  if (nt == 0) return;
  total = s_sum[0][0] + s_sum[0][1] + s_sum[0][2] + s_sum[0][3];
  const int u0 = s_sum[1][0] + s_sum[1][1] + s_sum[1][2] + s_sum[1][3] + hk * nt;
  const int share = (total + args.grid - 1) / args.grid;
  const int z0 = u0 / share, z1 = (u0 + nt - 1) / share;
  if (z0 == z1 || tid >= D) return;
  const int64_t stride = 2 * NC * (D + 2);
  // the first CTA's share begins with the unit (slot 1), those of the others in its middle (slot 0)
  for (int c = 0; c < n * a.G; ++c) {
    const float* first = a.part + z0 * stride + (NC + c) * (D + 2);
    const float* rest = a.part + c * (D + 2);
    float m = first[D];
    for (int z = z0 + 1; z <= z1; ++z) m = fmaxf(m, rest[z * stride + D]);
    const float w0 = first[D] == -INFINITY ? 0.f : exp2f(first[D] - m);
    float o = first[tid] * w0, l = first[D + 1] * w0;
    for (int z = z0 + 1; z <= z1; ++z) {
      const float* r = rest + z * stride;
      const float w = r[D] == -INFINITY ? 0.f : exp2f(r[D] - m);
      o = fmaf(r[tid], w, o);
      l = fmaf(r[D + 1], w, l);
    }
    const int t = c / a.G, hq = hk * a.G + c - t * a.G;
    a.out[b * a.so[0] + hq * a.so[1] + t * a.so[2] + tid] = __float2bfloat16_rn(o / l);
  }
}

// At most so many CTAs have tiles: `units` units of at most `tiles` tiles each.
int decode_grid(int64_t units, int64_t tiles) { return (int)std::min<int64_t>(kCtas, units * tiles); }

int64_t decode_workspace(int64_t units, int64_t tiles, int d, int cols) {
  return (int64_t)decode_grid(units, tiles) * 2 * (cols <= 8 ? 8 : 16) * (d + 2) * 4;
}

template <int D, int NC>
kvm_status_t launch_decode_nc(const DecodeArgs8& args, const CUtensorMap& mapK, const CUtensorMap& mapV, cudaStream_t s) {
  using Cfg = DecodeCfg<D, NC>;
  const int smem = Cfg::OFF_SEQ + args.a.p.batch * 8 + (args.a.p.batch + 1) * 4 + 1024;
  static std::atomic<uint64_t> ready{0};   // devices on which the limit has been raised
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
  if (dev > 63 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
    constexpr int most = Cfg::OFF_SEQ + kMaxBatch * 12 + 4 + 1024;
    if (cudaFuncSetAttribute(decode_kernel<D, NC>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) { cudaGetLastError(); return KVM_ERR_CUDA; }
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  decode_kernel<D, NC><<<args.grid, 256, smem, s>>>(mapK, mapV, args);
  combine_kernel<D, NC><<<args.a.p.batch * args.a.p.Hkv, 128, 0, s>>>(args);
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}

kvm_status_t launch_decode8(const AttendArgs& a, int64_t tiles, bool q_vec, cudaStream_t s) {
  DecodeArgs8 args;
  args.a = a;
  args.grid = decode_grid((int64_t)a.p.batch * a.p.Hkv, tiles);
  args.q_vec = q_vec ? 1 : 0;
  CUtensorMap mapK, mapV;
  const int64_t rows = a.p.n_pages * a.p.Hkv * a.p.page;
  if (!encode_tmap_codes(&mapK, a.p.k, a.d, rows, a.p.page) || !encode_tmap_codes(&mapV, a.p.v, a.d, rows, a.p.page)) return KVM_ERR_CUDA;
  const bool few = a.p.T * a.G <= 8;
  if (a.d == 128) return few ? launch_decode_nc<128, 8>(args, mapK, mapV, s) : launch_decode_nc<128, 16>(args, mapK, mapV, s);
  return few ? launch_decode_nc<64, 8>(args, mapK, mapV, s) : launch_decode_nc<64, 16>(args, mapK, mapV, s);
}

}  // namespace cache
}  // namespace kvm
