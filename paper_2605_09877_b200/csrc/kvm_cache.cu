// A cache of keys and values in 8 bits (e4m3 codes, one power-of-two scale per page and head): append, copies of pages, and the entry
// points of the operators over it.
//
// Append.  For the rows that a call adds to a block: e = max(e of the rows held, least e >= -64 with max |x| <= 448 * 2^e), codes
// x / 2^e to nearest even.  A scale that is a power of two makes x / 2^e exact, so a code is rounded once, and costs e4m3 nothing: its
// relative step does not depend on the scale.  2^e over a bf16 maximum (1 + M/128) * 2^(E-127): 448 = 1.75 * 2^8, so e = E - 135, and one
// more when M > 96.  One thread block per (block of tokens, head, k or v): every new row is read once into registers (16 bytes per
// thread and load, all loads in flight together), the maximum is taken on the bit patterns, and the codes are written from the registers.
// Reads 2 bytes and writes 1 per element: bound by HBM for prompts (4 x 8192 tokens, 32 heads, d = 128: 143 us, 5.6 TB/s, 86 % of the measured
// copy rate), by one chain of dependent loads (lengths, page, rows) for single tokens (64 sequences, 8 heads: 6 us on the GPU).
#include <algorithm>
#include <atomic>
#include <new>
#include <vector>

#include "kvm_cache.cuh"
#include "kvm_internal.h"
#include "tc_common.cuh"

namespace kvm {
namespace cache {

constexpr int kLeastExp = -64;

struct AppendArgs {
  Params p;
  uint8_t* codes[2];
  float* scales[2];
  const __nv_bfloat16* x[2];
  int64_t st[2][3];
  int vec;   // rows are 16-byte aligned
};

// 256 threads, TPP of them per page with CH pieces of 8 channels each: 256 / TPP pages per block, so that blocks of small pages do not
// spend their time on their chain of loads (16 x 64: 10.2 -> 8.4 us a call for 7 prompts of 1777 tokens and 5 heads).
template <int D, int TPP, int CH>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs a) {
  constexpr int CPR = D / 8;   // pieces of a row
  const Params& p = a.p;
  const int which = blockIdx.y & 1, hk = blockIdx.y >> 1, b = blockIdx.z, t = threadIdx.x % TPP;
  int start, n;
  const bool valid = seq_lengths(p, b, start, n);
  if (!valid) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) report(p.status, KVM_ERR_INVALID_ARG);
    return;
  }
  const int block = (start >> p.page_shift) + blockIdx.x * (256 / TPP) + threadIdx.x / TPP;
  const int64_t pos0 = (int64_t)block << p.page_shift;                         // position of the page's first row
  const int r0 = (int)max((int64_t)0, start - pos0);                           // rows [0, r0) are held, [r0, r1) are new
  int r1 = (int)max((int64_t)0, min((int64_t)p.page, (int64_t)start + n - pos0));
  int page = 0;
  if (r1 > r0) {
    page = p.pages[(int64_t)b * p.max_pages + block];
    if (page < 0 || page >= p.n_pages) {
      if (t == 0) report(p.status, KVM_ERR_INVALID_ARG);
      r1 = 0;
    }
  }
  const bool live = r1 > r0;
  const int64_t unit = (int64_t)page * p.Hkv + hk;
  uint8_t* codes = a.codes[which] + unit * p.page * D;
  float* scale = a.scales[which] + unit;
  const float old = live && r0 > 0 ? *scale : 0.f;
  const __nv_bfloat16* x = a.x[which] + b * a.st[which][0] + hk * a.st[which][1];
  const int64_t row_stride = a.st[which][2];
  uint4 raw[CH];
  uint32_t top2 = 0;   // largest |x| as bit patterns, two lanes of 16 bits
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int item = t + i * TPP, row = item / CPR, c = item % CPR;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (row >= r0 && row < r1) {
      const __nv_bfloat16* src = x + (pos0 + row - start) * row_stride + c * 8;
      if (a.vec) {
        raw[i] = __ldcs(reinterpret_cast<const uint4*>(src));
      } else {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          w[q] = (uint32_t)__bfloat16_as_ushort(src[2 * q]) | ((uint32_t)__bfloat16_as_ushort(src[2 * q + 1]) << 16);
        raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int q = 0; q < 4; ++q) top2 = __vmaxu2(top2, w[q] & 0x7fff7fffu);
  }
  uint32_t top = max(top2 & 0xffffu, top2 >> 16);
  top = __reduce_max_sync(0xffffffffu, top);
  if (TPP > 32) {
    __shared__ uint32_t s_top[8];
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) s_top[warp] = top;
    __syncthreads();
    const int w0 = warp / (TPP / 32) * (TPP / 32);
#pragma unroll
    for (int w = 0; w < TPP / 32; ++w) top = max(top, s_top[w0 + w]);
  } else {
    __syncwarp();   // (every lane has read the old scale before lane 0 writes the new one: the reduction above promises no order of memory)
  }
  if (!live) return;
  const int e_old = r0 > 0 ? max(scale_exp(old), kLeastExp) : kLeastExp;
  const bool poisoned = top >= 0x7f80u || e_old > 127;
  int e = max((int)(top >> 7) - 135 + ((top & 0x7fu) > 96u ? 1 : 0), kLeastExp);
  e = max(e, e_old);
  if (t == 0) *scale = poisoned ? __int_as_float(0x7fc00000) : exp2i(e);
  const float inv = poisoned ? 0.f : exp2i(-e);
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int item = t + i * TPP, row = item / CPR, c = item % CPR;
    if (row >= r1) continue;
    uint2* dst = reinterpret_cast<uint2*>(codes + (int64_t)row * D + c * 8);
    uint32_t o[2] = {0, 0};
    if (row >= r0) {
      if (!poisoned) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float lo = __uint_as_float(w[q] << 16) * inv, hi = __uint_as_float(w[q] & 0xffff0000u) * inv;
          o[q >> 1] |= to_e4m3x2(lo, hi) << (16 * (q & 1));
        }
      }
      *dst = make_uint2(o[0], o[1]);
    } else if (e > e_old && !poisoned) {
      const float f = e - e_old > 126 ? 0.f : exp2i(e_old - e);   // (codes are at most 448: below 2^-126 of it nothing is left)
      const uint2 held = *dst;
      const uint32_t w[2] = {held.x, held.y};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 x2 = e4m3x2_to_float2((w[q >> 1] >> (16 * (q & 1))) & 0xffffu);
        o[q >> 1] |= to_e4m3x2(x2.x * f, x2.y * f) << (16 * (q & 1));
      }
      *dst = make_uint2(o[0], o[1]);
    }
  }
}

template <int D, int TPP, int CH>
void launch_append_pages(const AppendArgs& a, cudaStream_t s) {
  const int64_t blocks = (a.p.T + a.p.page - 2) / a.p.page + 1;   // blocks that T consecutive tokens can touch
  append_kernel<D, TPP, CH><<<dim3((unsigned)((blocks + 256 / TPP - 1) / (256 / TPP)), 2 * a.p.Hkv, a.p.batch), 256, 0, s>>>(a);
}
template <int D>
void launch_append(const AppendArgs& a, cudaStream_t s) {
  switch (a.p.page * D / 8) {   // pieces of a page
    case 128: launch_append_pages<D, 32, 4>(a, s); break;
    case 256: launch_append_pages<D, 64, 4>(a, s); break;
    case 512: launch_append_pages<D, 128, 4>(a, s); break;
    case 1024: launch_append_pages<D, 256, 4>(a, s); break;
    default: launch_append_pages<D, 256, 8>(a, s); break;
  }
}

// Copies of pages: (source, destination) pairs in the launch's arguments.  Block (pair, part): a run of kCopyPart bytes of the pair's keys or
// values, all loads of a thread in flight before its first store; part 0 moves the scales too.  How many bytes of arguments, measured with 1, 4,
// 8, 16 and 32 KB, the last of which is all that a launch may have, in us between calls that follow one another on the GPU:
//   48 pages of 64 x 128, 8 heads: 4.2  4.2  4.2  4.2  5.9;   400: 23.1  14.5  14.5  14.5  14.7;   2500: 172  122  113  110  106;
//   48 pages of 16 x 64, 1 head:   4.1  4.2  4.2  3.5  5.8;   400: 16.3   4.2   4.2   3.7   6.9;   2500:  86  20.6  12.4  10.4  7.4
// and on the host a call of 1 to 120 pairs takes 3.5 to 4.1 us with 1 KB, 4.6 to 5.0 with 16: the arguments are copied whole.  So a list that 1 KB
// holds has a launch of its own kind, and others go 16 KB at a time.  20000 pages of 64 x 128, 8 heads: 850 us, 6.2 TB/s (94 % of the
// measured copy rate).
constexpr int kCopyPart = 256 * 16 * 4;
template <int BYTES>
struct CopyArgs {
  static constexpr int kPairs = (BYTES - 48) / 8;
  uint8_t* codes[2];
  float* scales[2];
  int64_t page_bytes;   // codes of one page, all heads
  int Hkv;
  int32_t src[kPairs], dst[kPairs];
};
template <int BYTES>
__global__ void __launch_bounds__(256) copy_pages_kernel(const __grid_constant__ CopyArgs<BYTES> a) {
  const int64_t src = a.src[blockIdx.x], dst = a.dst[blockIdx.x];
  const int which = blockIdx.z;
  const uint8_t* from = a.codes[which] + src * a.page_bytes;
  uint8_t* to = a.codes[which] + dst * a.page_bytes;
  const int64_t base = (int64_t)blockIdx.y * kCopyPart + threadIdx.x * 16;
  uint4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (base + i * 4096 < a.page_bytes) x[i] = __ldcs(reinterpret_cast<const uint4*>(from + base + i * 4096));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (base + i * 4096 < a.page_bytes) __stcs(reinterpret_cast<uint4*>(to + base + i * 4096), x[i]);
  if (blockIdx.y == 0)
    for (int h = threadIdx.x; h < a.Hkv; h += 256) a.scales[which][dst * a.Hkv + h] = a.scales[which][src * a.Hkv + h];
}

// Codes as rows of d bytes, a box of one page of one head; rows land swizzled as the tensor core reads them (128 or 64 bytes).
bool encode_tmap_codes(CUtensorMap* map, const void* base, int d, int64_t rows, int page) {
  typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                               const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                               CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static std::atomic<void*> fn{nullptr};
  void* f = fn.load(std::memory_order_acquire);
  if (!f) {
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &qres) != cudaSuccess || !f) {
      cudaGetLastError();
      return false;
    }
    fn.store(f, std::memory_order_release);
  }
  const cuuint64_t gdim[2] = {(cuuint64_t)d, (cuuint64_t)rows}, gstr[1] = {(cuuint64_t)d};
  const cuuint32_t box[2] = {(cuuint32_t)d, (cuuint32_t)page}, estr[2] = {1, 1};
  return reinterpret_cast<EncodeFn>(f)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), gdim, gstr, box, estr,
                                       CU_TENSOR_MAP_INTERLEAVE_NONE, d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BYTES>
static void launch_copies(const kvm_cache_t* cache, const int32_t* src, const int32_t* dst, int64_t n, int64_t page_bytes, cudaStream_t s) {
  using Args = CopyArgs<BYTES>;
  static_assert(sizeof(Args) <= BYTES, "arguments of a launch");
  Args a;
  a.codes[0] = (uint8_t*)cache->k; a.codes[1] = (uint8_t*)cache->v;
  a.scales[0] = cache->k_scale; a.scales[1] = cache->v_scale;
  a.Hkv = cache->n_kv_heads;
  a.page_bytes = page_bytes;
  const unsigned parts = (unsigned)((page_bytes + kCopyPart - 1) / kCopyPart);
  for (int64_t at = 0; at < n; at += Args::kPairs) {
    const int m = (int)std::min<int64_t>(Args::kPairs, n - at);
    std::copy(src + at, src + at + m, a.src);
    std::copy(dst + at, dst + at + m, a.dst);
    copy_pages_kernel<BYTES><<<dim3(m, parts, 2), 256, 0, s>>>(a);
  }
}

// ---- arguments ----

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

kvm_status_t check_cache(const kvm_cache_t* c, bool pointers) {
  if (!c || c->n_pages < 1 || c->n_kv_heads < 1) return KVM_ERR_INVALID_ARG;
  if (pointers) {
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return KVM_ERR_INVALID_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return KVM_ERR_INVALID_ARG;
  }
  if (c->head_dim != 64 && c->head_dim != 128) return KVM_ERR_UNSUPPORTED;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return KVM_ERR_UNSUPPORTED;
  // rows of the pool are numbered in 32 bits, heads in a grid dimension
  if (c->n_kv_heads > 16384 || c->n_pages > INT32_MAX || c->n_pages * c->n_kv_heads > INT32_MAX / c->page_tokens) return KVM_ERR_UNSUPPORTED;
  return KVM_OK;
}

kvm_status_t check_call(const kvm_cache_t* c, const kvm_cache_call_t* call, bool pointers) {
  if (!call || call->batch < 1 || call->max_pages < 1 || call->n_tokens < 1) return KVM_ERR_INVALID_ARG;
  if (pointers) {
    if (!call->pages || !call->start) return KVM_ERR_INVALID_ARG;
    if (!aligned(call->pages, 4) || !aligned(call->start, 4) || !aligned(call->count, 4)) return KVM_ERR_INVALID_ARG;
  }
  const int64_t room = (int64_t)call->max_pages * c->page_tokens;   // positions are 32-bit numbers
  if (call->n_tokens > room && !call->count) return KVM_ERR_INVALID_ARG;   // (with counts, n_tokens is only the padded extent)
  if (call->batch > kMaxBatch || room > (1 << 30) || call->n_tokens > (1 << 30)) return KVM_ERR_UNSUPPORTED;
  return KVM_OK;
}

int64_t tiles_most(const kvm_cache_t* c, const kvm_cache_call_t* call) { return ((int64_t)call->max_pages * c->page_tokens + kTile - 1) / kTile; }

// Whether what attention numbers in 32 bits fits: key tiles of the call, rows of queries of a unit, row tiles of the call.
bool attend_fits(const kvm_cache_t* c, const kvm_cache_call_t* call, int32_t n_q_heads) {
  const int64_t units = (int64_t)call->batch * c->n_kv_heads, rows = call->n_tokens * (n_q_heads / c->n_kv_heads);
  return tiles_most(c, call) * units <= INT32_MAX / 2 && rows <= INT32_MAX - 128 && (rows + 127) / 128 * units <= INT32_MAX;
}

Params params_of(const kvm_cache_t* c, const kvm_cache_call_t* call, int32_t* status) {
  Params p;
  p.k = (const uint8_t*)c->k; p.v = (const uint8_t*)c->v; p.ks = c->k_scale; p.vs = c->v_scale;
  p.pages = call->pages; p.start = call->start; p.count = call->count; p.status = status;
  p.n_pages = c->n_pages; p.T = call->n_tokens;
  p.Hkv = c->n_kv_heads; p.page = c->page_tokens; p.batch = call->batch; p.max_pages = call->max_pages;
  p.page_shift = c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7;
  return p;
}

// Strides of [batch, heads, tokens, d] (NULL: contiguous).  Rows that are written must not lie on one another: each dimension, in the order of
// the strides, has to step over all that the smaller ones span.
bool strides_of(const int64_t* st, int64_t B, int64_t H, int64_t T, int d, bool written, int64_t (&out)[3]) {
  if (!st) { out[0] = H * T * d; out[1] = T * d; out[2] = d; return true; }
  const int64_t n[3] = {B, H, T};
  int by[3] = {0, 1, 2};
  std::sort(by, by + 3, [&](int i, int j) { return st[i] < st[j]; });
  __int128 span = d;   // channels from the first to the last of the rows so far
  for (int i : by) {
    out[i] = st[i];
    if (st[i] < 0 || (written && n[i] > 1 && st[i] < span)) return false;
    if (n[i] > 1) span += (__int128)(n[i] - 1) * st[i];
  }
  return true;
}
bool rows_aligned(const void* p, const int64_t (&st)[3]) {
  return aligned(p, 16) && st[0] % 8 == 0 && st[1] % 8 == 0 && st[2] % 8 == 0;
}

}  // namespace cache
}  // namespace kvm

using namespace kvm;
using namespace kvm::cache;

#define KVM_API __attribute__((visibility("default")))

extern "C" {

KVM_API kvm_status_t kvm_cache_append(const kvm_cache_t* cache, const kvm_cache_call_t* call, const void* k, const void* v,
                                      const int64_t* k_strides, const int64_t* v_strides, int32_t* status, void* cuda_stream) {
  kvm_status_t rc = check_cache(cache, true);
  if (rc == KVM_OK) rc = check_call(cache, call, true);
  if (rc != KVM_OK) return rc;
  if (!k || !v || !aligned(k, 2) || !aligned(v, 2) || !aligned(status, 4)) return KVM_ERR_INVALID_ARG;
  AppendArgs a;
  a.p = params_of(cache, call, status);
  a.codes[0] = (uint8_t*)cache->k; a.codes[1] = (uint8_t*)cache->v;
  a.scales[0] = cache->k_scale; a.scales[1] = cache->v_scale;
  a.x[0] = (const __nv_bfloat16*)k; a.x[1] = (const __nv_bfloat16*)v;
  if (!strides_of(k_strides, a.p.batch, a.p.Hkv, a.p.T, cache->head_dim, false, a.st[0]) ||
      !strides_of(v_strides, a.p.batch, a.p.Hkv, a.p.T, cache->head_dim, false, a.st[1])) return KVM_ERR_INVALID_ARG;
  a.vec = rows_aligned(k, a.st[0]) && rows_aligned(v, a.st[1]) ? 1 : 0;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  if (cache->head_dim == 128) launch_append<128>(a, s); else launch_append<64>(a, s);
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}

KVM_API kvm_status_t kvm_cache_copy_pages(const kvm_cache_t* cache, const int32_t* src, const int32_t* dst, int64_t n, void* cuda_stream) {
  const kvm_status_t rc = check_cache(cache, true);
  if (rc != KVM_OK) return rc;
  if (n < 0 || (n > 0 && (!src || !dst))) return KVM_ERR_INVALID_ARG;
  if (n == 0) return KVM_OK;
  if (n > cache->n_pages) return KVM_ERR_INVALID_ARG;   // (some dst is named twice)
  // every dst once, no dst a src: an open-addressed table of the dsts
  try {
    size_t size = 64;
    while (size < (size_t)n * 2) size *= 2;
    std::vector<int32_t> table(size, -1);
    auto slot = [&](int32_t x) {
      size_t at = ((uint32_t)x * 2654435761u >> 7) & (size - 1);
      while (table[at] != -1 && table[at] != x) at = (at + 1) & (size - 1);
      return at;
    };
    for (int64_t i = 0; i < n; ++i) {
      if (src[i] < 0 || src[i] >= cache->n_pages || dst[i] < 0 || dst[i] >= cache->n_pages) return KVM_ERR_INVALID_ARG;
      const size_t at = slot(dst[i]);
      if (table[at] != -1) return KVM_ERR_INVALID_ARG;
      table[at] = dst[i];
    }
    for (int64_t i = 0; i < n; ++i)
      if (table[slot(src[i])] != -1) return KVM_ERR_INVALID_ARG;
  } catch (const std::bad_alloc&) {
    return KVM_ERR_OOM;
  }
  const int64_t page_bytes = (int64_t)cache->n_kv_heads * cache->page_tokens * cache->head_dim;
  if ((page_bytes + kCopyPart - 1) / kCopyPart > 65535) return KVM_ERR_UNSUPPORTED;
  if (n <= CopyArgs<1024>::kPairs) launch_copies<1024>(cache, src, dst, n, page_bytes, (cudaStream_t)cuda_stream);
  else launch_copies<16384>(cache, src, dst, n, page_bytes, (cudaStream_t)cuda_stream);
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}

KVM_API int64_t kvm_cache_workspace(const kvm_cache_t* cache, const kvm_cache_call_t* call, int32_t n_q_heads) {
  if (check_cache(cache, false) != KVM_OK || check_call(cache, call, false) != KVM_OK) return -1;
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads || !attend_fits(cache, call, n_q_heads)) return -1;
  const int64_t units = (int64_t)call->batch * cache->n_kv_heads, tiles = tiles_most(cache, call);
  const int64_t cols = call->n_tokens * (n_q_heads / cache->n_kv_heads);
  return cols <= kDecodeCols ? decode_workspace(units, tiles, cache->head_dim, (int)cols) : prompt_workspace(units, cols, tiles, cache->head_dim);
}

KVM_API kvm_status_t kvm_cache_attend(const kvm_cache_t* cache, const kvm_cache_call_t* call, const void* q, int32_t n_q_heads, float scale,
                                      int32_t window, int32_t sinks, void* out, const int64_t* q_strides, const int64_t* out_strides,
                                      void* workspace, int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  kvm_status_t rc = check_cache(cache, true);
  if (rc == KVM_OK) rc = check_call(cache, call, true);
  if (rc != KVM_OK) return rc;
  if (!q || !out || !aligned(q, 2) || !aligned(out, 2) || !aligned(status, 4)) return KVM_ERR_INVALID_ARG;
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads || window < 0 || sinks < 0) return KVM_ERR_INVALID_ARG;
  if (!(scale > 0.f) || scale > 3.0e38f) return KVM_ERR_INVALID_ARG;   // (a NaN is refused too)
  AttendArgs a;
  a.p = params_of(cache, call, status);
  a.q = (const __nv_bfloat16*)q; a.out = (__nv_bfloat16*)out;
  if (!strides_of(q_strides, a.p.batch, n_q_heads, a.p.T, cache->head_dim, false, a.sq) ||
      !strides_of(out_strides, a.p.batch, n_q_heads, a.p.T, cache->head_dim, true, a.so)) return KVM_ERR_INVALID_ARG;
  a.Hq = n_q_heads; a.G = n_q_heads / cache->n_kv_heads; a.d = cache->head_dim;
  a.window = window ? window : INT32_MAX; a.sinks = std::min(sinks, 1 << 30);
  if (!attend_fits(cache, call, n_q_heads)) return KVM_ERR_UNSUPPORTED;
  const int64_t tiles = tiles_most(cache, call);
  a.scale_log2 = scale * 1.4426950408889634f;
  const int64_t need = kvm_cache_workspace(cache, call, n_q_heads);
  if (need < 0) return KVM_ERR_UNSUPPORTED;
  if (need > 0 && (!workspace || !aligned(workspace, 16))) return KVM_ERR_INVALID_ARG;
  if (workspace_bytes < need) return KVM_ERR_CAPACITY;
  a.part = (float*)workspace;
  if (a.p.T * a.G <= kDecodeCols) return launch_decode8(a, tiles, rows_aligned(q, a.sq), (cudaStream_t)cuda_stream);
  return launch_prompt8(a, tiles, rows_aligned(q, a.sq), rows_aligned(out, a.so), (cudaStream_t)cuda_stream);
}

}  // extern "C"
