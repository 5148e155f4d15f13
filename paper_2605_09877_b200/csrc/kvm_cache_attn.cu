// Attention over the 8-bit cache, the plainest form: one warp per (sequence, head, token) walks the tiles that the token sees, D / 32
// channels per lane, running maximum and sum.
#include "kvm_cache.cuh"

namespace kvm {
namespace cache {

template <int D>
__global__ void __launch_bounds__(128) attend_rows_kernel(const AttendArgs a) {
  constexpr int E = D / 32;
  const Params& p = a.p;
  const int lane = threadIdx.x & 31, hq = blockIdx.y, b = blockIdx.z;
  const int64_t tok = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  int start, n;
  const bool valid = seq_lengths(p, b, start, n);
  if (!valid) { if (lane == 0) report(p.status, KVM_ERR_INVALID_ARG); n = 0; }
  if (tok >= n) return;
  const int pos = start + (int)tok, hk = hq / a.G;
  float q[E], acc[E];
  const __nv_bfloat16* qr = a.q + b * a.sq[0] + hq * a.sq[1] + tok * a.sq[2] + lane * E;
  for (int e = 0; e < E; ++e) { q[e] = __bfloat162float(qr[e]) * a.scale_log2; acc[e] = 0.f; }
  const Tiles t = tiles_of(pos, pos, a.window, a.sinks);
  float m = -INFINITY, l = 0.f;
  for (int i = 0; i < t.n; ++i) {
    const int base = tile_at(t, i) * kTile;
    for (int j = base; j < base + kTile && j <= pos; ++j) {
      if (!sees(pos, j, a.window, a.sinks)) continue;
      const int page = p.pages[(int64_t)b * p.max_pages + (j >> p.page_shift)];
      float s, vs = __int_as_float(0x7fc00000);
      const uint8_t* vr = nullptr;
      if (page < 0 || page >= p.n_pages) {
        if (lane == 0) report(p.status, KVM_ERR_INVALID_ARG);
        s = vs;
      } else {
        const int64_t unit = (int64_t)page * p.Hkv + hk, row = unit * p.page + (j & (p.page - 1));
        const uint8_t* kr = p.k + row * D + lane * E;
        vr = p.v + row * D + lane * E;
        vs = p.vs[unit];
        s = 0.f;
        for (int e = 0; e < E; ++e) s += q[e] * e4m3x2_to_float2(kr[e]).x;
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        s *= p.ks[unit];
      }
      const float mn = s > m || !(s == s) ? s : m;
      const float f = m == -INFINITY ? 0.f : exp2f(m - mn), w = exp2f(s - mn);
      l = l * f + w;
      for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + w * (vr ? e4m3x2_to_float2(vr[e]).x * vs : vs);
      m = mn;
    }
  }
  __nv_bfloat16* o = a.out + b * a.so[0] + hq * a.so[1] + tok * a.so[2] + lane * E;
  for (int e = 0; e < E; ++e) o[e] = __float2bfloat16_rn(acc[e] / l);
}

kvm_status_t launch_attend_rows(const AttendArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)((a.p.T + 3) / 4), a.Hq, a.p.batch);
  if (a.d == 128) attend_rows_kernel<128><<<grid, 128, 0, s>>>(a); else attend_rows_kernel<64><<<grid, 128, 0, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? KVM_OK : KVM_ERR_CUDA;
}

}  // namespace cache
}  // namespace kvm
