// Block attention against a dual cache held in 8 bits.
//
// As the attention over the bf16 cache, with key t of the row read as
// code * scale of its group outside the active block, and from k_new / v_new
// inside it. One wave per (request, query head, block row): lane t scores key t
// of each 64-key chunk, the weights are broadcast by lane shuffles for P V.
#include "bs_quant.h"

namespace bs {
namespace {

template <int FMT>
__global__ __launch_bounds__(256) void k_qattn(QAttnArgs a, int jblocks) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int jb = blockIdx.x % jblocks, rest = blockIdx.x / jblocks;
  const int h = rest % a.Hq, i = rest / a.Hq, j = jb * 4 + w;
  if (j >= a.L) return;
  const bs_req_desc r = a.reqs[i];
  const Geo geo = geo_of(r, a.L);
  const int c = h / a.G, D = a.D, pad = group_pad(r.p, a.lt), bs = geo.s, be = geo.s + geo.B;
  uint16_t* op = a.out + (((int64_t)i * a.L + j) * a.Hq + h) * D;
  if (j >= geo.B) {
    for (int d = lane; d < D; d += 64) op[d] = 0;
    return;
  }
  const uint16_t* qp = a.q + (((int64_t)i * a.L + j) * a.Hq + h) * D;
  const int64_t cell = (((int64_t)r.row * a.Hkv + c) * a.W + r.off) * D, sc0 = ((int64_t)r.row * a.Hkv + c) * a.S;
  const int64_t fstride = (int64_t)a.Hkv * D, fresh = ((int64_t)i * a.L * a.Hkv + c) * D;
  float o[2] = {0.0f, 0.0f}, m = -__builtin_inff(), l = 0.0f;
  for (int t0 = 0; t0 < geo.len; t0 += 64) {
    const int t = t0 + lane;
    float s = -__builtin_inff();
    if (t < geo.len) {
      float acc = 0.0f;
      if (t >= bs && t < be) {
        const uint16_t* kp = a.k_new + fresh + (t - bs) * fstride;
        for (int d = 0; d < D; ++d) acc = fmaf(bf_lo(qp[d]), bf_lo(kp[d]), acc);
      } else {
        for (int d = 0; d < D; d += 4) {
          float y[4];
          decode4<FMT>(*reinterpret_cast<const uint32_t*>(a.k8 + cell + (int64_t)t * D + d), y);
          for (int e = 0; e < 4; ++e) acc = fmaf(bf_lo(qp[d + e]), y[e], acc);
        }
        acc *= a.k_scale[sc0 + ((t + pad) >> a.lt)];
      }
      s = acc * a.scale_log2e;
    }
    float mx = s;
    for (int x = 32; x >= 1; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
    const float mn = fmaxf(m, mx), alpha = exp2f(m - mn);
    const float p = t < geo.len ? exp2f(s - mn) : 0.0f;
    float ps = p;
    for (int x = 32; x >= 1; x >>= 1) ps += __shfl_xor(ps, x, 64);
    l = l * alpha + ps;
    o[0] *= alpha;
    o[1] *= alpha;
    m = mn;
    const int nk = min(64, geo.len - t0);
    for (int x = 0; x < nk; ++x) {
      const float pt = __shfl(p, x, 64);
      const int tk = t0 + x;
      for (int u = 0; u < 2; ++u) {
        const int d = lane + 64 * u;
        if (d >= D) continue;
        float v;
        if (tk >= bs && tk < be) {
          v = bf_lo(a.v_new[fresh + (tk - bs) * fstride + d]);
        } else {
          float y[4];
          decode4<FMT>(a.v8[cell + (int64_t)tk * D + d], y);
          v = y[0] * a.v_scale[sc0 + ((tk + pad) >> a.lt)];
        }
        o[u] = fmaf(pt, v, o[u]);
      }
    }
  }
  for (int u = 0; u < 2; ++u)
    if (lane + 64 * u < D) op[lane + 64 * u] = (uint16_t)pack_bf16(o[u] / l, 0.0f);
}

}  // namespace

hipError_t launch_qattn(const QAttnArgs& a, bs_qformat fmt, hipStream_t s) {
  const int jblocks = (a.L + 3) / 4;
  const dim3 grid((unsigned)((int64_t)a.n * a.Hq * jblocks));
  if (fmt == BS_E4M3)
    hipLaunchKernelGGL(k_qattn<BS_E4M3>, grid, dim3(256), 0, s, a, jblocks);
  else
    hipLaunchKernelGGL(k_qattn<BS_I8>, grid, dim3(256), 0, s, a, jblocks);
  return hipGetLastError();
}

}  // namespace bs
