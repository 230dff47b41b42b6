// Quantising keys and values into the 8-bit cache, and reading them back.
//
// A scale group is T consecutive tokens of one head (bs_quant.h). With
// a = max(max |x| over the group, 2^-64) and Q the largest number of the format
// (448 for e4m3, 127 for int8):
//   scale = a / Q,   code = x * (Q / a) rounded to nearest even.
// Both quotients are rounded once, in fp32; the product is the only other
// rounding before the code's own.
//
// Both directions are bound by HBM: each element is read once and written
// once.
#include "bs_quant.h"

namespace bs {
namespace {

// One wave quantises RS * RP tokens (a multiple of T) of one head of K or V, a lane as
// many features as fill 16 bytes, so that its loads are whole lines.
template <typename E, int FMT, int D, int RP>
__global__ __launch_bounds__(256) void k_kv_quantize(QuantArgs a) {
  constexpr int F = 16 / sizeof(E);   // features per lane
  constexpr int GS = D / F;           // lanes per token
  constexpr int RS = 64 / GS;         // tokens per step
  constexpr int CT = RS * RP;         // tokens per wave
  const bs_req_desc r = a.reqs.get(blockIdx.y);
  const int h = blockIdx.z >> 1, tensor = blockIdx.z & 1;
  const int lane = threadIdx.x & 63, T = 1 << a.lt;
  const int pad = group_pad(r.p, a.lt), len = r.p + r.g;
  // virtual token v = t + pad: group v >> lt
  const int v0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * CT;
  if (v0 >= len + pad) return;
  const int64_t cell0 = (((int64_t)r.row * a.Hkv + h) * a.W + r.off) * D + (lane % GS) * F;
  const E* src = static_cast<const E*>(tensor ? a.v : a.k) + cell0;

  v4u x[RP];
  float top[RP];
#pragma unroll
  for (int i = 0; i < RP; ++i) {
    const int t = v0 + i * RS + lane / GS - pad;
    x[i] = v4u{0, 0, 0, 0};           // a token outside the row: no maximum, and not stored
    if (t >= 0 && t < len) x[i] = ld16(src + (int64_t)t * D);
  }
  auto get = [&](int i, int e) {
    if constexpr (F == 8)
      return e & 1 ? bf_hi(x[i][e >> 1]) : bf_lo(x[i][e >> 1]);
    else
      return __uint_as_float(x[i][e]);
  };
#pragma unroll
  for (int i = 0; i < RP; ++i) {
    top[i] = 0.0f;
#pragma unroll
    for (int e = 0; e < F; ++e) top[i] = fmaxf(top[i], fabsf(get(i, e)));
  }
  group_tops<GS>(top, a.lt);
  uint8_t* codes = (tensor ? a.v8 : a.k8) + cell0;
  float* scales = (tensor ? a.v_scale : a.k_scale) + ((int64_t)r.row * a.Hkv + h) * a.S;
#pragma unroll
  for (int i = 0; i < RP; ++i) {
    const int v = v0 + i * RS + lane / GS, t = v - pad;
    const float m = fmaxf(top[i], kQuantFloor);
    if (lane % GS == 0 && (v & (T - 1)) == 0 && v < len + pad) scales[v >> a.lt] = m / quant_max<FMT>();
    if (t < 0 || t >= len) continue;
    uint32_t w[F / 4];
    encode<FMT, F / 4>(m, [&](int e) { return get(i, e); }, w);
    if constexpr (F == 8)
      *reinterpret_cast<uint2*>(codes + (int64_t)t * D) = uint2{w[0], w[1]};
    else
      *reinterpret_cast<uint32_t*>(codes + (int64_t)t * D) = w[0];
  }
}

// Thread: as many codes of a token as fill 16 bytes read back, so that a wave's stores
// are whole lines (16 codes a thread, stores of every other 16 bytes: 97 us instead of
// 87 for 32 LLaDA-8B rows; two or four tokens a thread as well: 115).
template <typename E, int FMT, int D>
__global__ __launch_bounds__(256) void k_kv_dequantize(DequantArgs a) {
  constexpr int F = 16 / sizeof(E), GS = D / F;       // features per lane, lanes per token
  const bs_req_desc r = a.reqs.get(blockIdx.y);
  const int h = blockIdx.z >> 1, tensor = blockIdx.z & 1;
  const int u = blockIdx.x * 256 + threadIdx.x;
  const int t = u / GS;
  if (t >= r.p + r.g) return;
  const int64_t row_head = (int64_t)r.row * a.Hkv + h, cell = (row_head * a.W + r.off + t) * D + u % GS * F;
  const float sc = (tensor ? a.v_scale : a.k_scale)[row_head * a.S + ((t + group_pad(r.p, a.lt)) >> a.lt)];
  const uint8_t* codes = (tensor ? a.v8 : a.k8) + cell;
  uint32_t w[F / 4];
  if constexpr (F == 8) {
    const uint2 x = *reinterpret_cast<const uint2*>(codes);
    w[0] = x.x;
    w[1] = x.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(codes);
  }
  float y[F];
#pragma unroll
  for (int k = 0; k < F / 4; ++k) {
    float z[4];
    decode4<FMT>(w[k], z);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[4 * k + e] = z[e] * sc;
  }
  v4u o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = F == 8 ? pack_bf16(y[2 * e % F], y[(2 * e + 1) % F]) : __float_as_uint(y[e]);
  st16(static_cast<E*>(tensor ? a.v : a.k) + cell, o);
}

template <typename E, int FMT, int D>
void quantize(const QuantArgs& a, int n, int max_len, hipStream_t s) {
  constexpr int RS = 64 / (D * (int)sizeof(E) / 16);
  const int T = 1 << a.lt;
  auto go = [&](auto kernel, int rp) {
    const int per = 4 * RS * rp;    // tokens per workgroup
    const dim3 grid((unsigned)((max_len + T - 1 + per - 1) / per), (unsigned)n, (unsigned)(2 * a.Hkv));
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
  };
  // eight loads in flight a lane, more where a group needs them
  if (T > 16 * RS)
    go(k_kv_quantize<E, FMT, D, 32>, 32);
  else if (T > 8 * RS)
    go(k_kv_quantize<E, FMT, D, 16>, 16);
  else
    go(k_kv_quantize<E, FMT, D, 8>, 8);
}

template <typename E, int FMT, int D>
void dequantize(const DequantArgs& a, int n, int max_len, hipStream_t s) {
  const int64_t lanes = (int64_t)max_len * (D * sizeof(E) / 16);
  const dim3 grid((unsigned)((lanes + 255) / 256), (unsigned)n, (unsigned)(2 * a.Hkv));
  hipLaunchKernelGGL((k_kv_dequantize<E, FMT, D>), grid, dim3(256), 0, s, a);
}

// f(E{}, format, D) with the three as compile-time values
template <class F>
void dispatch(bs_dtype dt, bs_qformat fmt, int D, F f) {
  auto by_d = [&](auto e, auto m) { D == 64 ? f(e, m, QInt<64>{}) : f(e, m, QInt<128>{}); };
  auto by_f = [&](auto e) { fmt == BS_E4M3 ? by_d(e, QInt<BS_E4M3>{}) : by_d(e, QInt<BS_I8>{}); };
  dt == BS_BF16 ? by_f(uint16_t{}) : by_f(float{});
}

}  // namespace

hipError_t launch_kv_quantize(const QuantArgs& a, bs_dtype dt, bs_qformat fmt, int D, int n, int max_len,
                              hipStream_t s) {
  dispatch(dt, fmt, D, [&](auto e, auto m, auto d) {
    quantize<decltype(e), decltype(m)::value, decltype(d)::value>(a, n, max_len, s);
  });
  return hipGetLastError();
}

hipError_t launch_kv_dequantize(const DequantArgs& a, bs_dtype dt, bs_qformat fmt, int D, int n, int max_len,
                                hipStream_t s) {
  dispatch(dt, fmt, D, [&](auto e, auto m, auto d) {
    dequantize<decltype(e), decltype(m)::value, decltype(d)::value>(a, n, max_len, s);
  });
  return hipGetLastError();
}

}  // namespace bs
