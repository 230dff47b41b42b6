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
// once. A wave takes 64 / (D / 16) tokens at a time, 16 features a lane, so that
// codes are stored and loaded as 16 bytes a lane and a wave's run is contiguous.
#include "bs_quant.h"

namespace bs {
namespace {

// 16 consecutive elements of a lane, held as loaded
template <typename E>
struct Sixteen {
  static constexpr int NV = sizeof(E);   // 16-byte vectors: 2 (bf16) or 4 (fp32)
  v4u x[NV];
  __device__ void load(const E* p) {
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = ld16(reinterpret_cast<const char*>(p) + 16 * i);
  }
  __device__ float get(int e) const {
    if constexpr (sizeof(E) == 2) {
      const uint32_t w = x[e >> 3][(e >> 1) & 3];
      return e & 1 ? bf_hi(w) : bf_lo(w);
    } else {
      return __uint_as_float(x[e >> 2][e & 3]);
    }
  }
};

// One wave quantises RS * RP tokens (a multiple of T) of one head of K or V.
template <typename E, int FMT, int D, int RP>
__global__ __launch_bounds__(256) void k_kv_quantize(QuantArgs a) {
  constexpr int GS = D / 16;        // lanes per token
  constexpr int RS = 64 / GS;       // tokens per step
  constexpr int CT = RS * RP;       // tokens per wave
  const bs_req_desc r = a.reqs[blockIdx.y];
  const int h = blockIdx.z >> 1, tensor = blockIdx.z & 1;
  const int lane = threadIdx.x & 63, T = 1 << a.lt;
  const int pad = group_pad(r.p, a.lt), len = r.p + r.g;
  // virtual token v = t + pad: group v >> lt
  const int v0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * CT;
  if (v0 >= len + pad) return;
  const int64_t cell0 = (((int64_t)r.row * a.Hkv + h) * a.W + r.off) * D + (lane % GS) * 16;
  const E* src = static_cast<const E*>(tensor ? a.v : a.k) + cell0;

  Sixteen<E> x[RP];
  float top[RP];
  bool ok[RP];
#pragma unroll
  for (int i = 0; i < RP; ++i) {
    const int t = v0 + i * RS + lane / GS - pad;
    ok[i] = t >= 0 && t < len;
    if (ok[i]) x[i].load(src + (int64_t)t * D);
  }
#pragma unroll
  for (int i = 0; i < RP; ++i) {
    top[i] = 0.0f;
    if (ok[i]) {
#pragma unroll
      for (int e = 0; e < 16; ++e) top[i] = fmaxf(top[i], fabsf(x[i].get(e)));
    }
  }
  group_tops<GS>(top, a.lt);
  uint8_t* codes = (tensor ? a.v8 : a.k8) + cell0;
  float* scales = (tensor ? a.v_scale : a.k_scale) + ((int64_t)r.row * a.Hkv + h) * a.S;
#pragma unroll
  for (int i = 0; i < RP; ++i) {
    const int v = v0 + i * RS + lane / GS;
    const float m = fmaxf(top[i], kQuantFloor);
    if (lane % GS == 0 && (v & (T - 1)) == 0 && v < len + pad) scales[v >> a.lt] = m / quant_max<FMT>();
    if (ok[i]) st16(codes + (int64_t)(v - pad) * D, encode16<FMT>(m, [&](int e) { return x[i].get(e); }));
  }
}

// Thread: 16 codes of one token.
template <typename E, int FMT, int D>
__global__ __launch_bounds__(256) void k_kv_dequantize(DequantArgs a) {
  constexpr int GS = D / 16;
  const bs_req_desc r = a.reqs[blockIdx.y];
  const int h = blockIdx.z >> 1, tensor = blockIdx.z & 1;
  const int u = blockIdx.x * 256 + threadIdx.x;
  const int t = u / GS, col = (u % GS) * 16;
  if (t >= r.p + r.g) return;
  const int64_t cell = (((int64_t)r.row * a.Hkv + h) * a.W + r.off + t) * D + col;
  const float sc = (tensor ? a.v_scale : a.k_scale)[((int64_t)r.row * a.Hkv + h) * a.S + ((t + group_pad(r.p, a.lt)) >> a.lt)];
  const v4u w = ld16((tensor ? a.v8 : a.k8) + cell);
  E* out = static_cast<E*>(tensor ? a.v : a.k) + cell;
  float y[16];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float z[4];
    decode4<FMT>(w[k], z);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[4 * k + e] = z[e] * sc;
  }
  if constexpr (sizeof(E) == 2) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v4u o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = pack_bf16(y[8 * i + 2 * e], y[8 * i + 2 * e + 1]);
      st16(out + 8 * i, o);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      st16(out + 4 * i, v4u{__float_as_uint(y[4 * i]), __float_as_uint(y[4 * i + 1]), __float_as_uint(y[4 * i + 2]),
                            __float_as_uint(y[4 * i + 3])});
  }
}

template <typename E, int FMT, int D>
void quantize(const QuantArgs& a, int n, int max_len, hipStream_t s) {
  constexpr int RS = 64 / (D / 16);
  const int T = 1 << a.lt;
  auto go = [&](auto kernel, int rp) {
    const int per = 4 * RS * rp;    // tokens per workgroup
    const dim3 grid((unsigned)((max_len + T - 1 + per - 1) / per), (unsigned)n, (unsigned)(2 * a.Hkv));
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
  };
  if (T > 4 * RS)
    go(k_kv_quantize<E, FMT, D, 8>, 8);
  else
    go(k_kv_quantize<E, FMT, D, 4>, 4);
}

template <typename E, int FMT, int D>
void dequantize(const DequantArgs& a, int n, int max_len, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)max_len * (D / 16) + 255) / 256), (unsigned)n, (unsigned)(2 * a.Hkv));
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
