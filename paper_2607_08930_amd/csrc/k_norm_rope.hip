// Per-head norm of queries and keys and their position rotation, in one pass.
//
// For a head row x [D] of a token at position t (norm over the head's own
// features, rotate-half pairing):
//   y = x / sqrt(mean(x^2) + eps) * w
//   (y_f, y_{f + D/2}) -> turned by the angle t * base^(-2 f / D)
// The host passes each pair's turns per position as a high and a low fp32 part.
// t * high is split into its rounded product and the product's error (fma), so
// the fraction of a turn is good to about 2^-24 for any position below 2^24,
// where a single fp32 product is off by position * 2^-24.
//
// HBM-bound: every element is read once and written once. D / 16 lanes own a
// head row; a lane holds 8 features and their 8 partners (one 16-byte load of
// bf16 each), so the pair stays in one lane and the sum of squares needs log2(D
// / 16) exchanges. A lane group walks kHeads heads of one token with the angles
// computed once.
#include "bs_quant.h"

namespace bs {
namespace {

constexpr int kHeads = 4;   // heads of one token per lane group

template <typename E>
__device__ inline void load8(const E* p, float (&y)[8]) {
  if constexpr (sizeof(E) == 2) {
    const v4u w = ld16(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = bf_lo(w[i]);
      y[2 * i + 1] = bf_hi(w[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const v4u w = ld16(p + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[4 * i + e] = __uint_as_float(w[e]);
    }
  }
}

template <typename E>
__device__ inline void store8(E* p, const float (&y)[8]) {
  if constexpr (sizeof(E) == 2) {
    st16(p, v4u{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])});
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      st16(p + 4 * i, v4u{__float_as_uint(y[4 * i]), __float_as_uint(y[4 * i + 1]), __float_as_uint(y[4 * i + 2]),
                          __float_as_uint(y[4 * i + 3])});
  }
}

// GS lanes per head row, of which D / 16 work (GS = D / 16 rounded up to a power of 2)
template <typename E, int GS>
__global__ __launch_bounds__(256) void k_norm_rope(NormRopeArgs a) {
  const bs_req_desc r = a.reqs.get(blockIdx.y);
  const Geo geo = geo_of(r, a.L);
  const int D = a.D, H = a.Hq + a.Hkv, NHC = (H + kHeads - 1) / kHeads;
  const int u = (blockIdx.x * 256 + threadIdx.x) / GS, c = threadIdx.x % GS;
  const int j = u / NHC, h0 = u % NHC * kHeads;
  if (j >= (a.rows ? geo.len : geo.B)) return;   // all lanes of a group alike
  const bool on = c < D / 16;
  const int f0 = on ? 8 * c : 0;
  const int64_t token = a.rows ? (int64_t)r.row * a.W + r.off + j : (int64_t)blockIdx.y * a.L + j;
  const float pos = (float)(a.rows ? j : geo.s + j);
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.0f;
    sn[e] = 0.0f;
    if (a.rope) {
      const float2 fr = a.freq[f0 + e];
      const float p = pos * fr.x;
      const float turns = __builtin_amdgcn_fractf(p) + fmaf(pos, fr.y, fmaf(pos, fr.x, -p));
      if constexpr (sizeof(E) == 2) {
        sn[e] = __builtin_amdgcn_sinf(turns);
        cs[e] = __builtin_amdgcn_cosf(turns);
      } else {
        sincospif(2.0f * turns, &sn[e], &cs[e]);
      }
    }
  }
  for (int h = h0; h < min(h0 + kHeads, H); ++h) {
    const bool key = h >= a.Hq;
    const E* x = key ? static_cast<const E*>(a.k) + token * a.k_stride + (int64_t)(h - a.Hq) * D
                     : static_cast<const E*>(a.q) + token * a.q_stride + (int64_t)h * D;
    E* out = key ? static_cast<E*>(a.k_out) + (token * a.Hkv + (h - a.Hq)) * D
                 : static_cast<E*>(a.q_out) + (token * a.Hq + h) * D;
    const E* w = static_cast<const E*>(key ? a.kw : a.qw);
    float x1[8], x2[8];
    load8(x + f0, x1);
    load8(x + D / 2 + f0, x2);
    if (a.norm) {
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x1[e], x1[e], fmaf(x2[e], x2[e], ss));
      if (!on) ss = 0.0f;
#pragma unroll
      for (int o = 1; o < GS; o <<= 1) ss += __shfl_xor(ss, o, 64);
      const float rs = rsqrtf(ss / (float)D + a.eps);
      float w1[8], w2[8];
      if (w) {
        load8(w + f0, w1);
        load8(w + D / 2 + f0, w2);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x1[e] *= w ? rs * w1[e] : rs;
        x2[e] *= w ? rs * w2[e] : rs;
      }
    }
    float y1[8], y2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y1[e] = x1[e] * cs[e] - x2[e] * sn[e];
      y2[e] = x2[e] * cs[e] + x1[e] * sn[e];
    }
    if (on) {
      store8(out + f0, y1);
      store8(out + D / 2 + f0, y2);
    }
  }
}

template <typename E>
void norm_rope(const NormRopeArgs& a, int n, int max_tokens, hipStream_t s) {
  const int units = (a.Hq + a.Hkv + kHeads - 1) / kHeads;
  auto go = [&](auto kernel, int gs) {
    const dim3 grid((unsigned)(((int64_t)max_tokens * units * gs + 255) / 256), (unsigned)n);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
  };
  const int lanes = a.D / 16;
  if (lanes <= 1)
    go(k_norm_rope<E, 1>, 1);
  else if (lanes <= 2)
    go(k_norm_rope<E, 2>, 2);
  else if (lanes <= 4)
    go(k_norm_rope<E, 4>, 4);
  else if (lanes <= 8)
    go(k_norm_rope<E, 8>, 8);
  else
    go(k_norm_rope<E, 16>, 16);
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs& a, bs_dtype dt, int n, int max_tokens, hipStream_t s) {
  dt == BS_BF16 ? norm_rope<uint16_t>(a, n, max_tokens, s) : norm_rope<float>(a, n, max_tokens, s);
  return hipGetLastError();
}

}  // namespace bs
