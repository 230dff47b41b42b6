// Internal declarations of the operators around a dual cache held in 8 bits:
// per-head norm with the position rotation, quantising and reading back, and
// the block attention over codes and scales.
#pragma once

#include "bs_internal.h"

namespace bs {

// Scale groups of a row: token t of a request with prompt length p belongs to
// group (t + pad) >> lt, pad = -p mod T, T = 1 << lt. The grid starts at the
// first generated token (t = p, a group border) and runs both ways from there,
// so a block of L tokens is whole groups whenever T divides L, whatever p is; only
// the first group of the prompt and the last one of the row can be short.
__host__ __device__ inline int group_pad(int p, int lt) { return (int)(-(unsigned)p & ((1u << lt) - 1u)); }

// Least maximum of a group. Below it (zeros, mostly) the scale stays this
// large, so that neither the scale nor its reciprocal leaves fp32's range.
constexpr float kQuantFloor = 5.421010862427522e-20f;   // 2^-64
constexpr float kE4m3Max = 448.0f, kI8Max = 127.0f;

struct NormRopeArgs {
  const bs_req_desc* reqs;
  const float2* freq;        // [D / 2]: turns per position of feature pair f, as high + low part
  int L, W, Hq, Hkv, D;
  int rows;                  // 0: blocks [n][L], 1: whole rows of the box [R][W]
  int norm, rope;
  float eps;
  const void* q;
  const void* k;
  int64_t q_stride, k_stride;   // elements between tokens
  const void* qw;               // [D] or NULL (ones)
  const void* kw;
  void* q_out;               // [tokens][Hq][D]
  void* k_out;
};
hipError_t launch_norm_rope(const NormRopeArgs& a, bs_dtype dt, int n, int max_tokens, hipStream_t s);

// Quantising: token t of head h of request i is read at
//   box   (block == 0)  src[row_i][h][off_i + t]     t in [0, len_i)
//   block (block == 1)  src[i][t - s_i][h]           t in [s_i, s_i + B_i)
// and written to the cache cell of the box either way.
struct QuantArgs {
  const bs_req_desc* reqs;
  int L, Hkv, W, S, lt;
  int block;
  const void* k;
  const void* v;
  uint8_t* k8;               // [R][Hkv][W][D]
  uint8_t* v8;
  float* k_scale;            // [R][Hkv][S]
  float* v_scale;
};
hipError_t launch_kv_quantize(const QuantArgs& a, bs_dtype dt, bs_qformat fmt, int D, int n, int max_tokens,
                              hipStream_t s);

struct DequantArgs {
  const bs_req_desc* reqs;
  int Hkv, W, S, lt;
  const uint8_t* k8;
  const uint8_t* v8;
  const float* k_scale;
  const float* v_scale;
  void* k;                   // [R][Hkv][W][D]
  void* v;
};
hipError_t launch_kv_dequantize(const DequantArgs& a, bs_dtype dt, bs_qformat fmt, int D, int n, int max_len,
                                hipStream_t s);

// Attention work item: the row tiles of one (request, KV head) that one workgroup
// serves, against the cached keys [v0, v1) of its piece in virtual keys (below) and,
// where `fresh` is set, the block's own keys.
// Virtual keys count the cached keys without the active block from pad = -p mod 64:
// v < s + pad is cell v - pad, v >= s + pad is cell v - pad + B; nv ends them. Groups
// of T <= 64 tokens and 64-key tiles then share borders. v0 and v1 are multiples of
// 64, but for v1 = nv of the last piece.
struct QItem {
  int32_t req, kvh, rt0;     // request, KV head, first row tile
  int32_t row, off, s, B;
  int32_t pad, nv, v0, v1;
  int32_t part;              // partial slot of a split row, or -1
  int32_t fresh;
  int32_t pad_[3];
};

struct QMerge {
  int32_t req, kvh, rt0, B, part0, nparts, pad_[2];
};

constexpr int kQTile = 64;   // virtual keys per planning unit
constexpr int kQRowTiles = 8;   // most 32-row tiles (waves) per workgroup

struct QAttnArgs {
  const QItem* items;
  const QMerge* merges;
  int n_items, n_merge;
  int RTW;                   // row tiles per workgroup
  int L, Hq, Hkv, D, G, W, S, lt;
  float scale_log2e;
  const uint16_t* q;         // [n][L][Hq][D] bf16
  const uint16_t* k_new;     // [n][L][Hkv][D]
  const uint16_t* v_new;
  const uint8_t* k8;
  const uint8_t* v8;
  const float* k_scale;
  const float* v_scale;
  uint16_t* out;             // [n][L][Hq][D]
  float* parts;              // part_wave_floats(D) per wave of a partial slot
};
hipError_t launch_qattn(const QAttnArgs& a, bs_qformat fmt, hipStream_t s);

// ---------------------------------------------------------------- codes
typedef float qf2 __attribute__((ext_vector_type(2)));

// The four codes of a word as the numbers they stand for (in units of the scale).
template <int FMT>
__device__ inline void decode4(uint32_t w, float (&y)[4]) {
  if constexpr (FMT == BS_E4M3) {
    const qf2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    y[0] = a[0]; y[1] = a[1]; y[2] = b[0]; y[3] = b[1];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (float)((int)(w << (24 - 8 * e)) >> 24);
  }
}

// Four numbers (within the format's range) rounded to nearest even and packed.
// int8: adding 1.5 * 2^23 leaves the rounded integer, in two's complement, in
// the low byte of the sum.
template <int FMT>
__device__ inline uint32_t encode4(const float (&y)[4]) {
  if constexpr (FMT == BS_E4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  } else {
    uint32_t b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(y[e] + 12582912.0f);
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u);
    return lo | (hi << 16);
  }
}

template <int FMT>
__host__ __device__ constexpr float quant_max() { return FMT == BS_E4M3 ? kE4m3Max : kI8Max; }

__device__ inline float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
typedef __bf16 qb2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(qf2{lo, hi}, qb2));
}

}  // namespace bs
