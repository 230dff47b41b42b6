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

// Descriptors that travel in the kernel's arguments: lists of up to kNear entries need
// no upload, no slot and no event, and the launch can be captured as it stands. A
// launch takes up to 4 KiB of arguments.
constexpr int kNear = 64;
// Entry i (uniform) of a list in device memory, or of `near` in the kernel's arguments.
// Both are constant memory to the launch, so the entry comes in scalar loads.
template <class T>
__device__ inline T list_entry(const T* far, const T* near, int i) {
  static_assert(sizeof(T) % 4 == 0);
  typedef const __attribute__((address_space(4))) uint32_t* cptr;
  const cptr p = (cptr)(far ? far : near) + (int64_t)i * (sizeof(T) / 4);
  union {
    uint32_t w[sizeof(T) / 4];
    T t;
  } u;
#pragma unroll
  for (int k = 0; k < (int)(sizeof(T) / 4); ++k) u.w[k] = p[k];
  return u.t;
}
struct ReqList {
  const bs_req_desc* far;    // in device memory, or NULL: in `near`
  bs_req_desc near[kNear];
  __device__ bs_req_desc get(int i) const { return list_entry(far, near, i); }
};

struct NormRopeArgs {
  ReqList reqs;
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

// Whole rows of the box: k, v [R][Hkv][W][D] of the call's type
struct QuantArgs {
  ReqList reqs;
  int Hkv, W, S, lt;
  const void* k;
  const void* v;
  uint8_t* k8;               // [R][Hkv][W][D]
  uint8_t* v8;
  float* k_scale;            // [R][Hkv][S]
  float* v_scale;
};
hipError_t launch_kv_quantize(const QuantArgs& a, bs_dtype dt, bs_qformat fmt, int D, int n, int max_len,
                              hipStream_t s);

struct DequantArgs {
  ReqList reqs;
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

// Attention work: a request's row, or a piece of it, for all heads alike: the cached
// keys [v0, v1) in virtual keys (below) and, where `fresh` is set, the block's own keys.
// Virtual keys count the cached keys without the active block from pad = -p mod 64:
// v < s + pad is cell v - pad, v >= s + pad is cell v - pad + B; nv ends them. Groups
// of T <= 64 tokens and 64-key tiles then share borders. v0 and v1 are multiples of
// 64, but for v1 = nv of the last piece.
struct QPiece {
  int32_t req;               // request
  int32_t row, off, s;
  int32_t nv, v0, v1;
  int32_t part;              // partial slot of a split row's first head and workgroup, or -1
  int32_t np;                // pieces of the row
  int32_t split;             // of entry m of the list: the first piece of the m-th split row
  uint8_t B, pad, fresh, pad_;
};

// what one workgroup takes on: the row tiles from rt0 of one KV head of a piece
struct QItem : QPiece {
  int kvh, rt0;
};

constexpr int kQTile = 64;   // virtual keys per planning unit
constexpr int kQRowTiles = 4;   // most 32-row tiles (waves) per workgroup
constexpr int kQIssuers = 2;    // waves of it that issue the DMA

struct QAttnArgs {
  const QPiece* far;         // the pieces in device memory, or NULL: in `near`
  QPiece near[kNear];
  int n_pieces, n_split;
  int groups;                // workgroups that share a head's row tiles
  int spare;                 // waves of the last of them without a row tile or a share of the DMA
  int RTW;                   // row tiles per workgroup
  int KS;                    // RTW = 1: waves that share a row's keys (8, 4 or 2)
  int L, Hq, Hkv, D, G, W, S, lt;
  float scale_log2e;
  const uint16_t* q;         // [n][L][Hq][D] bf16
  const uint16_t* k_new;     // [n][L][Hkv][D]
  const uint16_t* v_new;
  uint8_t* k8;               // written at the block's cells and groups only, with write_back
  uint8_t* v8;
  float* k_scale;
  float* v_scale;
  int write_back;
  uint16_t* out;             // [n][L][Hq][D]
  float* parts;              // part_wave_floats(D) per wave of a partial slot
  __device__ QPiece piece(int i) const { return list_entry(far, near, i); }
};
static_assert(sizeof(QAttnArgs) <= 4096, "kernel arguments");
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
// compile-time integer passed to a generic lambda
template <int V>
struct QInt {
  static constexpr int value = V;
  __host__ __device__ constexpr operator int() const { return V; }
};

// The larger of x and its value in the lane that differs in bit O (compile time),
// where the lanes below that bit agree already: swaps within the VALU, no LDS round
// trip (a mirror reaches a lane that holds the same as the one with the bit flipped).
template <int O>
__device__ inline float max_across(float x) {
  const int v = (int)__float_as_uint(x);
  if constexpr (O == 1)
    return fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true)));     // quad 1 0 3 2
  else if constexpr (O == 2)
    return fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true)));     // quad 2 3 0 1
  else if constexpr (O == 4)
    return fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true)));    // mirror of 8
  else if constexpr (O == 8)
    return fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, true)));    // mirror of 16
  else if constexpr (O == 16) {
    const auto p = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  } else {
    const auto p = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
}

// Group maxima of a wave's rows: lane group i (GS lanes a row) of step p holds row
// p * RS + i, RS = 64 / GS, groups of T = 1 << lt rows from row 0 on; top[p] is the
// lane's own maximum on entry and its row's group's on return.
template <int GS, int RP>
__device__ inline void group_tops(float (&top)[RP], int lt) {
  constexpr int RS = 64 / GS;
  const int T = 1 << lt;
  auto stage = [&](auto o) {
    if (GS * T > decltype(o)::value) {          // uniform
#pragma unroll
      for (int i = 0; i < RP; ++i) top[i] = max_across<decltype(o)::value>(top[i]);
    }
  };
  stage(QInt<1>{});
  stage(QInt<2>{});
  stage(QInt<4>{});
  stage(QInt<8>{});
  stage(QInt<16>{});
  stage(QInt<32>{});
  // groups of several steps
#pragma unroll
  for (int b = 1; b < RP; b <<= 1)
    if (T > b * RS) {
#pragma unroll
      for (int i = 0; i < RP; ++i)
        if (!(i & b)) top[i] = top[i | b] = fmaxf(top[i], top[i | b]);
    }
}

// 4 N numbers, x(e), as codes in units of m / Q
template <int FMT, int N, class X>
__device__ inline void encode(float m, X x, uint32_t (&w)[N]) {
  // x * (Q / m) is rounded by itself, not within the addition that rounds it to an integer
#pragma clang fp contract(off)
  const float inv = quant_max<FMT>() / m;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float y[4] = {x(4 * k) * inv, x(4 * k + 1) * inv, x(4 * k + 2) * inv, x(4 * k + 3) * inv};
    w[k] = encode4<FMT>(y);
  }
}

typedef __bf16 qb2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(qf2{lo, hi}, qb2));
}

}  // namespace bs
