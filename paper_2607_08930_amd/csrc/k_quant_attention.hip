// Block attention against a dual cache held in 8 bits.
//
// As the attention over the bf16 cache (k_attention.hip), with key t of the row
// read as code * scale of its group outside the active block, and from k_new /
// v_new inside it.
//
// Row tiles. The query rows of a KV head's group are counted r = j G + h' (block
// row j, head h' of the group), so that short blocks of grouped heads fill the 32
// columns of an MFMA; a wave owns 32 of them, a workgroup of several row tiles up to
// four waves that share the K/V tiles.
//
// Virtual keys. The cached keys (prefix and suffix without the active block) are
// counted v = pad + 0, 1, ..., pad = -p mod 64. Block borders lie at multiples
// of T in v, and so does the seam where the block was left out, so groups of 32
// and 64 tokens cover whole 32-key sub-tiles and their scale is one number for the
// whole wave (UNI). Smaller groups take a scale for each key from LDS.
//
// Per sub-tile: S^T = K Q^T with v_mfma_f32_32x32x16_bf16 (keys on the M axis),
// online softmax on one query column a lane, O^T += V^T P^T with the weights fed
// straight from the accumulators. V's codes, and K's of e4m3 with one row tile, become
// bf16 in registers, exactly (e4m3 has 4 significant bits, int8 7, bf16 8); a K read of
// 16 codes feeds two MFMAs, since the order of the contraction is free, and V comes out
// of LDS transposed, 8 keys of one feature a lane (ds_read_b64_tr_b8). Elsewhere K's
// codes meet the queries as they are (SplitQueries). The K scale is folded into the
// exponent's factor and the V scale into its offset:
//   p' = vs 2^(s ks c - m) = 2^(s ks c - (m - log2 vs)),
// so neither costs an instruction per key; the row sum takes (sum p') / vs.
// The weights are rounded to bf16, whose range holds any scale allowed; fp16 would
// round eight times finer, but a weight times a small scale leaves its range.
#include <type_traits>

#include "bs_lds.h"
#include "bs_quant.h"

namespace bs {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4;
typedef __attribute__((address_space(3))) i32x2_t lds_i32x2;

__device__ inline float vmax(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// 64 lanes x 4 bytes, HBM -> the 256 bytes of LDS at `lds` (wave-uniform)
__device__ inline void dma4(uint32_t lds, const void* gptr) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(gptr)
               : "memory");
}

// eight codes as bf16
template <int FMT>
__device__ inline bf16x8_t widen8(uint32_t lo, uint32_t hi) {
  bf16x2_t x[4];
  if constexpr (FMT == BS_E4M3) {
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.0f, false);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.0f, true);
    x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.0f, false);
    x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.0f, true);
  } else {
    float y[8];
    float (&a)[4] = *reinterpret_cast<float (*)[4]>(y);
    float (&b)[4] = *reinterpret_cast<float (*)[4]>(y + 4);
    decode4<FMT>(lo, a);
    decode4<FMT>(hi, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_convertvector(qf2{y[2 * i], y[2 * i + 1]}, bf16x2_t);
  }
  return bf16x8_t{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

// XOR swizzles of a row's 16-byte slots, for an LDS that serves 256 bytes a cycle.
// Codes: a row has D / 16 slots, so 256 bytes are two rows (D = 128) or four
// (64). K reads take one chunk of 16 consecutive rows: the row pairs (quadruples)
// get distinct slots. V reads take chunks c and c ^ 1 of rows 0-3 and 8-11 (or 4-7
// and 12-15): bits 0 and 2 of the pair's number go to slot bits 1 and 2.
template <int D>
__device__ inline int swz8(int row) {
  if constexpr (D == 128) {
    const int rp = row >> 1;
    return (rp & 4) | ((rp & 1) << 1) | ((rp >> 1) & 1);
  }
  return (row >> 2) & 3;
}
// bf16 rows of the block: D / 8 slots, as in k_attention.hip
template <int D>
__device__ inline int swz16(int row) {
  if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  return ((row & 3) << 1) | ((row >> 2) & 1);
}

// The write of one tensor of an active block into the cache, by one wave, with
// k_kv_quantize's arithmetic: 16 features a lane, row(p) the 16 bf16 numbers of block
// row p RS + lane / GS (rows past B repeat the last one: it counts for no group that
// is stored). In a workgroup of several row tiles it reads the block's staged copy,
// beside the other waves' first MFMAs. With one row tile it would stand before a
// wave's first tiles and cost 3 to 5 us a launch: there waves of the launch's last
// workgroups read k_new / v_new again, where attention waves are done early. (Several
// row tiles the same way: a CU holds one such workgroup, so these would run after
// the others, 3 us.)
template <int FMT, int D, int RP, class Row>
__device__ inline void store_block(const QAttnArgs& a, const QPiece& it, int c, int tensor, int lane, Row row) {
  constexpr int GS = D / 16, RS = 64 / GS;
  const int col = (lane % GS) * 16, T = 1 << a.lt;
  float top[RP];
#pragma unroll
  for (int p = 0; p < RP; ++p) {
    top[p] = 0.0f;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const v4u x = row(p, hh);
#pragma unroll
      for (int e = 0; e < 4; ++e) top[p] = fmaxf(top[p], fmaxf(fabsf(bf_lo(x[e])), fabsf(bf_hi(x[e]))));
    }
  }
  group_tops<GS>(top, a.lt);
  const int64_t row_head = (int64_t)it.row * a.Hkv + c;
  uint8_t* codes = (tensor ? a.v8 : a.k8) + (row_head * a.W + it.off + it.s) * D + col;
  float* scales = (tensor ? a.v_scale : a.k_scale) + row_head * a.S + ((it.s + (it.pad & (T - 1))) >> a.lt);
#pragma unroll
  for (int p = 0; p < RP; ++p) {
    const int r = p * RS + lane / GS;
    if (r >= it.B) continue;
    const float m = fmaxf(top[p], kQuantFloor);
    if (col == 0 && (r & (T - 1)) == 0) scales[r >> a.lt] = m / quant_max<FMT>();
    const v4u x[2] = {row(p, 0), row(p, 1)};
    uint32_t y[4];
    encode<FMT, 4>(m, [&](int e) {
      const uint32_t z = x[e >> 3][(e >> 1) & 3];
      return e & 1 ? bf_hi(z) : bf_lo(z);
    }, y);
    st16(codes + (int64_t)r * D, v4u{y[0], y[1], y[2], y[3]});
  }
}

// An exponent factor that masked scores of -inf can be multiplied by: a product of
// small factors that fell to zero would turn them into NaN. Scores that this
// changes are zero either way. A NaN stays one.
__device__ inline float factor(float x) { return vmax(x, 1.17549435e-38f); }

// a quotient of uniform numbers, which comes out of the vector unit, back in a scalar register
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// What workgroup b takes on. The pieces' heads are counted piece by piece; the workgroups
// of a head, which read the same keys, stand eight apart, which is the same XCD and
// its L2.
__device__ inline QItem item_of(const QAttnArgs& a, int b) {
  int k = b, gr = 0;
  if (a.groups > 1) {
    const int k0 = uniform(b / (8 * a.groups)) * 8, left = a.n_pieces * a.Hkv - k0, w = left < 8 ? left : 8, u = b - k0 * a.groups;
    gr = uniform(u / w);
    k = k0 + u - gr * w;
  }
  const int i = uniform(k / a.Hkv);
  QItem it;
  static_cast<QPiece&>(it) = a.piece(i);
  it.kvh = k - i * a.Hkv;
  it.rt0 = gr * a.RTW;
  if (it.part >= 0) it.part += (it.kvh * a.groups + gr) * it.np;
  return it;
}

// One tensor of a block of up to 32 * TILES rows, read from k_new / v_new
template <int FMT, int D, int TILES>
__device__ inline void store_new(const QAttnArgs& a, const QPiece& it, int c, int tensor, int lane) {
  constexpr int GS = D / 16, RS = 64 / GS, RP = 32 * TILES / RS;
  const uint16_t* src = (tensor ? a.v_new : a.k_new) + ((int64_t)it.req * a.L * a.Hkv + c) * D + (lane % GS) * 16;
  v4u x[RP][2];
#pragma unroll
  for (int p = 0; p < RP; ++p) {
    const uint16_t* xp = src + (int64_t)min(p * RS + lane / GS, it.B - 1) * a.Hkv * D;
    x[p][0] = ld16(xp);
    x[p][1] = ld16(xp + 8);
  }
  store_block<FMT, D, RP>(a, it, c, tensor, lane, [&](int p, int hh) { return x[p][hh]; });
}

// Unit u of the launch's last workgroups: one tensor of one (piece, KV head)
template <int FMT, int D>
__device__ inline void quantize_block(const QAttnArgs& a, int u, int lane) {
  if (u >= a.n_pieces * a.Hkv * 2) return;
  const int tensor = u & 1, i = uniform((u >> 1) / a.Hkv), c = (u >> 1) - i * a.Hkv;
  const QPiece it = a.piece(i);
  if (it.fresh) store_new<FMT, D, 1>(a, it, c, tensor, lane);      // a single row tile: L <= 32
}

// ---------------------------------------------------------------- softmax state of a wave
// One wave's 32 query columns: running max (log2 units), row sums and O^T. Lane (g,
// n) holds column n and, of each 32-key sub-tile, keys 8 (rr / 4) + 4 g + rr % 4;
// its half-wave partner n holds the other 16.
template <int D>
struct Column {
  static constexpr int NDT = D / 32;
  f32x16_t o[NDT];
  float mrun, mtop, lsum;
  bf16x8_t pp[2];             // weights of the sub-tile, as the B operands of P V

  __device__ void clear() {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) o[dt][rr] = 0.0f;
    mrun = mtop = -__builtin_inff();
    lsum = 0.0f;
  }
  // raises the running max when a score exceeds it by 2^8: mx is this lane's maximum
  __device__ void raise(float mx) {
    if (__builtin_amdgcn_ballot_w64(mx > mtop) == 0) return;
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    const float mnew = fmaxf(mrun, vmax(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
    const float alpha = __builtin_amdgcn_exp2f(mrun - mnew);
    lsum *= alpha;
    mrun = mnew;
    mtop = mnew + 8.0f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) o[dt][rr] *= alpha;
  }
  // weights 2^(s f - m); returns the sum of what the MFMA consumes
  __device__ float weights(const f32x16_t& s, float f, float m) {
    float t = 0.0f;
#pragma unroll
    for (int rr = 0; rr < 16; ++rr) pp[rr >> 3][rr & 7] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[rr], f, -m));
    const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      t = __builtin_amdgcn_fdot2_f32_bf16(bf16x2_t{pp[i >> 2][2 * (i & 3)], pp[i >> 2][2 * (i & 3) + 1]}, one, t, false);
    return t;
  }
  // weights 2^(s f - m) times the keys' own V scales
  __device__ void weights_by_key(const f32x16_t& s, float f, const f32x4_t (&vs)[4]) {
#pragma unroll
    for (int rr = 0; rr < 16; ++rr) {
      const float y = __builtin_amdgcn_exp2f(fmaf(s[rr], f, -mrun));
      lsum += y;
      pp[rr >> 3][rr & 7] = (__bf16)(y * vs[rr >> 2][rr & 3]);
    }
  }
};

__device__ inline float top16(const f32x16_t& s) {
  float m = s[0];
#pragma unroll
  for (int rr = 1; rr < 16; ++rr) m = vmax(m, s[rr]);
  return m;
}
__device__ inline int key_of(int rr, int g) { return 8 * (rr >> 2) + 4 * g + (rr & 3); }
__device__ inline float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// Query columns of row tile `tile` as B operands: row r = j G + h' of the group; feature
// 32 c + 16 g + 8 h + e at MFMA 2 c + h. Rows past the block's repeat its last one.
template <int D>
__device__ inline void load_queries(const QAttnArgs& a, const QItem& it, int r, int g, bf16x8_t (&qb)[D / 16]) {
  const int rq = min(r, a.G * it.B - 1), j = (int)(((float)rq + 0.5f) * (1.0f / (float)a.G));
  const uint16_t* qp = a.q + (((int64_t)it.req * a.L + j) * a.Hq + it.kvh * a.G + (rq - j * a.G)) * D + 16 * g;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) qb[kk] = __builtin_bit_cast(bf16x8_t, ld16(qp + 32 * (kk >> 1) + 8 * (kk & 1)));
}

// V fragment i (K-step i / NDT, feature tile i % NDT) of 32 bf16 rows in LDS
template <int D>
__device__ inline bf16x8_t fresh_v(const uint8_t* vt, int i, int lane) {
  const int ks = i / (D / 32), dt = i % (D / 32), q16 = lane >> 4, j16 = lane & 15;
  bf16x4_t h[2];
#pragma unroll
  for (int h2 = 0; h2 < 2; ++h2) {
    const int row = 16 * ks + 8 * h2 + 4 * (q16 >> 1) + (j16 >> 2);
    const int col = 32 * dt + 16 * (q16 & 1) + 4 * (j16 & 3);
    h[h2] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        (lds_bf16x4*)(vt + row * D * 2 + (((col >> 3) ^ swz16<D>(row)) * 16) + (col & 7) * 2));
  }
  return __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// Output row r = j G + h' of a (request, KV head). r / G by a product: exact for r < 512.
template <int D>
__device__ inline uint16_t* out_row(const QAttnArgs& a, int req, int kvh, int r, float rg) {
  const int j = (int)(((float)r + 0.5f) * rg);
  return a.out + (((int64_t)req * a.L + j) * a.Hq + kvh * a.G + (r - j * a.G)) * D;
}

// Stores of a row tile leave as whole rows, 16 bytes a lane, over LDS (8 KiB at D =
// 128): straight from the accumulators they are 8 bytes a lane, which took 5 us of
// the 64 Dream-7B requests' 59. Features 8 k + 4 g .. + 3 of column n:
template <int D>
__device__ inline void stage_out(uint8_t* tile, int n, int k, int g, f32x4_t x, float inv, bool on) {
  typedef uint32_t v2u __attribute__((ext_vector_type(2)));
  const uint32_t w0 = pack_bf16(x[0] * inv, x[1] * inv), w1 = pack_bf16(x[2] * inv, x[3] * inv);
  // a row behind the block is zero whatever its unused column held
  *reinterpret_cast<v2u*>(tile + n * D * 2 + ((k ^ (n & (D / 8 - 1))) * 16) + 8 * g) = on ? v2u{w0, w1} : v2u{0, 0};
}
// 16-byte pieces first, first + step, ... of the tile's rows r0 ..
template <int D>
__device__ inline void send_out(const QAttnArgs& a, int req, int kvh, int r0, const uint8_t* tile, int first, int step) {
  const float rg = 1.0f / (float)a.G;
#pragma unroll 4
  for (int x = first; x < 32 * (D / 8); x += step) {
    const int row = x / (D / 8), ch = x % (D / 8), r = r0 + row;
    if (r < a.G * a.L)
      st16(out_row<D>(a, req, kvh, r, rg) + ch * 8, *reinterpret_cast<const v4u*>(tile + row * D * 2 + ((ch ^ (row & (D / 8 - 1))) * 16)));
  }
}

// Where a workgroup's cached keys lie
template <int D>
struct Keys {
  const uint8_t *k, *v;      // cell of virtual key pad
  const float *ks, *vs;      // scale of group v >> lt
  int pad, nv, seam, B, lt, glen;
  __device__ Keys(const QAttnArgs& a, const QItem& it) {
    const int64_t row_head = (int64_t)it.row * a.Hkv + it.kvh;
    pad = it.pad; nv = it.nv; seam = it.s + it.pad; B = it.B; lt = a.lt; glen = a.L >> a.lt;
    k = a.k8 + (row_head * a.W + it.off) * D;
    v = a.v8 + (row_head * a.W + it.off) * D;
    // groups count from the row's own pad, -p mod T
    const int g0 = (pad - (pad & ((1 << lt) - 1))) >> lt;
    ks = a.k_scale + row_head * a.S - g0;
    vs = a.v_scale + row_head * a.S - g0;
  }
  __device__ int cell(int x) const { return x - pad + (x >= seam ? B : 0); }
  __device__ int group(int x) const { return (x >> lt) + (x >= seam ? glen : 0); }
  // a key that exists: those before the first and past the last repeat it (masked later)
  __device__ int clamp(int x) const { return min(max(x, pad), nv - 1); }
  __device__ bool whole(int x, int n) const { return x >= pad && x + n <= nv && (x + n <= seam || x >= seam); }
};

// ---------------------------------------------------------------- queries in the codes' terms
// The queries as numbers of the codes' own kind, so that codes enter the scores' MFMAs
// as they are: a query is the sum of two of them, which costs two MFMAs of twice the
// bf16 rate (no more time) and saves the widening of K (32 to 96 VALU instructions a
// sub-tile).
//   e4m3: x 2^k = hi + lo, k putting the row's largest element into [128, 256). hi
//         holds the four leading bits, lo the four that are left of a bf16 number; lo
//         loses at most 2^-10, which is 2^-17 of the row's largest.
//   int8: x 16256 / max|x| rounded to an integer (2^-15 of the largest) = 128 hi + lo;
//         the sums of hi are shifted by 7 before lo's are added. |128 hi + lo| <=
//         16256, so the sums stay below 128 * 16256 * 128 < 2^29.
// Lane (g, n) of operand i holds features 32 i + 16 g .. + 15, as a 16-byte read of K
// finds them; e4m3's MFMAs take operands 2 j and 2 j + 1 together.
template <int FMT, int D>
struct SplitQueries {
  static constexpr int N = D / 32;
  i32x4_t hi[N], lo[N];
  float back;              // a score in these units times this is the score

  __device__ void set(const bf16x8_t (&qb)[D / 16]) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)qb[i][e]));
    top = max_across<32>(top);             // the other half-wave holds the row's other features
    float mul;
    if constexpr (FMT == BS_E4M3) {
      const int ex = min(max((int)(__float_as_uint(top) >> 23), 1 + 8), 254);
      mul = __uint_as_float((uint32_t)(254 + 7 - ex) << 23);        // 2^(7 - exponent)
      back = __uint_as_float((uint32_t)(ex - 7) << 23);
    } else {
      top = fmaxf(top, 1.17549435e-38f);
      mul = 16256.0f / top;
      back = top * (1.0f / 16256.0f);
    }
    if (!(top < __builtin_inff())) back = __uint_as_float(0x7fc00000u);   // an infinite query: no weight is a number
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (float)qb[2 * i + (w >> 1)][4 * (w & 1) + e] * mul;
        if constexpr (FMT == BS_E4M3) {
          const uint32_t h = encode4<FMT>(x);
          float y[4];
          decode4<FMT>(h, y);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = x[e] - y[e];
          hi[i][w] = (int)h;
          lo[i][w] = (int)encode4<FMT>(y);
        } else {
          uint32_t h = 0, l = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = (int)__builtin_rintf(x[e]), a = (v + 64) >> 7;
            h |= ((uint32_t)a & 255u) << (8 * e);
            l |= ((uint32_t)(v - 128 * a) & 255u) << (8 * e);
          }
          hi[i][w] = (int)h;
          lo[i][w] = (int)l;
        }
      }
  }
};

// ---------------------------------------------------------------- one row tile: waves share the keys out
// A query group of up to 32 rows (MHA blocks, single tokens of grouped heads) fills
// one wave's columns, so KS waves of a workgroup take the keys in KS runs, each with a
// ring of its own (no barrier in the loop), and join their columns through LDS at the
// end. The last wave also takes the block's own keys.
//
// What bounds it: HBM. A lone wave on a SIMD issues VALU work at half rate, and its
// sub-tile (about 150 VALU instructions, 16 exponentials, 16 MFMAs) then takes
// longer than its share of the memory's time, so the ring is sized for eight waves a
// CU (two per SIMD): two K and two V slots of 4 KiB, refilled as soon as each is read.
template <int FMT, int D, int KS, bool UNI>
__global__ __launch_bounds__(64 * KS, 2) void k_qattn_keys(QAttnArgs a) {
  constexpr int KT = 4096 / D, SPT = KT / 32;      // keys per slot, sub-tiles
  constexpr int NKK = D / 16, NDT = D / 32, NC = D / 16, NCB = D / 8;
  constexpr int SLOT = 4096, SCB = 2 * KT * 4;     // bytes of a slot, of a tile's scales
  constexpr int RING = 4 * SLOT + 2 * SCB;         // K0 K1 V0 V1, scales
  constexpr int NB = SLOT / 1024, NSC = SCB / 256;   // DMA instructions of a slot, of the scales
  constexpr int FT = 32 * D * 2;                   // bytes of the block's values
  __shared__ __align__(1024) uint8_t rings[KS * RING];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int items = a.n_pieces * a.Hkv;
  if ((int)blockIdx.x >= items) {
    quantize_block<FMT, D>(a, ((int)blockIdx.x - items) * KS + w, threadIdx.x & 63);
    return;
  }
  const QItem it = item_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63, g = lane >> 5, n = lane & 31, q16 = lane >> 4, j16 = lane & 15;
  const Keys<D> kk_(a, it);
  const int pad = kk_.pad, nv = kk_.nv, r = it.rt0 * 32 + n;
  // this wave's run of KT-key tiles: equal shares, the block's own keys counted as two tiles
  const int vfirst = it.v0 ? it.v0 : pad & ~(KT - 1);
  const int total = it.v1 > vfirst ? (it.v1 - vfirst + KT - 1) / KT : 0;
  const int own = it.fresh ? 2 : 0, share = (total + own + KS - 1) / KS;
  const int ta = min(total, w * share), cnt = min(total, w == KS - 1 ? total : ta + share) - ta;
  const int v0 = vfirst + ta * KT;
  const bool fresh = it.fresh && w == KS - 1;
  uint8_t* ring = rings + w * RING;
  const uint32_t ring_lds = __builtin_amdgcn_readfirstlane(lds_addr(rings) + (uint32_t)(w * RING));

  bf16x8_t qb[NKK];
  load_queries<D>(a, it, r, g, qb);

  // tensor (0: K, with the tile's scales, 1: V) of tile u
  auto issue = [&](auto tensor_tag, int u) {
    constexpr int tensor = decltype(tensor_tag)::value;
    const int slot = u & 1, vb = v0 + u * KT;
    const uint32_t dst = ring_lds + (uint32_t)((2 * tensor + slot) * SLOT);
    const uint8_t* cb = tensor ? kk_.v : kk_.k;
    const bool whole = kk_.whole(vb, KT);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int row = b * (1024 / D) + lane / NC, chunk = (lane % NC) ^ swz8<D>(row);
      if (whole)
        dma16_sv_once(dst + b * 1024, uniform64(cb + (int64_t)kk_.cell(vb) * D), (uint32_t)(row * D + chunk * 16));
      else
        dma16_once(dst + b * 1024, cb + (int64_t)kk_.cell(kk_.clamp(vb + row)) * D + chunk * 16);
    }
    if constexpr (tensor == 0) {
      // scales by key: K's, then V's
#pragma unroll
      for (int b = 0; b < NSC; ++b) {
        const int x = b * 64 + lane, v = kk_.clamp(vb + x % KT);
        dma4(ring_lds + (uint32_t)(4 * SLOT + slot * SCB + b * 256), (x >= KT ? kk_.vs : kk_.ks) + kk_.group(v));
      }
    }
  };
  // every LDS read so far has returned (a refill may follow)
  auto reads_done = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };

  Column<D> col;
  col.clear();
  if (fresh) {
    // values through the V slots, keys straight into the A operands
    const int foff = 4 * SLOT - FT;
#pragma unroll
    for (int b = 0; b < FT / 1024; ++b) {
      const int row = b * (1024 / (2 * D)) + lane / NCB, chunk = (lane % NCB) ^ swz16<D>(row);
      dma16(ring_lds + (uint32_t)(foff + b * 1024),
            a.v_new + (((int64_t)it.req * a.L + min(row, it.B - 1)) * a.Hkv + it.kvh) * D + chunk * 8);
    }
    const uint16_t* kp = a.k_new + (((int64_t)it.req * a.L + min(n, it.B - 1)) * a.Hkv + it.kvh) * D + 16 * g;
    f32x16_t s;
#pragma unroll
    for (int rr = 0; rr < 16; ++rr) s[rr] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, ld16(kp + 32 * (kk >> 1) + 8 * (kk & 1))),
                                                  qb[kk], s, 0, 0, 0);
    if (it.B < 32) {
#pragma unroll
      for (int rr = 0; rr < 16; ++rr)
        if (key_of(rr, g) >= it.B) s[rr] = -__builtin_inff();
    }
    col.raise(top16(s) * a.scale_log2e);
    col.lsum += col.weights(s, a.scale_log2e, col.mrun);
    wait_vm_c<0>();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 2 * NDT; ++i)
      col.o[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fresh_v<D>(ring + foff, i, lane), col.pp[i / NDT],
                                                               col.o[i % NDT], 0, 0, 0);
    reads_done();
  }
  for (int u = 0; u < min(2, cnt); ++u) {
    issue(QInt<0>{}, u);
    issue(QInt<1>{}, u);
  }

  // int8: the queries as integers, 64 VALU instructions a sub-tile less than widening K
  SplitQueries<FMT, D> sq;
  float qscale = a.scale_log2e;
  if constexpr (FMT == BS_I8) {
    sq.set(qb);
    qscale *= sq.back;
  }
  qscale = factor(qscale);

  // LDS byte offsets of this lane's K and V reads (V rows 16 apart and K rows 32
  // apart have the same swizzle)
  int koff[D / 32], voff[NDT];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) koff[i] = n * D + (((2 * i + g) ^ swz8<D>(n)) * 16);
  const int vrow = ((j16 >> 1) & 3) + 4 * g + (j16 >= 8 ? 8 : 0);
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) voff[dt] = 2 * SLOT + vrow * D + (((2 * dt + (q16 & 1)) ^ swz8<D>(vrow)) * 16) + 8 * (j16 & 1);

  constexpr int PK = NB + NSC, PV = NB;
  for (int u = 0; u < cnt; ++u) {
    const int slot = u & 1;
    if (u + 1 < cnt)
      wait_vm_c<PV + PK + PV>();               // K of u; its V and tile u + 1 may be in flight
    else
      wait_vm_c<PV>();
    asm volatile("" ::: "memory");
    const float* sc = reinterpret_cast<const float*>(ring + 4 * SLOT + slot * SCB);
    f32x16_t s[SPT];
    float f[SPT], vs[SPT];
    bool on[SPT];
#pragma unroll
    for (int sub = 0; sub < SPT; ++sub) {
      const int vb = v0 + u * KT + sub * 32;
      on[sub] = SPT == 1 || (vb + 32 > pad && vb < it.v1);   // wave-uniform
      if (!on[sub]) continue;
      const uint8_t* kt = ring + slot * SLOT + sub * 32 * D;
      if constexpr (FMT == BS_I8) {
        i32x4_t x[D / 32];
        i32x16_t t;
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) t[rr] = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          x[i] = *reinterpret_cast<const i32x4_t*>(kt + koff[i]);
          t = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[i], sq.hi[i], t, 0, 0, 0);
        }
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) t[rr] <<= 7;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) t = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[i], sq.lo[i], t, 0, 0, 0);
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) s[sub][rr] = (float)t[rr];
      } else {
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) s[sub][rr] = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const v4u x = *reinterpret_cast<const v4u*>(kt + koff[i]);
          s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>(x[0], x[1]), qb[2 * i], s[sub], 0, 0, 0);
          s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>(x[2], x[3]), qb[2 * i + 1], s[sub], 0, 0, 0);
        }
      }
      if constexpr (UNI) {
        f[sub] = factor(uniform(sc[sub * 32]) * qscale);
        vs[sub] = uniform(sc[KT + sub * 32]);
      } else {
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const f32x4_t k4 = *reinterpret_cast<const f32x4_t*>(sc + sub * 32 + 8 * qd + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[sub][4 * qd + e] *= k4[e];
        }
      }
      if (vb < pad || vb + 32 > nv) {
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) {
          const int v = vb + key_of(rr, g);
          if (v < pad || v >= nv) s[sub][rr] = -__builtin_inff();
        }
      }
    }
    // K is read: its slot takes tile u + 2's (the scales' slot too, once V's are read)
    f32x4_t vsk[UNI ? 1 : SPT][4];
    if constexpr (!UNI) {
#pragma unroll
      for (int sub = 0; sub < SPT; ++sub)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd)
          vsk[sub][qd] = *reinterpret_cast<const f32x4_t*>(sc + KT + sub * 32 + 8 * qd + 4 * g);
    }
    reads_done();
    if (u + 2 < cnt) issue(QInt<0>{}, u + 2);
#pragma unroll
    for (int sub = 0; sub < SPT; ++sub) {
      if (on[sub]) {
        if constexpr (UNI) {
          col.raise(top16(s[sub]) * f[sub]);
          col.lsum = fmaf(col.weights(s[sub], f[sub], col.mrun - __builtin_amdgcn_logf(vs[sub])),
                          __builtin_amdgcn_rcpf(vs[sub]), col.lsum);
        } else {
          col.raise(top16(s[sub]) * qscale);
          col.weights_by_key(s[sub], qscale, vsk[UNI ? 0 : sub]);
        }
      }
      if (sub == 0) {
        if (u + 2 < cnt)
          wait_vm_c<PK + PV + PK>();           // V of u; tile u + 1 and K of u + 2 may be in flight
        else if (u + 1 < cnt)
          wait_vm_c<PK + PV>();
        else
          wait_vm_c<0>();
        asm volatile("" ::: "memory");
      }
      if (!on[sub]) continue;
      const uint8_t* vt = ring + slot * SLOT + sub * 32 * D;
#pragma unroll
      for (int i = 0; i < 2 * NDT; ++i) {
        const i32x2_t x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vt + voff[i % NDT] + i / NDT * 16 * D));
        col.o[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>((uint32_t)x[0], (uint32_t)x[1]), col.pp[i / NDT],
                                                                 col.o[i % NDT], 0, 0, 0);
      }
    }
    reads_done();
    if (u + 2 < cnt) issue(QInt<1>{}, u + 2);
  }

  // join: every wave leaves O^T (in accumulator order), max and sum in its ring; wave
  // w then folds feature groups w, w + KS, ...
  col.lsum += __shfl_xor(col.lsum, 32, 64);
  static_assert(D / 8 * 1024 <= 4 * SLOT && 512 <= 2 * SCB, "a wave's column fits its ring");
#pragma unroll
  for (int k = 0; k < D / 8; ++k)
    *reinterpret_cast<f32x4_t*>(ring + (k * 64 + lane) * 16) =
        f32x4_t{col.o[k >> 2][4 * (k & 3)], col.o[k >> 2][4 * (k & 3) + 1], col.o[k >> 2][4 * (k & 3) + 2], col.o[k >> 2][4 * (k & 3) + 3]};
  float* ml = reinterpret_cast<float*>(ring + 4 * SLOT);
  ml[lane] = col.mrun;
  ml[64 + lane] = col.lsum;
  __syncthreads();
  float m = -__builtin_inff(), l = 0.0f, wgt[KS];
#pragma unroll
  for (int y = 0; y < KS; ++y) m = fmaxf(m, reinterpret_cast<const float*>(rings + y * RING + 4 * SLOT)[lane]);
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    const float* o = reinterpret_cast<const float*>(rings + x * RING + 4 * SLOT);
    wgt[x] = __builtin_amdgcn_exp2f(o[lane] - m);              // 0 for a wave without keys
    l = fmaf(o[64 + lane], wgt[x], l);
  }
  constexpr int NG = (D / 8 + KS - 1) / KS;
  f32x4_t x[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int k = w + i * KS;
    x[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int y = 0; y < KS; ++y) x[i] += *reinterpret_cast<const f32x4_t*>(rings + y * RING + (k * 64 + lane) * 16) * wgt[y];
  }
  if (it.part >= 0) {
    float* pw = a.parts + (int64_t)it.part * part_wave_floats(D);
#pragma unroll
    for (int i = 0; i < NG; ++i) *reinterpret_cast<f32x4_t*>(pw + ((w + i * KS) * 64 + lane) * 4) = x[i];
    if (w == 0) {
      pw[D / 8 * 256 + lane] = m;
      pw[D / 8 * 256 + 64 + lane] = l;
    }
    return;
  }
  __syncthreads();                             // the columns are read: their place takes the rows
  const bool on = r < a.G * it.B;
  const float inv = 1.0f / l;
#pragma unroll
  for (int i = 0; i < NG; ++i) stage_out<D>(rings, n, w + i * KS, g, x[i], inv, on);
  __syncthreads();
  send_out<D>(a, it.req, it.kvh, it.rt0 * 32, rings, threadIdx.x, 64 * KS);
}

// ---------------------------------------------------------------- several row tiles: waves share the ring
// One wave a row tile; up to four waves share the K/V tiles of a 4-stage ring, and two
// such workgroups a CU (two waves per SIMD). Eight waves in one workgroup a CU, which
// read each tile once and shared the widening of V, took 67 us instead of 77 for 64
// Dream-7B rows of equal length, but 57 instead of 52 for ragged ones: a row's two
// workgroups share their CUs with shorter rows'.
//
// What bounds it: the vector unit, then latencies that two waves a SIMD do not cover. A
// sub-tile is 104 vector instructions (five cycles each from two waves, an exponential
// ten; an MFMA hides six of them) beside 510 cycles of MFMAs, and takes 1200 cycles in a lone
// wave; raises, masks, the queries' split and the output add half as many instructions.
// A workgroup's start and end take 10 us, and under full load the clock falls from 2.4 to
// 2.0 GHz.
template <int FMT, int D, bool UNI>
__global__ __launch_bounds__(64 * kQRowTiles, 2) void k_qattn_group(QAttnArgs a) {
  constexpr int KT = 64, NS = 4, NI = kQIssuers;   // keys per stage, stages, waves that issue the DMA
  constexpr int NKK = D / 16, NDT = D / 32, NC = D / 16, NCB = D / 8;
  constexpr int TILE = KT * D, STAGE = 2 * TILE;   // bytes: K tile, then V tile
  constexpr int RPB = 1024 / D;                    // rows per 1 KiB DMA block
  constexpr int RPI = KT / RPB / NI;               // blocks per tensor and issuing wave
  constexpr int PB = 2 * RPI + 1;                  // DMA instructions per stage and issuing wave
  constexpr int SCB = 2 * KT * 4;                  // bytes of a stage's scales
  static_assert(KT / RPB % NI == 0, "issuing waves split a tile evenly");
  __shared__ __align__(1024) uint8_t ring[NS * STAGE + NS * SCB];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const QItem it = item_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63, g = lane >> 5, n = lane & 31, q16 = lane >> 4, j16 = lane & 15;
  const Keys<D> keys(a, it);
  const int B = it.B, pad = it.pad, nv = it.nv, v0 = it.v0, v1 = it.v1;
  const int ntiles = (v1 - v0 + KT - 1) / KT;
  const bool issuer = w < NI;
  const int seam_ = keys.seam;
  const int r = (it.rt0 + w) * 32 + n;
  const int nsub = v1 > v0 ? (v1 - v0 + 31) / 32 : 0;
  // The last of a head's workgroups may have waves to spare (a.spare of them, without a row
  // and without a share of the DMA): they keep step with the others, then write the block
  // into the cache, which otherwise the first workgroup's last waves do before their
  // first tiles (64 Dream-7B requests, seven row tiles a head, of one length: 55 us
  // instead of 59; ragged: 49.7 instead of 50.6).
  if (it.rt0 + a.RTW == a.groups * a.RTW && w >= a.RTW - a.spare) {
    const int steps = (it.fresh ? 2 : 0) + (nsub > 0 ? 1 + nsub / 2 : 0);
    for (int i = 0; i < steps; ++i) __builtin_amdgcn_s_barrier();
    if (a.write_back && it.fresh)
      for (int tensor = w - (a.RTW - a.spare); tensor < 2; tensor += a.spare) {
        if (a.L > 32)
          store_new<FMT, D, 2>(a, it, it.kvh, tensor, lane);
        else
          store_new<FMT, D, 1>(a, it, it.kvh, tensor, lane);
      }
    if (it.part < 0) __builtin_amdgcn_s_barrier();     // ahead of the staged rows
    return;
  }

  bf16x8_t qb[NKK];
  load_queries<D>(a, it, r, g, qb);

  const uint32_t ring_lds = __builtin_amdgcn_readfirstlane(lds_addr(ring));
  // This lane's 16 bytes of a DMA block: the blocks of a wave lie NI * RPB rows apart, a
  // multiple of the swizzle's period, so one offset serves them all.
  static_assert(NI * RPB % 16 == 0, "the swizzle repeats every 16 rows");
  const int row0 = w * RPB + lane / NC;
  const uint32_t lane_off = (uint32_t)(row0 * D + (((lane % NC) ^ swz8<D>(row0)) * 16));
  auto issue = [&](int u, int slot) {
    if (!issuer) return;
    const int vb = v0 + u * KT;
    const uint32_t sbase = ring_lds + (uint32_t)(slot * STAGE + w * 1024);
    const uint32_t ssc = ring_lds + (uint32_t)(NS * STAGE + slot * SCB + (w & 1) * KT * 4);
    const float* sp = w & 1 ? keys.vs : keys.ks;   // scales by key: K's, then V's
    if (keys.whole(vb, KT)) {
      const int64_t at = (int64_t)keys.cell(vb) * D;
#pragma unroll
      for (int k = 0; k < 2 * RPI; ++k) {
        const int tensor = k / RPI, blk = k % RPI * NI;
        dma16_sv_once(sbase + (uint32_t)(tensor * TILE + blk * 1024), uniform64((tensor ? keys.v : keys.k) + at + blk * 1024), lane_off);
      }
      dma4(ssc, sp + (vb >= seam_ ? keys.glen : 0) + ((vb + lane) >> keys.lt));
    } else {
      // rows before the first key and past the last repeat one of them (masked later)
#pragma unroll
      for (int k = 0; k < 2 * RPI; ++k) {
        const int tensor = k / RPI, blk = k % RPI * NI, row = blk * RPB + row0;
        dma16_once(sbase + (uint32_t)(tensor * TILE + blk * 1024),
                   (tensor ? keys.v : keys.k) + (int64_t)keys.cell(keys.clamp(vb + row)) * D + (int)lane_off % D);
      }
      dma4(ssc, sp + keys.group(keys.clamp(vb + lane)));
    }
  };
  auto wait_stages = [&](int x) {
    if (!issuer) return;
    if (x <= 0)
      wait_vm_c<0>();
    else if (x == 1)
      wait_vm_c<PB>();
    else if (x == 2)
      wait_vm_c<2 * PB>();
    else
      wait_vm_c<3 * PB>();
  };
  // every LDS read of this wave has returned, then all waves are here
  auto barrier = [] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  Column<D> col;
  col.clear();
  int issued = 0;
  if (it.fresh) {
    // the block's own rows, as bf16 in the last part of the ring
    const int RB = (a.L + 31) / 32, FT = RB * 32 * D * 2;    // bytes per tensor
    const int foff = NS * STAGE - 2 * FT;
    constexpr int FR = 1024 / (2 * D);                       // rows per DMA block
    if (issuer)
      for (int b = w; b < 2 * FT / 1024; b += NI) {
        const int tensor = b >= FT / 1024, bb = b - (tensor ? FT / 1024 : 0);
        const int row = bb * FR + lane / NCB, chunk = (lane % NCB) ^ swz16<D>(row);
        const uint16_t* src = (tensor ? a.v_new : a.k_new) +
                              (((int64_t)it.req * a.L + min(row, B - 1)) * a.Hkv + it.kvh) * D + chunk * 8;
        dma16(ring_lds + (uint32_t)(foff + b * 1024), src);
      }
    for (const int lim = min(NS - (2 * FT + STAGE - 1) / STAGE, min(NS - 1, ntiles)); issued < lim; ++issued) issue(issued, issued);
    wait_stages(issued);
    barrier();
    for (int sub = 0; sub * 32 < B; ++sub) {
      const uint8_t* kt = ring + foff + sub * 32 * D * 2;
      f32x16_t s;
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) s[rr] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        const int chunk = 4 * (kk >> 1) + 2 * g + (kk & 1);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *reinterpret_cast<const bf16x8_t*>(kt + n * D * 2 + ((chunk ^ swz16<D>(n)) * 16)), qb[kk], s, 0, 0, 0);
      }
      if (sub * 32 + 32 > B) {
#pragma unroll
        for (int rr = 0; rr < 16; ++rr)
          if (sub * 32 + key_of(rr, g) >= B) s[rr] = -__builtin_inff();
      }
      col.raise(top16(s) * a.scale_log2e);
      col.lsum += col.weights(s, a.scale_log2e, col.mrun);
#pragma unroll
      for (int i = 0; i < 2 * NDT; ++i)
        col.o[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fresh_v<D>(kt + FT, i, lane), col.pp[i / NDT],
                                                                 col.o[i % NDT], 0, 0, 0);
    }
    // K and V by the last two waves: where there are enough, those that issue no DMA, so
    // that no stage waits for the stores
    const int wt = w - (a.RTW - 2);
    if (a.write_back && a.spare == 0 && it.rt0 == 0 && (wt == 0 || wt == 1)) {
      constexpr int GS = D / 16, RS = 64 / GS;
      auto row = [&](int p, int hh) {
        const int x = p * RS + lane / GS, ch = 2 * (lane % GS) + hh;
        return *reinterpret_cast<const v4u*>(ring + foff + wt * FT + x * D * 2 + ((ch ^ swz16<D>(x)) * 16));
      };
      if (RB == 2)
        store_block<FMT, D, 64 / RS>(a, it, it.kvh, wt, lane, row);
      else
        store_block<FMT, D, 32 / RS>(a, it, it.kvh, wt, lane, row);
    }
    barrier();
  }
  for (const int lim = min(NS - 1, ntiles); issued < lim; ++issued) issue(issued, issued);

  // LDS byte offsets of this lane's K and V reads (V rows 16 apart and K rows 32
  // apart have the same swizzle)
  int koff[D / 32], voff[NDT];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) koff[i] = n * D + (((2 * i + g) ^ swz8<D>(n)) * 16);
  const int vrow = ((j16 >> 1) & 3) + 4 * g + (j16 >= 8 ? 8 : 0);
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
    voff[dt] = TILE + vrow * D + (((2 * dt + (q16 & 1)) ^ swz8<D>(vrow)) * 16) + 8 * (j16 & 1);
  // K codes of operand i, V codes of MFMA i
  auto kraw = [&](int slot, int half, int i) {
    return *reinterpret_cast<const i32x4_t*>(ring + koff[i] + slot * STAGE + half * 32 * D);
  };
  auto vraw = [&](int slot, int half, int i) {
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(ring + voff[i % NDT] + slot * STAGE + (2 * half + i / NDT) * 16 * D));
  };
  auto scales = [&](int slot, int half) { return reinterpret_cast<const float*>(ring + NS * STAGE + slot * SCB) + half * 32; };
  // x is computed here: keeps the compiler from sinking it past a fence
  auto pin = [](float& x) { asm volatile("" : "+v"(x)); };
  // t + the q-th pair of weights, as the MFMA takes them
  auto add_pair = [&](int q, float t) {
    const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(bf16x2_t{col.pp[q >> 2][2 * (q & 3)], col.pp[q >> 2][2 * (q & 3) + 1]}, one, t, false);
  };

  SplitQueries<FMT, D> sq;
  sq.set(qb);
  const float qscale = factor(a.scale_log2e * sq.back);
  // MFMAs of P V; of the scores (e4m3: 64 features each, twice as long)
  constexpr int NPV = 2 * NDT, NSC = FMT == BS_E4M3 ? D / 32 : D / 16, NSL = NPV + NSC;
  using acc_t = typename std::conditional<FMT == BS_E4M3, f32x16_t, i32x16_t>::type;
  const int u0 = v0 + 32 <= pad ? 1 : 0;             // a first sub-tile without keys
  acc_t sA, sB;
  i32x4_t rk[D / 32];                                // K codes of a sub-tile
  i32x2_t rv[4];                                     // V codes read three MFMAs ahead
  bf16x8_t fr[2];                                    // V operands, widened one MFMA ahead
  float kf = 0.0f, vs = 0.0f;                        // UNI: scales of the sub-tile whose scores are in
  auto score_mfma = [&](int i, acc_t& s) {
    if (i == 0) {
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) s[rr] = 0;
    }
    if constexpr (FMT == BS_E4M3) {
      const int j = i >> 1;
      const i32x4_t& q0 = i & 1 ? sq.lo[2 * j] : sq.hi[2 * j];
      const i32x4_t& q1 = i & 1 ? sq.lo[2 * j + 1] : sq.hi[2 * j + 1];
      // scale operands of 0: the MFMA without scales
      s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(__builtin_shufflevector(rk[2 * j], rk[2 * j + 1], 0, 1, 2, 3, 4, 5, 6, 7),
                                                          __builtin_shufflevector(q0, q1, 0, 1, 2, 3, 4, 5, 6, 7), s, 0, 0, 0, 0, 0, 0);
    } else {
      constexpr int N = D / 32;
      if (i == N) {
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) s[rr] <<= 7;
      }
      s = __builtin_amdgcn_mfma_i32_32x32x32_i8(rk[i % N], i < N ? sq.hi[i] : sq.lo[i - N], s, 0, 0, 0);
    }
  };

  // One sub-tile u, half H of ring slot S (compile time in the unrolled loop, where
  // every LDS address is then an immediate): ss holds its scores, col.pp the weights
  // of u - 1; writes the scores of u + 1 to sn and the weights of u to col.pp. Slots
  // of one MFMA each, in an order fixed by scheduling fences: P V of u - 1 (none for
  // the first sub-tile), then the scores of u + 1 (of stale LDS contents, and
  // discarded, for the last); beside them the widening of V's operands and the softmax
  // of u in 16 steps, for a wave's MFMAs overlap its own VALU work only.
  auto sub_tile = [&](auto S, auto half_tag, auto first_tag, int u, acc_t& ss, acc_t& sn) {
    constexpr int H = decltype(half_tag)::value;
    constexpr bool FIRST = decltype(first_tag)::value != 0;
    const int s0 = S, sp = H ? s0 : (s0 + NS - 1) % NS, sx = H ? (s0 + 1) % NS : s0;
    if constexpr (H == 1) {
      // the next tile has landed once only later ones are in flight; past the barrier
      // every wave is done with the tile before this one, whose slot is refilled
      const int t = u >> 1;
      wait_stages(min(t == 0 ? 2 : 1, max(ntiles - 2 - t, 0)));
      barrier();
      if (t + 3 < ntiles && t > 0) issue(t + 3, (s0 + NS - 1) % NS);
    }
    const int vb = v0 + u * 32;
    f32x4_t k4[4], v4[4];                            // scales by key: V's are read as they are needed
    if constexpr (!UNI) {
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) k4[qd] = *reinterpret_cast<const f32x4_t*>(scales(s0, H) + 8 * qd + 4 * g);
    }
    const float f = UNI ? factor(kf * qscale) : qscale;
    f32x16_t sc;
    float m3[4], mx = 0.0f, off = 0.0f, ivs = 0.0f, alpha = 1.0f, sum = 0.0f;
    bool resc = false;
    // step st of the softmax of u
    auto step = [&](int st) {
      if (!UNI && st >= 2 && st <= 8 && st % 2 == 0)
        v4[st / 2 - 1] = *reinterpret_cast<const f32x4_t*>(scales(s0, H) + KT + 8 * (st / 2 - 1) + 4 * g);
      if (st == 0) {
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) {
          sc[rr] = (float)ss[rr];
          if constexpr (!UNI) sc[rr] *= k4[rr >> 2][rr & 3];
        }
        if (vb < pad || vb + 32 > nv) {
#pragma unroll
          for (int rr = 0; rr < 16; ++rr) {
            const int v = vb + key_of(rr, g);
            if (v < pad || v >= nv) sc[rr] = -__builtin_inff();
          }
        }
      } else if (st == 1) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          m3[q] = vmax(vmax(sc[3 * q], sc[3 * q + 1]), sc[3 * q + 2]);
          pin(m3[q]);
        }
      } else if (st == 2) {
        m3[0] = vmax(vmax(sc[12], sc[13]), m3[0]);
        m3[1] = vmax(vmax(sc[14], sc[15]), m3[1]);
        m3[0] = vmax(vmax(m3[0], m3[1]), m3[2]);
        mx = vmax(m3[0], m3[3]) * f;                   // log2 units
        pin(mx);
      } else if (st == 3) {
        // lazily raised running max (Column::raise, with O rescaled after P V of u - 1)
        resc = __builtin_amdgcn_ballot_w64(mx > col.mtop) != 0;
        if (resc) {
          const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
          const float mnew = fmaxf(col.mrun, vmax(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
          alpha = __builtin_amdgcn_exp2f(col.mrun - mnew);
          col.lsum *= alpha;
          col.mrun = mnew;
          col.mtop = mnew + 8.0f;
        }
        off = UNI ? col.mrun - __builtin_amdgcn_logf(vs) : col.mrun;
        if (UNI) ivs = __builtin_amdgcn_rcpf(vs);
        pin(off);
      } else if (st < 12) {
#pragma unroll
        for (int y = 2 * (st - 4); y < 2 * (st - 4) + 2; ++y) {
          float p = __builtin_amdgcn_exp2f(fmaf(sc[y], f, -off));
          if constexpr (!UNI) {
            col.lsum += p;
            p *= v4[y >> 2][y & 3];
          }
          pin(p);
          sc[y] = p;
        }
      }
      if (st >= 8) {
        // P V has read the old weights by now
        const int e = 2 * (st - 8);
        col.pp[e >> 3][e & 7] = (__bf16)sc[e];
        col.pp[e >> 3][(e & 7) + 1] = (__bf16)sc[e + 1];
        if (UNI && e >= 2) sum = add_pair(e / 2 - 1, sum);
      }
    };
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NSL; ++i) {
      // operands: V's three MFMAs ahead (past the end: of the next sub-tile's P V), K's
      // beside the last MFMAs of P V
      const int jv = i + 3;
      if (jv >= NSL)
        rv[(jv - NSL) & 3] = vraw(s0, H, jv - NSL);
      else if (jv < NPV && !FIRST)
        rv[jv & 3] = vraw(sp, 1 - H, jv);
      if (i < NPV && i >= NPV - D / 32) rk[i - (NPV - D / 32)] = kraw(sx, 1 - H, i - (NPV - D / 32));
      if (i < NPV) {
        if constexpr (!FIRST)
          col.o[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i & 1], col.pp[i / NDT], col.o[i % NDT], 0, 0, 0);
      } else {
        score_mfma(i - NPV, sn);
      }
      // widen the next MFMA's operand (past the end: the next sub-tile's first)
      if (i + 1 < NPV ? !FIRST : i + 1 == NSL) {
        const i32x2_t& x = rv[i + 1 == NSL ? 0 : (i + 1) & 3];
        fr[i + 1 == NSL ? 0 : (i + 1) & 1] = widen8<FMT>((uint32_t)x[0], (uint32_t)x[1]);
      }
      // the softmax: steps 0 .. 3 beside P V, which has V's widening, 4 .. 15 beside the
      // scores (half and half: 1 us of 50 more for 64 Dream-7B requests)
      const int b0 = i < NPV ? i * 4 / NPV : 4 + (i - NPV) * 12 / NSC, b1 = i < NPV ? (i + 1) * 4 / NPV : 4 + (i + 1 - NPV) * 12 / NSC;
#pragma unroll
      for (int st = b0; st < b1; ++st)
        step(st);
      __builtin_amdgcn_sched_barrier(0);
      if (!FIRST && i == NPV - 1 && resc) {               // after P V of u - 1, before that of u
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int rr = 0; rr < 16; ++rr) col.o[dt][rr] *= alpha;
      }
    }
    if (FIRST && resc) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) col.o[dt][rr] *= alpha;
    }
    if constexpr (UNI) {
      col.lsum = fmaf(add_pair(7, sum), ivs, col.lsum);
      kf = scales(sx, 1 - H)[0];                          // stale for the last sub-tile, and unused
      vs = scales(sx, 1 - H)[KT];
    }
  };

  if (nsub > 0) {
    wait_stages(min(NS - 2, ntiles - 1));
    barrier();
    if (3 < ntiles) issue(3, 3);
    // scores of the first sub-tile
#pragma unroll
    for (int i = 0; i < D / 32; ++i) rk[i] = kraw(0, u0, i);
#pragma unroll
    for (int i = 0; i < NSC; ++i) score_mfma(i, sA);
    if constexpr (UNI) {
      kf = scales(0, u0)[0];
      vs = scales(0, u0)[KT];
    }
    using C0 = QInt<0>;
    using C1 = QInt<1>;
    // tile 0, then four tiles a trip with compile-time slots, then the rest; the
    // scores of an even sub-tile are in sA, of an odd one in sB
    if (u0 == 0) {
      sub_tile(C0{}, C0{}, C1{}, 0, sA, sB);
      if (nsub > 1) sub_tile(C0{}, C1{}, C0{}, 1, sB, sA);
    } else {
      sB = sA;
      sub_tile(C0{}, C1{}, C1{}, 1, sB, sA);
    }
    int u = 2;
    for (; u + 7 < nsub; u += 8) {
      sub_tile(QInt<1>{}, C0{}, C0{}, u, sA, sB);
      sub_tile(QInt<1>{}, C1{}, C0{}, u + 1, sB, sA);
      sub_tile(QInt<2>{}, C0{}, C0{}, u + 2, sA, sB);
      sub_tile(QInt<2>{}, C1{}, C0{}, u + 3, sB, sA);
      sub_tile(QInt<3>{}, C0{}, C0{}, u + 4, sA, sB);
      sub_tile(QInt<3>{}, C1{}, C0{}, u + 5, sB, sA);
      sub_tile(QInt<0>{}, C0{}, C0{}, u + 6, sA, sB);
      sub_tile(QInt<0>{}, C1{}, C0{}, u + 7, sB, sA);
    }
    for (; u < nsub; u += 2) {
      const int slot = (u >> 1) % NS;
      sub_tile(slot, C0{}, C0{}, u, sA, sB);
      if (u + 1 < nsub) sub_tile(slot, C1{}, C0{}, u + 1, sB, sA);
    }
    // P V of the last sub-tile
    const int ul = nsub - 1, sl = (ul >> 1) % NS, hl = ul & 1;
    // its first operand is widened, the next two are read
#pragma unroll
    for (int i = 0; i < NPV; ++i) {
      if (i + 3 < NPV) rv[(i + 3) & 3] = vraw(sl, hl, i + 3);
      col.o[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i & 1], col.pp[i / NDT], col.o[i % NDT], 0, 0, 0);
      if (i + 1 < NPV) fr[(i + 1) & 1] = widen8<FMT>((uint32_t)rv[(i + 1) & 3][0], (uint32_t)rv[(i + 1) & 3][1]);
    }
  }

  col.lsum += __shfl_xor(col.lsum, 32, 64);
  // lane (g, n): O^T[feature 8 k + 4 g + e][query n]
  auto group4 = [&](int k) {
    return f32x4_t{col.o[k >> 2][4 * (k & 3)], col.o[k >> 2][4 * (k & 3) + 1], col.o[k >> 2][4 * (k & 3) + 2], col.o[k >> 2][4 * (k & 3) + 3]};
  };
  if (it.part >= 0) {
    float* pw = a.parts + ((int64_t)it.part * a.RTW + w) * part_wave_floats(D);
#pragma unroll
    for (int k = 0; k < D / 8; ++k) *reinterpret_cast<f32x4_t*>(pw + (k * 64 + lane) * 4) = group4(k);
    pw[D / 8 * 256 + lane] = col.mrun;
    pw[D / 8 * 256 + 64 + lane] = col.lsum;
    return;
  }
  barrier();                                   // the ring is read: each wave's share takes its rows
  static_assert(kQRowTiles * 32 * D * 2 <= NS * STAGE, "the row tiles fit the ring");
  uint8_t* tile = ring + w * 32 * D * 2;
  const bool on = r < a.G * B;
  const float inv = 1.0f / col.lsum;
#pragma unroll
  for (int k = 0; k < D / 8; ++k) stage_out<D>(tile, n, k, g, group4(k), inv, on);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  send_out<D>(a, it.req, it.kvh, (it.rt0 + w) * 32, tile, lane, 64);
}

// Joins the pieces of a split row: one wave per (row, row tile, group of 4
// features), folding the pieces' partials by their running maxima, eight loads in
// flight.
template <int D>
__global__ __launch_bounds__(256) void k_qattn_merge(QAttnArgs a) {
  constexpr int NG = D / 8, CH = kMergeBatch;
  const int wv = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int heads = a.Hkv * a.groups;
  if (wv >= a.n_split * heads * a.RTW * NG) return;
  const int k = wv % NG, tw = uniform(wv / NG / a.RTW), t = wv / NG - tw * a.RTW;
  const int mi = uniform(tw / heads), hg = tw - mi * heads;
  const QPiece mg = a.piece(a.piece(mi).split);
  const int64_t stride = (int64_t)a.RTW * part_wave_floats(D);
  const float* pw = a.parts + ((int64_t)(mg.part + hg * mg.np) * a.RTW + t) * part_wave_floats(D);
  f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
  float m = -__builtin_inff(), l = 0.0f;
  for (int p0 = 0; p0 < mg.np; p0 += CH) {
    float mp[CH], lp[CH];
    f32x4_t op[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const bool ok = p0 + i < mg.np;
      const float* pp = pw + (ok ? p0 + i : p0) * stride;
      mp[i] = ok ? pp[NG * 256 + lane] : -__builtin_inff();
      lp[i] = pp[NG * 256 + 64 + lane];
      op[i] = *reinterpret_cast<const f32x4_t*>(pp + (k * 64 + lane) * 4);
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < CH; ++i) mn = fmaxf(mn, mp[i]);
    const float sa = __builtin_amdgcn_exp2f(m - mn);
    l *= sa;
    acc *= sa;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const float sb = __builtin_amdgcn_exp2f(mp[i] - mn);     // 0 for the padding entries
      l = fmaf(lp[i], sb, l);
      acc += op[i] * sb;
    }
    m = mn;
  }
  const int kvh = uniform(hg / a.groups), r = ((hg - kvh * a.groups) * a.RTW + t) * 32 + (lane & 31);
  if (r >= a.G * a.L) return;
  const float inv = 1.0f / l;
  typedef uint32_t v2u __attribute__((ext_vector_type(2)));
  const v2u y = {pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
  *reinterpret_cast<v2u*>(out_row<D>(a, mg.req, kvh, r, 1.0f / (float)a.G) + 8 * k + 4 * (lane >> 5)) =
      r < a.G * mg.B ? y : v2u{0, 0};
}

template <int FMT, int D>
void attend(const QAttnArgs& a, hipStream_t s) {
  auto go = [&](auto kernel, int waves) {
    // one row tile: workgroups that write the blocks into the cache stand last
    const int heads = a.n_pieces * a.Hkv, wb = a.write_back && a.RTW == 1 ? (heads * 2 + waves - 1) / waves : 0;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(heads * a.groups + wb)), dim3((unsigned)(64 * waves)), 0, s, a);
  };
  auto by_groups = [&](auto uni_tag) {
    constexpr bool UNI = decltype(uni_tag)::value != 0;
    if (a.RTW > 1)
      go(k_qattn_group<FMT, D, UNI>, a.RTW);
    else if (a.KS == 8)
      go(k_qattn_keys<FMT, D, 8, UNI>, 8);
    else if (a.KS == 4)
      go(k_qattn_keys<FMT, D, 4, UNI>, 4);
    else
      go(k_qattn_keys<FMT, D, 2, UNI>, 2);
  };
  a.lt >= 5 ? by_groups(QInt<1>{}) : by_groups(QInt<0>{});
  if (a.n_split)
    hipLaunchKernelGGL(k_qattn_merge<D>, dim3((unsigned)(((int64_t)a.n_split * a.Hkv * a.groups * a.RTW * (D / 8) + 3) / 4)), dim3(256), 0,
                       s, a);
}

}  // namespace

hipError_t launch_qattn(const QAttnArgs& a, bs_qformat fmt, hipStream_t s) {
  if (a.D == 64)
    fmt == BS_E4M3 ? attend<BS_E4M3, 64>(a, s) : attend<BS_I8, 64>(a, s);
  else
    fmt == BS_E4M3 ? attend<BS_E4M3, 128>(a, s) : attend<BS_I8, 128>(a, s);
  return hipGetLastError();
}

}  // namespace bs
