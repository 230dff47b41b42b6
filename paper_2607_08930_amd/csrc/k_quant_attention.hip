// Block attention against a dual cache held in 8 bits.
//
// As the attention over the bf16 cache (k_attention.hip), with key t of the row
// read as code * scale of its group outside the active block, and from k_new /
// v_new inside it.
//
// Row tiles. The query rows of a KV head's group are counted r = j G + h' (block
// row j, head h' of the group), so that short blocks of grouped heads fill the 32
// columns of an MFMA; a wave owns 32 of them, a workgroup up to eight waves that
// share the K/V tiles.
//
// Virtual keys. The cached keys (prefix and suffix without the active block) are
// counted v = pad + 0, 1, ..., pad = -p mod 64. Block borders lie at multiples
// of T in v, and so does the seam where the block was left out, so groups of 32
// and 64 tokens cover whole 32-key sub-tiles and their scale is one number for the
// whole wave (UNI). Smaller groups take a scale for each key from LDS.
//
// Per sub-tile: S^T = K Q^T with v_mfma_f32_32x32x16_bf16 (keys on the M axis),
// online softmax on one query column a lane, O^T += V^T P^T with the weights fed
// straight from the accumulators. Codes become bf16 in registers, exactly (e4m3
// has 4 significant bits, int8 7, bf16 8); a K read of 16 codes feeds two MFMAs,
// since the order of the contraction is free, and V comes out of LDS transposed,
// 8 keys of one feature a lane (ds_read_b64_tr_b8). The K scale is folded into the
// exponent's factor and the V scale into its offset:
//   p' = vs 2^(s ks c - m) = 2^(s ks c - (m - log2 vs)),
// so neither costs an instruction per key; the row sum takes (sum p') / vs.
// The weights are rounded to bf16, whose range holds any scale allowed; fp16 would
// round eight times finer, but a weight times a small scale leaves its range.
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

// The write of the active blocks into the cache: wave u of the launch's last
// workgroups quantises one tensor of one (request, KV head), with k_kv_quantize's
// arithmetic. It reads k_new / v_new again instead of the attention's staged copy:
// inside the attention's waves the same work stood before their first tiles and cost
// 3 to 5 us a launch, while these waves run where attention waves are done early.
template <int FMT, int D, int RP>
__device__ inline void quantize_block(const QAttnArgs& a, int u, int lane) {
  constexpr int GS = D / 16, RS = 64 / GS;
  if (u >= a.n * a.Hkv * 2) return;
  const int tensor = u & 1, c = (u >> 1) % a.Hkv, i = (u >> 1) / a.Hkv;
  const QItem it = a.rows[i];
  const int col = (lane % GS) * 16, T = 1 << a.lt;
  const uint16_t* src = (tensor ? a.v_new : a.k_new) + ((int64_t)i * a.L * a.Hkv + c) * D + col;
  v4u x[RP][2];
  float top[RP];
#pragma unroll
  for (int p = 0; p < RP; ++p) {
    // rows past B repeat the last one: it counts for no group that is stored
    const uint16_t* xp = src + (int64_t)min(p * RS + lane / GS, it.B - 1) * a.Hkv * D;
    x[p][0] = ld16(xp);
    x[p][1] = ld16(xp + 8);
  }
#pragma unroll
  for (int p = 0; p < RP; ++p) {
    top[p] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top[p] = fmaxf(top[p], fmaxf(fabsf(bf_lo(x[p][e >> 2][e & 3])), fabsf(bf_hi(x[p][e >> 2][e & 3]))));
  }
  group_tops<GS>(top, a.lt);
  const int64_t row_head = (int64_t)it.row * a.Hkv + c;
  const int tpad = it.pad & (T - 1);
  uint8_t* codes = (tensor ? a.v8 : a.k8) + (row_head * a.W + it.off + it.s) * D + col;
  float* scales = (tensor ? a.v_scale : a.k_scale) + row_head * a.S + ((it.s + tpad) >> a.lt);
#pragma unroll
  for (int p = 0; p < RP; ++p) {
    const int row = p * RS + lane / GS;
    if (row >= it.B) continue;
    const float m = fmaxf(top[p], kQuantFloor);
    if (col == 0 && (row & (T - 1)) == 0) scales[row >> a.lt] = m / quant_max<FMT>();
    st16(codes + (int64_t)row * D, encode16<FMT>(m, [&](int e) {
           const uint32_t y = x[p][e >> 3][(e >> 1) & 3];
           return e & 1 ? bf_hi(y) : bf_lo(y);
         }));
  }
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
  // weights 2^(s - m) times the keys' own V scales
  __device__ void weights_by_key(const f32x16_t& s, const f32x4_t (&vs)[4]) {
#pragma unroll
    for (int rr = 0; rr < 16; ++rr) {
      const float y = __builtin_amdgcn_exp2f(s[rr] - mrun);
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
  const int rq = min(r, a.G * it.B - 1), j = rq / a.G;
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

// Four output features (group k: 8 k + 4 g ..) of row r, or zeros behind the block
template <int D>
__device__ inline void store_out(const QAttnArgs& a, int req, int kvh, int B, int r, int k, int g, f32x4_t x, float l) {
  if (r >= a.G * a.L) return;
  const int j = r / a.G;
  const float inv = r < a.G * B ? 1.0f / l : 0.0f;
  uint16_t* op = a.out + (((int64_t)req * a.L + j) * a.Hq + kvh * a.G + (r - j * a.G)) * D + 8 * k + 4 * g;
  typedef uint32_t v2u __attribute__((ext_vector_type(2)));
  // a row behind the block is zero whatever its unused column held
  const bool on = r < a.G * B;
  const uint32_t w0 = pack_bf16(x[0] * inv, x[1] * inv), w1 = pack_bf16(x[2] * inv, x[3] * inv);
  *reinterpret_cast<v2u*>(op) = on ? v2u{w0, w1} : v2u{0, 0};
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
  if ((int)blockIdx.x >= a.n_items) {
    quantize_block<FMT, D, D / 32>(a, ((int)blockIdx.x - a.n_items) * KS + w, threadIdx.x & 63);
    return;
  }
  const QItem it = a.items[blockIdx.x];
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
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) s[sub][rr] = 0.0f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const v4u x = *reinterpret_cast<const v4u*>(kt + koff[i]);
        s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>(x[0], x[1]), qb[2 * i], s[sub], 0, 0, 0);
        s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>(x[2], x[3]), qb[2 * i + 1], s[sub], 0, 0, 0);
      }
      if constexpr (UNI) {
        f[sub] = uniform(sc[sub * 32]) * a.scale_log2e;
        vs[sub] = uniform(sc[KT + sub * 32]);
      } else {
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const f32x4_t k4 = *reinterpret_cast<const f32x4_t*>(sc + sub * 32 + 8 * qd + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[sub][4 * qd + e] *= k4[e] * a.scale_log2e;
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
          col.raise(top16(s[sub]));
          col.weights_by_key(s[sub], vsk[UNI ? 0 : sub]);
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
  for (int x = 0; x < KS; ++x) m = fmaxf(m, reinterpret_cast<const float*>(rings + x * RING + 4 * SLOT)[lane]);
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    const float* o = reinterpret_cast<const float*>(rings + x * RING + 4 * SLOT);
    wgt[x] = __builtin_amdgcn_exp2f(o[lane] - m);              // 0 for a wave without keys
    l = fmaf(o[64 + lane], wgt[x], l);
  }
  float* pw = a.parts + (int64_t)it.part * part_wave_floats(D);
#pragma unroll
  for (int k = w; k < D / 8; k += KS) {
    f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int y = 0; y < KS; ++y) x += *reinterpret_cast<const f32x4_t*>(rings + y * RING + (k * 64 + lane) * 16) * wgt[y];
    if (it.part >= 0)
      *reinterpret_cast<f32x4_t*>(pw + (k * 64 + lane) * 4) = x;
    else
      store_out<D>(a, it.req, it.kvh, it.B, r, k, g, x, l);
  }
  if (it.part >= 0 && w == 0) {
    pw[D / 8 * 256 + lane] = m;
    pw[D / 8 * 256 + 64 + lane] = l;
  }
}

// ---------------------------------------------------------------- several row tiles: waves share the ring
// One wave a row tile; up to MAXW waves share the K/V tiles of a 4-stage ring.
template <int MAXW>
struct Shape {
  static constexpr int KT = 64;                   // keys per stage
  static constexpr int NS = 4;                    // stages
  static constexpr int NI = MAXW == 4 ? 2 : 4;    // waves that issue the DMA
};

template <int FMT, int D, int MAXW, bool UNI>
__global__ __launch_bounds__(64 * MAXW, 2) void k_qattn_group(QAttnArgs a) {
  using SH = Shape<MAXW>;
  constexpr int KT = SH::KT, NS = SH::NS, NI = SH::NI, SPT = KT / 32;
  constexpr int NKK = D / 16, NDT = D / 32, NC = D / 16, NCB = D / 8;
  constexpr int TILE = KT * D, STAGE = 2 * TILE;   // bytes: K tile, then V tile
  constexpr int RPB = 1024 / D;                    // rows per 1 KiB DMA block
  constexpr int RPI = KT / RPB / NI;               // blocks per tensor and issuing wave
  constexpr int PB = 2 * RPI + 1;                  // DMA instructions per stage and issuing wave
  constexpr int SCB = 2 * KT * 4;                  // bytes of a stage's scales
  static_assert(KT / RPB % NI == 0, "issuing waves split a tile evenly");
  __shared__ __align__(1024) uint8_t ring[NS * STAGE + NS * SCB];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x >= a.n_items) {
    const int u = ((int)blockIdx.x - a.n_items) * a.RTW + w;
    if (a.L > 32)
      quantize_block<FMT, D, D / 16>(a, u, threadIdx.x & 63);
    else
      quantize_block<FMT, D, D / 32>(a, u, threadIdx.x & 63);
    return;
  }
  const QItem it = a.items[blockIdx.x];
  const int lane = threadIdx.x & 63, g = lane >> 5, n = lane & 31, q16 = lane >> 4, j16 = lane & 15;
  const Keys<D> keys(a, it);
  const int B = it.B, pad = it.pad, nv = it.nv, v0 = it.v0, v1 = it.v1;
  const int ntiles = (v1 - v0 + KT - 1) / KT;
  const bool issuer = w < NI;
  const int r = (it.rt0 + w) * 32 + n;

  bf16x8_t qb[NKK];
  load_queries<D>(a, it, r, g, qb);

  const uint32_t ring_lds = __builtin_amdgcn_readfirstlane(lds_addr(ring));
  auto issue = [&](int u) {
    if (!issuer) return;
    const int slot = u % NS, vb = v0 + u * KT;
    const uint32_t sbase = ring_lds + (uint32_t)(slot * STAGE + w * 1024);
    const bool whole = keys.whole(vb, KT);
#pragma unroll
    for (int k = 0; k < 2 * RPI; ++k) {
      const int tensor = k / RPI, blk = k % RPI * NI;
      const int row = (blk + w) * RPB + lane / NC, chunk = (lane % NC) ^ swz8<D>(row);
      const uint32_t dst = sbase + (uint32_t)(tensor * TILE + blk * 1024);
      const uint8_t* cb = tensor ? keys.v : keys.k;
      if (whole)
        dma16_sv_once(dst, uniform64(cb + (int64_t)keys.cell(vb) * D), (uint32_t)(row * D + chunk * 16));
      else
        dma16_once(dst, cb + (int64_t)keys.cell(keys.clamp(vb + row)) * D + chunk * 16);
    }
    // scales by key: K's, then V's; of four issuing waves two fetch the same
    dma4(ring_lds + (uint32_t)(NS * STAGE + slot * SCB + (w & 1) * KT * 4),
         (w & 1 ? keys.vs : keys.ks) + keys.group(keys.clamp(vb + lane)));
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
    for (const int lim = min(NS - (2 * FT + STAGE - 1) / STAGE, min(NS - 1, ntiles)); issued < lim; ++issued) issue(issued);
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
    barrier();
  }
  for (const int lim = min(NS - 1, ntiles); issued < lim; ++issued) issue(issued);

  // LDS byte offsets of this lane's K and V reads (V rows 16 apart and K rows 32
  // apart have the same swizzle)
  int koff[D / 32], voff[NDT];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) koff[i] = n * D + (((2 * i + g) ^ swz8<D>(n)) * 16);
  const int vrow = ((j16 >> 1) & 3) + 4 * g + (j16 >= 8 ? 8 : 0);
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
    voff[dt] = TILE + vrow * D + (((2 * dt + (q16 & 1)) ^ swz8<D>(vrow)) * 16) + 8 * (j16 & 1);

  for (int u = 0; u < ntiles; ++u) {
    wait_stages(min(NS - 2, ntiles - 1 - u));
    barrier();
    if (u + NS - 1 < ntiles) issue(u + NS - 1);
    const int slot = u % NS;
#pragma unroll
    for (int sub = 0; sub < SPT; ++sub) {
      const int vb = v0 + u * KT + sub * 32;
      if (vb + 32 <= pad || vb >= v1) continue;              // wave-uniform
      const uint8_t* tile = ring + slot * STAGE + sub * 32 * D;
      const float* sc = reinterpret_cast<const float*>(ring + NS * STAGE + slot * SCB) + sub * 32;
      f32x16_t s;
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) s[rr] = 0.0f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const v4u x = *reinterpret_cast<const v4u*>(tile + koff[i]);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>(x[0], x[1]), qb[2 * i], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>(x[2], x[3]), qb[2 * i + 1], s, 0, 0, 0);
      }
      if constexpr (!UNI) {
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const f32x4_t k4 = *reinterpret_cast<const f32x4_t*>(sc + 8 * qd + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * qd + e] *= k4[e] * a.scale_log2e;
        }
      }
      if (vb < pad || vb + 32 > nv) {
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) {
          const int v = vb + key_of(rr, g);
          if (v < pad || v >= nv) s[rr] = -__builtin_inff();
        }
      }
      if constexpr (UNI) {
        const float f = uniform(sc[0]) * a.scale_log2e, vs = uniform(sc[KT]);
        col.raise(top16(s) * f);
        col.lsum = fmaf(col.weights(s, f, col.mrun - __builtin_amdgcn_logf(vs)), __builtin_amdgcn_rcpf(vs), col.lsum);
      } else {
        f32x4_t vs[4];
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) vs[qd] = *reinterpret_cast<const f32x4_t*>(sc + KT + 8 * qd + 4 * g);
        col.raise(top16(s));
        col.weights_by_key(s, vs);
      }
#pragma unroll
      for (int i = 0; i < 2 * NDT; ++i) {
        const i32x2_t x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(tile + voff[i % NDT] + i / NDT * 16 * D));
        col.o[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>((uint32_t)x[0], (uint32_t)x[1]), col.pp[i / NDT],
                                                                 col.o[i % NDT], 0, 0, 0);
      }
    }
  }

  col.lsum += __shfl_xor(col.lsum, 32, 64);
  // lane (g, n): O^T[feature 8 k + 4 g + e][query n]
  float* pw = a.parts + ((int64_t)it.part * a.RTW + w) * part_wave_floats(D);
#pragma unroll
  for (int k = 0; k < D / 8; ++k) {
    const f32x4_t x = {col.o[k >> 2][4 * (k & 3)], col.o[k >> 2][4 * (k & 3) + 1], col.o[k >> 2][4 * (k & 3) + 2], col.o[k >> 2][4 * (k & 3) + 3]};
    if (it.part >= 0)
      *reinterpret_cast<f32x4_t*>(pw + (k * 64 + lane) * 4) = x;
    else
      store_out<D>(a, it.req, it.kvh, B, r, k, g, x, col.lsum);
  }
  if (it.part >= 0) {
    pw[D / 8 * 256 + lane] = col.mrun;
    pw[D / 8 * 256 + 64 + lane] = col.lsum;
  }
}

// Joins the pieces of a split row: one wave per (row, row tile, group of 4
// features), folding the pieces' partials by their running maxima, eight loads in
// flight.
template <int D>
__global__ __launch_bounds__(256) void k_qattn_merge(QAttnArgs a) {
  constexpr int NG = D / 8, CH = kMergeBatch;
  const int wv = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  if (wv >= a.n_merge * a.RTW * NG) return;
  const int k = wv % NG, t = wv / NG % a.RTW;
  const QMerge mg = a.merges[wv / NG / a.RTW];
  const int64_t stride = (int64_t)a.RTW * part_wave_floats(D);
  const float* pw = a.parts + ((int64_t)mg.part0 * a.RTW + t) * part_wave_floats(D);
  f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
  float m = -__builtin_inff(), l = 0.0f;
  for (int p0 = 0; p0 < mg.nparts; p0 += CH) {
    float mp[CH], lp[CH];
    f32x4_t op[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const bool ok = p0 + i < mg.nparts;
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
  store_out<D>(a, mg.req, mg.kvh, mg.B, (mg.rt0 + t) * 32 + (lane & 31), k, lane >> 5, acc, l);
}

template <int FMT, int D>
void attend(const QAttnArgs& a, hipStream_t s) {
  auto go = [&](auto kernel, int waves) {
    const int wb = a.write_back ? (a.n * a.Hkv * 2 + waves - 1) / waves : 0;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.n_items + wb)), dim3((unsigned)(64 * waves)), 0, s, a);
  };
  auto by_groups = [&](auto uni_tag) {
    constexpr bool UNI = decltype(uni_tag)::value != 0;
    if (a.RTW > 4)
      go(k_qattn_group<FMT, D, 8, UNI>, a.RTW);
    else if (a.RTW > 1)
      go(k_qattn_group<FMT, D, 4, UNI>, a.RTW);
    else if (a.KS == 8)
      go(k_qattn_keys<FMT, D, 8, UNI>, 8);
    else if (a.KS == 4)
      go(k_qattn_keys<FMT, D, 4, UNI>, 4);
    else
      go(k_qattn_keys<FMT, D, 2, UNI>, 2);
  };
  a.lt >= 5 ? by_groups(QInt<1>{}) : by_groups(QInt<0>{});
  if (a.n_merge)
    hipLaunchKernelGGL(k_qattn_merge<D>, dim3((unsigned)((a.n_merge * a.RTW * (D / 8) + 3) / 4)), dim3(256), 0, s, a);
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
