// Building blocks of the packed kernels (pack_fwd.hpp, pack_dq.hpp,
// pack_dkdv.hpp): attention over a packed batch of graphs with capped scores,
// a prefix mask and dropout.
//
//   u_ij = scale q_i . k_j,   c_ij = cap tanh(u_ij / cap)   (u_ij without a cap)
//   S_ij = c_ij + table[h, spd_ij]
//   key j is visible to query i of its graph if j < max(prefix, i + nk - nq + 1)
//   P = softmax of S over the visible keys,   O_i = sum_j P_ij z_ij V_j / (1 - p)
// with z_ij in {0, 1} drawn by Philox4x32 (below) in every kernel that needs it.
//
// Layout. A wave has 32 stationary rows (lane & 31) and computes 32 x 32 score
// blocks whose streamed rows lie on the registers: lane half g (lane >> 5) holds
// streamed rows 16 g + r in register r, in the order that the next product
// takes them (perm32). Two policies give the products and the staging: Bf16Pack
// (v_mfma_f32_32x32x16_bf16) and F32Pack (v_mfma_f32_32x32x2_f32).
//
// Tiles of bf16 rows go straight to LDS, tiles of fp32 rows, whose LDS rows are
// padded, through registers.
#pragma once
#include <type_traits>

#include "common.hpp"
#include "f32_mfma.hpp"
#include "pack_plan.hpp"
#include "stage.hpp"

namespace gt {

// A tensor of heads x rows x d with unit feature stride (strides in elements).
struct PackTensor {
  void* p;
  int64_t hs, rs;
};

struct PackArgs {
  PackTensor q, k, v, o, d_o, dq, dk, dv;
  float* lse;               // [H, ld_lse]
  int64_t ld_lse;
  const uint8_t* spd;
  const float* table;       // [H, n_buckets]
  int32_t n_buckets, H;
  float scale, cap;
  int32_t thr;              // pairs whose signed 16 random bits are below it are dropped
  float rp;                 // 1 / (1 - p)
  uint32_t seed0, seed1, offset;
  const uint32_t* offset_dev;   // added to offset, or null
  const PackWave* jobs;     // 4 per job
  int32_t njobs;
  int32_t slots;            // key-stationary: workgroups per head
  int32_t hist;             // and buckets of its histogram, a power of two from n_buckets up
  const PackMerge* merges;
  int32_t nmerges;
  float* o_part;            // [slot, H, 32, d]
  float* lse_part;          // [slot, H, 32]
  float* dlt;               // [H, ld_dlt] rowsum(dO * O)
  int64_t ld_dlt;
  float2* dmax;             // [H, njobs_dq] of each job of the dQ kernel: largest |dS|, and largest
                            // correction of a row's D
  int32_t njobs_dq;
  double* dtab_part;        // [H, slots, n_buckets]
  float* dtable;            // [H, n_buckets]
};

namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int kPackThreads = kPackWaves * 64;
// Table entries at or below it are masks, as -inf. The backward takes P from the
// log-sum-exp, whose last bit grows with it: of a row whose entries are all near
// -6e4, P is off by 0.4 %, near -1e9 it would be off by powers of e^64.
constexpr float kNoScore = -6e4f;

// Wave-uniform values that the compiler took for divergent (a buffer resource of
// such is read lane by lane).
__device__ __forceinline__ bool uniform(bool x) { return __builtin_amdgcn_readfirstlane((int)x) != 0; }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const uint8_t*>((uint64_t)(uint32_t)uniform((int)(uint32_t)x) |
                                          (uint64_t)(uint32_t)uniform((int)(uint32_t)(x >> 32)) << 32);
}

// ---------------------------------------------------------------------------
// Philox4x32 with 7 rounds (Salmon et al., Parallel random numbers: as easy as
// 1, 2, 3, 2011: the fewest rounds that pass their whole battery; 10 is their
// margin). Counter (key / 8, packed query row, head, offset), key = seed: one
// draw gives the 8 keys of a row from a multiple of 8 on 16 bits each, key 2 w
// in the low half of word w. 16 bits place p within 2^-17, and the kept pairs
// are scaled by the exact inverse of the rate so placed.
//
// A 64-bit product costs some eight simple instructions, and a draw has 14. The
// counter's words meet only after two rounds: up to then each product goes by
// the row alone, or the keys alone, or neither. RowDraw and KeyDraw hold what the
// products of one side leave, made once per row and once per 8 keys; 9 products
// remain for the pair.
// ---------------------------------------------------------------------------
constexpr uint32_t kPhiloxM0 = 0xD2511F53u, kPhiloxM1 = 0xCD9E8D57u;
constexpr uint32_t kPhiloxW0 = 0x9E3779B9u, kPhiloxW1 = 0xBB67AE85u;
__device__ __forceinline__ uint32_t mul_hi_lo(uint32_t x, uint32_t m, uint32_t& lo) {
  const uint64_t y = (uint64_t)x * m;
  lo = (uint32_t)y;
  return (uint32_t)(y >> 32);
}

struct RowDraw { uint32_t xh, xl; };             // second round's product of the row's word
struct Philox {
  uint32_t k0, k1, offset;                       // (wave-uniform)
  uint32_t hh, hl;                               // first round's product of the head's word
  __device__ __forceinline__ Philox(const PackArgs& a, int h)
      : k0(a.seed0), k1(a.seed1), offset(a.offset + (a.offset_dev ? *a.offset_dev : 0u)) {
    hh = mul_hi_lo((uint32_t)h, kPhiloxM1, hl);
  }
  __device__ __forceinline__ RowDraw row(uint32_t packed_row) const {
    RowDraw r;
    r.xh = mul_hi_lo(hh ^ packed_row ^ k0, kPhiloxM0, r.xl);
    return r;
  }
  // Keys 8 j8 .. + 7: what the third round takes of the first two, and its own
  // product of the first word.
  __device__ __forceinline__ uint4 keys(uint32_t j8) const {
    uint4 k;
    uint32_t x1, y2, x3;
    const uint32_t c2 = mul_hi_lo(j8, kPhiloxM0, x1) ^ offset ^ k1;
    const uint32_t c0 = mul_hi_lo(c2, kPhiloxM1, y2) ^ hl ^ (k0 + kPhiloxW0);
    k.z = mul_hi_lo(c0, kPhiloxM0, x3) ^ (k1 + 2u * kPhiloxW1);
    k.x = x1 ^ (k1 + kPhiloxW1);
    k.y = y2 ^ (k0 + 2u * kPhiloxW0);
    k.w = x3;
    return k;
  }
  __device__ __forceinline__ void draw(const RowDraw& r, const uint4& k, uint32_t* w) const {
    uint32_t c1, c0 = mul_hi_lo(r.xh ^ k.x, kPhiloxM1, c1) ^ k.y, c2 = r.xl ^ k.z, c3 = k.w;
#pragma unroll
    for (uint32_t i = 3; i < 7; ++i) {
      uint32_t x, y;
      const uint32_t n0 = mul_hi_lo(c2, kPhiloxM1, y) ^ c1 ^ (k0 + i * kPhiloxW0);
      c2 = mul_hi_lo(c0, kPhiloxM0, x) ^ c3 ^ (k1 + i * kPhiloxW1);
      c0 = n0;
      c1 = y;
      c3 = x;
    }
    w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
  }
};
// Pair r of 16 (two draws).
__device__ __forceinline__ bool kept(const uint32_t (&w)[8], int r, int thr) {
  return (int)(int16_t)(w[r >> 1] >> (16 * (r & 1))) >= thr;
}
// The same of a word's two pairs: all ones in the halves of the kept ones (the
// saturating difference keeps its sign; below: thr - 1 in both halves).
__device__ __forceinline__ uint32_t kept2(uint32_t w, uint32_t below) {
  const s16x2 d = __builtin_elementwise_sub_sat(__builtin_bit_cast(s16x2, below), __builtin_bit_cast(s16x2, w));
  return __builtin_bit_cast(uint32_t, (s16x2)(d >> (short)15));
}

// ---------------------------------------------------------------------------
// Scores. Units: bf16 works in base 2 (x = S log2 e), fp32 in S itself.
// ---------------------------------------------------------------------------
struct ScoreConst {
  float mul;                // bf16: uncapped score = s mul; capped: e^(2 u / cap) = 2^(s mul)
  float add;                // bf16, capped: score = cap log2 e - add / (e^(2 u / cap) + 1)
  float cap;                // fp32
};

// Capped scores are bounded, and with them, table and all, the exponents: where
// they span at most kSpan, the forward's softmax needs no running reference but takes
// one for the whole head, `ref`, which the table's entries carry: no addition per
// score, no test per block, and no rescaling. It is 0 where that keeps the exponents
// within kTop - kSpan .. kTop (a table around 0), so that an entry is the backward's to
// the last bit; else a whole number that does. exp stays within 2^-91 .. 2^70: sums over n
// keys of values below 2^57 / n are finite, and of a row whose scores are all at the low end,
// values from 2^-35 on keep all their bits. (A cap of 50 spans 144; 16 are left for the
// biases.)
constexpr float kSpan = 160.0f, kTop = 70.0f;
struct ScoreRef {
  bool fixed;
  float ref;
};
// The largest of a wave's values, wave-uniform (NaN passed over): within rows of 16
// lanes by DPP, a hop of some cycles where one through LDS takes a hundred.
__device__ __forceinline__ float wave_max(float x) {
  const auto hop = [&](auto ctrl) {
    const int y = __builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true);
    x = fmaxf(x, __int_as_float(y));
  };
  hop(std::integral_constant<int, 0xB1>{});        // quad_perm 1 0 3 2
  hop(std::integral_constant<int, 0x4E>{});        // quad_perm 2 3 0 1
  hop(std::integral_constant<int, 0x141>{});       // row_half_mirror
  hop(std::integral_constant<int, 0x140>{});       // row_mirror
  const int v = __float_as_int(x);
  return fmaxf(fmaxf(__int_as_float(__builtin_amdgcn_readlane(v, 0)), __int_as_float(__builtin_amdgcn_readlane(v, 16))),
               fmaxf(__int_as_float(__builtin_amdgcn_readlane(v, 32)), __int_as_float(__builtin_amdgcn_readlane(v, 48))));
}

// Thread t's of the head's 256 entries (bias log2 e; 0 past the table) as bf16 capped
// scores take them, and the reference. Every wave looks at all of them: no exchange.
template <class M>
__device__ __forceinline__ float capped_entry(const PackArgs& a, int h, ScoreRef& r) {
  const int lane = threadIdx.x & 63, wave = wave_id();
  const float cap2 = a.cap * kLog2e;
  float own = 0.0f, hi = -INFINITY, lo = INFINITY;
#pragma unroll
  for (int w = 0; w < kPackWaves; ++w) {
    const int b = w * 64 + lane;
    const float e = M::entry(b < a.n_buckets ? a.table[(int64_t)h * a.n_buckets + b] : 0.0f, a, false);
    hi = fmaxf(hi, e == -INFINITY ? hi : e);
    lo = fminf(lo, e == -INFINITY ? lo : e);
    own = wave == w ? e : own;
  }
  hi = wave_max(hi);
  lo = -wave_max(-lo);
  r.fixed = hi >= lo && hi - lo + 2.0f * cap2 <= kSpan;      // (not if all entries are masks)
  const bool centred = hi + cap2 <= kTop && lo - cap2 >= kTop - kSpan;
  r.ref = r.fixed && !centred ? ceilf(hi + cap2 - kTop) : 0.0f;
  return (own + cap2) - r.ref;
}

// D: the tile's head dim (32 or 64); DS <= D: the tensors'.
template <int D_, int DS_>
struct Bf16Pack {
  static constexpr int D = D_, DS = DS_;
  static constexpr bool BF16 = true;
  using T = uint16_t;
  static constexpr int NA = D / 32;                  // accumulators of D x 32
  static constexpr int TILE = 32 * D;                // elements of a wave's staged rows
  static constexpr int CPR = D / 8;                  // 16-byte chunks per row
  static constexpr int DCH = DS / 8;                 // of them with data
  struct Operand { bf16x8 f[D / 16]; };

  __device__ __forceinline__ static int lds_off(int row, int ch) { return row * D + swz_tile<D>(row, ch) * 8; }

  // The lane's stationary row (features past DS zero), times a power of two.
  __device__ __forceinline__ static void load_operand(const T* row, bool ok, float mul, Operand& x) {
    const int g = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int kc = 0; kc < D / 16; ++kc)
      x.f[kc] = ok && kc * 16 + g * 8 < DS ? *reinterpret_cast<const bf16x8*>(row + kc * 16 + g * 8) : zero_bf16x8();
    if (mul != 1.0f) {
#pragma unroll
      for (int kc = 0; kc < D / 16; ++kc)
#pragma unroll
        for (int e = 0; e < 8; ++e) x.f[kc][e] = (__bf16)((float)x.f[kc][e] * mul);
    }
  }
  // Dot product of two operands' features in this lane half.
  __device__ __forceinline__ static float dot(const Operand& x, const Operand& y) {
    float s = 0.0f;
#pragma unroll
    for (int kc = 0; kc < (DS + 15) / 16; ++kc)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf((float)x.f[kc][e], (float)y.f[kc][e], s);
    return s;
  }
  __device__ __forceinline__ static void rows(const T* tile, const Operand& x, f32x16& s) {
#pragma unroll
    for (int kc = 0; kc < (DS + 15) / 16; ++kc) s = mfma32(lds_b128(tile + row_operand_off<D>(kc)), x.f[kc], s);
  }
  __device__ __forceinline__ static void cols(const T* tile, const bf16x8& p0, const bf16x8& p1, f32x16 (&acc)[NA]) {
#pragma unroll
    for (int cb = 0; cb < NA; ++cb) {
      const int o0 = tr_operand_off<D>(0, cb), o1 = tr_operand_off<D>(1, cb);
      acc[cb] = mfma32(lds_tr_operand(tile, o0, o1), p0, acc[cb]);
      acc[cb] = mfma32(lds_tr_operand(tile + 8 * D, o0, o1), p1, acc[cb]);
    }
  }
  __device__ __forceinline__ static void cols(const T* tile, const float (&p)[16], f32x16 (&acc)[NA]) {
    cols(tile, cvt_bf16x8(p), cvt_bf16x8(p + 8), acc);
  }
  // Two products of one tile.
  __device__ __forceinline__ static void cols2(const T* tile, const float (&p)[16], f32x16 (&acc)[NA],
                                               const float (&q)[16], f32x16 (&acc2)[NA]) {
    const bf16x8 p0 = cvt_bf16x8(p), p1 = cvt_bf16x8(p + 8), q0 = cvt_bf16x8(q), q1 = cvt_bf16x8(q + 8);
#pragma unroll
    for (int cb = 0; cb < NA; ++cb) {
      const int o0 = tr_operand_off<D>(0, cb), o1 = tr_operand_off<D>(1, cb);
      const bf16x8 t0 = lds_tr_operand(tile, o0, o1), t1 = lds_tr_operand(tile + 8 * D, o0, o1);
      acc[cb] = mfma32(t0, p0, acc[cb]);
      acc2[cb] = mfma32(t0, q0, acc2[cb]);
      acc[cb] = mfma32(t1, p1, acc[cb]);
      acc2[cb] = mfma32(t1, q1, acc2[cb]);
    }
  }
  // Both of p's products' bf16 operand with the dropped pairs (16 draws' bits) zero.
  __device__ __forceinline__ static void cols_kept(const T* tile, const float (&p)[16], const uint32_t (&w)[8],
                                                   uint32_t below, int, f32x16 (&acc)[NA]) {
    uint4 x = __builtin_bit_cast(uint4, cvt_bf16x8(p)), y = __builtin_bit_cast(uint4, cvt_bf16x8(p + 8));
    x.x &= kept2(w[0], below); x.y &= kept2(w[1], below); x.z &= kept2(w[2], below); x.w &= kept2(w[3], below);
    y.x &= kept2(w[4], below); y.y &= kept2(w[5], below); y.z &= kept2(w[6], below); y.w &= kept2(w[7], below);
    cols(tile, __builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc);
  }
  // put(feature, 4 values) for the lane's column.
  template <typename F>
  __device__ __forceinline__ static void features(const f32x16 (&acc)[NA], F put) {
    const int g = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int cb = 0; cb < NA; ++cb)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = cb * 32 + 8 * u + 4 * g;
        if (c < DS) put(c, make_float4(acc[cb][4 * u], acc[cb][4 * u + 1], acc[cb][4 * u + 2], acc[cb][4 * u + 3]));
      }
  }
  __device__ __forceinline__ static void store4(T* p, float4 v) {
    uint2 pk;
    pk.x = (uint32_t)f2bf(v.x) | ((uint32_t)f2bf(v.y) << 16);
    pk.y = (uint32_t)f2bf(v.z) | ((uint32_t)f2bf(v.w) << 16);
    *reinterpret_cast<uint2*>(p) = pk;
  }

  __device__ __forceinline__ static float operand_mul(const PackArgs&, bool) { return 1.0f; }
  __device__ __forceinline__ static ScoreConst consts(const PackArgs& a, bool cap) {
    ScoreConst c{};
    c.mul = a.scale * kLog2e * (cap ? 2.0f / a.cap : 1.0f);
    c.add = 2.0f * a.cap * kLog2e;
    return c;
  }
  // Table entry in LDS: bias log2 e, or, as the start of the score accumulator,
  // bias / scale.
  __device__ __forceinline__ static float entry(float bias, const PackArgs& a, bool start) {
    return bias <= kNoScore ? -INFINITY : (start ? bias / a.scale : bias * kLog2e);
  }
  // x = S log2 e from the products s and the entries in x (which hold the cap's
  // log2 e too, cap tanh(u / cap) = cap - 2 cap / (e^(2 u / cap) + 1); uncapped: s holds
  // them already). SLOPE: slope = -dc/du / 4. (The exponential and the reciprocal run
  // at half rate: a polynomial for scores below 3/4 of the cap, 7 instructions, was
  // no faster.)
  template <bool CAP, bool SLOPE>
  __device__ __forceinline__ static void scores(const f32x16& s, float (&x)[16], float (&slope)[16],
                                                const ScoreConst& c) {
    static_assert(CAP, "uncapped scores come out of the product");
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e = __builtin_amdgcn_rcpf(-1.0f - exp2_fast(s[r] * c.mul));
      if constexpr (SLOPE) slope[r] = fmaf(e, e, e);               // 1 - tanh^2 = -4 (e^2 + e)
      x[r] = fmaf(e, c.add, x[r]);
    }
  }
  // What the sums of slope times anything are multiplied by.
  static constexpr float kSlope = -4.0f;
  __device__ __forceinline__ static float expo(float x) { return exp2_fast(x); }
  __device__ __forceinline__ static float to_unit(float lse) { return lse * kLog2e; }
  __device__ __forceinline__ static float log_sum(float m, float l) { return (m + __log2f(l)) * kLn2; }
};

template <int D_>
struct F32Pack {
  static constexpr int D = D_, DS = D_;
  static constexpr bool BF16 = false;
  using T = float;
  static constexpr int NA = kBlocksF<D>;
  static constexpr int TILE = 32 * kRowF<D>;
  static constexpr int CPR = D / 4;
  static constexpr int DCH = CPR;
  struct Operand { float f[D / 2]; };

  __device__ __forceinline__ static int lds_off(int row, int ch) { return row * kRowF<D> + ch * 4; }
  __device__ __forceinline__ static void load_operand(const T* row, bool ok, float mul, Operand& x) {
    const int g = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      const float4 v = ok ? *reinterpret_cast<const float4*>(row + 8 * c + 4 * g) : make_float4(0.f, 0.f, 0.f, 0.f);
      x.f[4 * c] = v.x * mul;
      x.f[4 * c + 1] = v.y * mul;
      x.f[4 * c + 2] = v.z * mul;
      x.f[4 * c + 3] = v.w * mul;
    }
  }
  __device__ __forceinline__ static float dot(const Operand& x, const Operand& y) {
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < D / 2; ++e) s = fmaf(x.f[e], y.f[e], s);
    return s;
  }
  __device__ __forceinline__ static void rows(const T* tile, const Operand& x, f32x16& s) {
    product_rows<D>(tile, x.f, s);
  }
  __device__ __forceinline__ static void cols(const T* tile, const float (&p)[16], f32x16 (&acc)[NA]) {
    product_cols<D>(tile, p, acc);
  }
  __device__ __forceinline__ static void cols_kept(const T* tile, const float (&p)[16], const uint32_t (&w)[8],
                                                   uint32_t, int thr, f32x16 (&acc)[NA]) {
    float z[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = kept(w, r, thr) ? p[r] : 0.0f;
    cols(tile, z, acc);
  }
  template <typename F>
  __device__ __forceinline__ static void features(const f32x16 (&acc)[NA], F put) { for_features<D>(acc, put); }
  __device__ __forceinline__ static void store4(T* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }

  // The stationary operand of the score product carries scale (/ cap).
  __device__ __forceinline__ static float operand_mul(const PackArgs& a, bool cap) {
    return cap ? a.scale / a.cap : a.scale;
  }
  __device__ __forceinline__ static ScoreConst consts(const PackArgs& a, bool) {
    ScoreConst c{};
    c.cap = a.cap;
    return c;
  }
  __device__ __forceinline__ static float entry(float bias, const PackArgs&, bool) {
    return bias <= kNoScore ? -INFINITY : bias;
  }
  // x = S. (The entries are added after the product: as the accumulator's start they
  // would raise the rounding of every step.) tanh(y) / y is a polynomial in y^2 up to
  // |y| = 0.75, off by 3e-8 of it (fitted to the least largest relative error); beyond,
  // 1 - 2 / (e^(2 y) + 1) is off by about 2^-23 against a value of at least 0.63. Blocks
  // whose scores all stay below take the polynomial alone.
  template <bool CAP, bool SLOPE>
  __device__ __forceinline__ static void scores(const f32x16& s, float (&x)[16], float (&slope)[16],
                                                const ScoreConst& c) {
    if constexpr (!CAP) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] += s[r];
      return;
    }
    float top = 0.0f, t[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float y = s[r], z = y * y;
      const float k = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -0.00471626f, 0.01958291f), -0.05334443f), 0.13325406f),
                                   -0.33332959f), 0.99999997f);
      t[r] = y * k;
      top = fmaxf(top, z);
    }
    if (__any(!(top <= 0.5625f))) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float y = fabsf(s[r]);
        const float big = fmaf(-2.0f, __builtin_amdgcn_rcpf(exp2_fast(y * (2.0f * kLog2e)) + 1.0f), 1.0f);
        t[r] = y <= 0.75f ? t[r] : copysignf(big, s[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if constexpr (SLOPE) slope[r] = fmaf(-t[r], t[r], 1.0f);
      x[r] = fmaf(c.cap, t[r], x[r]);
    }
  }
  static constexpr float kSlope = 1.0f;
  __device__ __forceinline__ static float expo(float x) { return exp2_fast(x * kLog2e); }
  __device__ __forceinline__ static float to_unit(float lse) { return lse; }
  __device__ __forceinline__ static float log_sum(float m, float l) { return m + logf(l); }
};

// ---------------------------------------------------------------------------
// Staging: 32 rows of one tensor per wave, global -> registers -> LDS.
// ---------------------------------------------------------------------------
template <class M>
struct PackStage {
  static constexpr int N = 32 * M::CPR / 64;         // 16-byte chunks per lane
  uint4 r[N];
  // Rows [r0, r0 + 32) of a graph's `rows` rows from p on (rows past them zero).
  __device__ __forceinline__ void load(const typename M::T* p, int64_t rs, int64_t r0, int64_t rows) {
    constexpr int ES = sizeof(typename M::T);
    const int64_t n = rows - r0 < 32 ? rows - r0 : 32;
    const uint32_t rsb = (uint32_t)rs * ES;
    const __amdgpu_buffer_rsrc_t rc = make_rsrc_n(p + r0 * rs, n > 0 ? (n - 1) * (int64_t)rsb + M::DS * ES : 0);
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * 64 + lane, row = u / M::CPR, ch = u % M::CPR;
      r[i] = buf_b128(rc, ch < M::DCH ? (uint32_t)row * rsb + (uint32_t)ch * 16u : kZeroChunk);
    }
  }
  __device__ __forceinline__ void store(typename M::T* tile) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * 64 + lane;
      opaque(r[i]);
      *reinterpret_cast<uint4*>(tile + M::lds_off(u / M::CPR, u % M::CPR)) = r[i];
    }
  }
};

// bf16: straight to LDS (buffer_load_dwordx4 ... lds), 1 KiB per instruction; the
// lane that fills chunk c of a row reads the chunk that the swizzle keeps there.
template <class M>
struct PackDma {
  static constexpr int ROWB = M::D * 2;
  static constexpr int N = 32 * ROWB / 1024;         // instructions per tile
  uint32_t voff[N];
  __device__ __forceinline__ explicit PackDma(int64_t rs) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * 64 + lane, row = u / M::CPR;
      const int ch = swz_tile<M::D>(row, u % M::CPR);
      voff[i] = ch < M::DCH ? (uint32_t)row * ((uint32_t)rs * 2u) + (uint32_t)ch * 16u : kZeroChunk;
    }
  }
  // Rows [r0, r0 + 32) of a graph's `rows` rows from p on (rows past them zero).
  __device__ __forceinline__ void load(const uint16_t* p, int64_t rs, int64_t r0, int64_t rows, uint16_t* tile) const {
    const int64_t n = rows - r0 < 32 ? rows - r0 : 32;
    const __amdgpu_buffer_rsrc_t rc = make_rsrc_n(p + r0 * rs, n > 0 ? (n - 1) * rs * 2 + M::DS * 2 : 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // (device pass only: see TileDma)
#if __HIP_DEVICE_COMPILE__
      typedef __attribute__((address_space(3))) void* lds_void;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rc, (lds_void)(void*)(tile + i * 512), 16, voff[i], 0, 0, 0);
#else
      (void)rc;
      (void)tile;
#endif
    }
  }
};

// The workgroup's job and head, of `jobs` and a.H. Workgroups go to the 8 XCDs
// round robin: with many jobs, a job's heads, which share its distances, stay on
// one XCD, and the jobs, longest first, are dealt over the XCDs in turn.
constexpr int kXcdJobs = 64;
__host__ __device__ inline unsigned pack_grid(int jobs, int H) {
  return jobs >= kXcdJobs ? (unsigned)((jobs + 7) / 8 * 8) * (unsigned)H : (unsigned)jobs * (unsigned)H;
}
struct PackPlace {
  int job, h;
  __device__ __forceinline__ PackPlace(const PackArgs& a, int jobs) {
    const int w = (int)blockIdx.x;
    if (jobs >= kXcdJobs) {
      const int i = w >> 3;
      h = i % a.H;
      job = i / a.H * 8 + (w & 7);
    } else {
      h = w % a.H;
      job = w / a.H;
    }
  }
};

// A record of the plan in scalar registers.
template <typename T>
__device__ __forceinline__ T scalar_record(const T* p) {
  T r = *p;
  int w[sizeof(T) / 4];
  __builtin_memcpy(w, &r, sizeof(T));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i) w[i] = uniform(w[i]);
  __builtin_memcpy(&r, w, sizeof(T));
  return r;
}

template <typename T>
__device__ __forceinline__ T* rows_at(const PackTensor& t, int h, int64_t row) {
  return reinterpret_cast<T*>(t.p) + h * t.hs + row * t.rs;
}

// x[r] where r < rem, else fill.
__device__ __forceinline__ void keep_below(float (&x)[16], int rem, float fill) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = r < rem ? x[r] : fill;
}

// The distances of a query-stationary wave: the lane's row, groups of 16 keys
// from key j (wave-uniform) + 16 g on, at any address.
struct PackSpdRow {
  const uint8_t* base;
  int range;
  uint32_t voff, sh;
  // first: the wave's first row; rows: the query rows from there on (at least 1);
  // nk: the keys, 0 where there is nothing to read (all loads then give 0).
  __device__ __forceinline__ PackSpdRow(const uint8_t* first, int64_t ld, int64_t rows, int nk) {
    const int lane = threadIdx.x & 63;
    const int64_t n = rows < 32 ? rows : 32;
    const uint32_t rem = (uint32_t)(reinterpret_cast<uintptr_t>(first) & 15u);
    const int64_t i = (lane & 31) < n ? (lane & 31) : n - 1;
    base = uniform(first - rem);
    range = uniform(rsrc_range(nk > 0 ? ((n - 1) * ld + nk + rem + 3) & ~(int64_t)3 : 0));
    voff = (uint32_t)(i * ld) + 16u * (uint32_t)(lane >> 5) + rem;
    sh = voff & 3u;
    voff -= sh;
  }
  __device__ __forceinline__ void fetch(int j, uint32_t (&w)[5]) const {
    load_spd5(make_rsrc_from(base, range, j), voff, w);
  }
};

// Bias entries of the lane's 16 distances.
__device__ __forceinline__ void bias16(const float* tab, const uint32_t* w, float (&b)[16]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) b[r] = tab[(w[r >> 2] >> (8 * (r & 3))) & 0xffu];
}

// Terms of the table gradient: floor(x + 0.5) for even r, -floor(0.5 - x), added by
// subtraction, for odd r. The instruction rounds ties up, and ties are a quarter of all
// values between 2^21 and 2^22 and half of those up to 2^23: with one direction for all
// the bias grows with the pairs where the sum grows with their root (7651 nodes: the
// table gradient off by 3e-5 against 1e-6). Rounding to even takes one
// instruction more per pair (16384 nodes, d = 64: 2151 us, 2125 so).
template <int ODD>
__device__ __forceinline__ void add_term(unsigned long long* at, float x) {
  int r;
  if constexpr (ODD) {
    asm("v_cvt_rpi_i32_f32 %0, -%1" : "=v"(r) : "v"(x));
    __hip_atomic_fetch_sub(at, (unsigned long long)(long long)r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  } else {
    asm("v_cvt_rpi_i32_f32 %0, %1" : "=v"(r) : "v"(x));
    __hip_atomic_fetch_add(at, (unsigned long long)(long long)r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
}

// Buckets of the table gradient's histogram, and its bytes: 32 copies and one more
// bucket, or 16 copies of 256.
inline int hist_buckets(int n_buckets) { return n_buckets <= 32 ? 32 : (n_buckets <= 64 ? 64 : (n_buckets <= 128 ? 128 : 256)); }
inline int hist_bytes(int n_buckets) {
  const int n = hist_buckets(n_buckets);
  return n == 256 ? 256 * 16 * 8 : (n + 1) * 32 * 8;
}

// Workgroups of the bf16 dK / dV kernel on a compute unit.
inline int dkdv_resident(int d, bool cap, bool drop, int n_buckets) {
  return d <= 32 && !(cap && drop) && n_buckets <= 64 ? 3 : 2;
}
// Workgroups of the one-pass backward of short graphs on a compute unit, by registers
// and LDS: they are as many as fit, and take job after job.
constexpr int short_lds(int D, int blocks) { return 1024 + kPackWaves * (3 * 32 * D * 2 + blocks * 32 * 32 * 2 + 8); }
inline int short_resident(int d, int blocks, bool cap, bool drop, int n_buckets) {
  const int lds = short_lds(d == 64 ? 64 : 32, blocks) + hist_bytes(n_buckets);
  const int by_lds = 160 * 1024 / lds, by_registers = d == 64 || blocks == 4 || (cap && drop) ? 2 : 3;
  return by_lds < by_registers ? by_lds : by_registers;
}

// Adds up the accumulators of groups that have the same rows (wave gw of group
// ks into wave gw of group 0), pairwise and in a fixed order. buf: two waves'
// accumulators. on_write(slot) and weights(slot, wa, wo) as in combine_groups.
template <int NA, typename W, typename R>
__device__ __forceinline__ void pack_combine(float* buf, int log2w, int ks, int gw, f32x16 (&acc)[NA], W on_write, R weights) {
  constexpr int XW = NA * 16 * 64;
  const int lane = threadIdx.x & 63;
  for (int half = (kPackWaves >> log2w) / 2; half >= 1; half >>= 1) {
    __syncthreads();
    if (ks >= half && ks < 2 * half) {
      const int slot = ((ks - half) << log2w) + gw;
      float4* x = reinterpret_cast<float4*>(buf + slot * XW) + lane;
      on_write(slot);
#pragma unroll
      for (int c = 0; c < NA; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          x[(c * 4 + u) * 64] = make_float4(acc[c][4 * u], acc[c][4 * u + 1], acc[c][4 * u + 2], acc[c][4 * u + 3]);
    }
    __syncthreads();
    if (ks < half) {
      const int slot = (ks << log2w) + gw;
      const float4* x = reinterpret_cast<const float4*>(buf + slot * XW) + lane;
      float wa, wo;
      weights(slot, wa, wo);
#pragma unroll
      for (int c = 0; c < NA; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float4 y = x[(c * 4 + u) * 64];
          acc[c][4 * u] = fmaf(acc[c][4 * u], wa, y.x * wo);
          acc[c][4 * u + 1] = fmaf(acc[c][4 * u + 1], wa, y.y * wo);
          acc[c][4 * u + 2] = fmaf(acc[c][4 * u + 2], wa, y.z * wo);
          acc[c][4 * u + 3] = fmaf(acc[c][4 * u + 3], wa, y.w * wo);
        }
    }
  }
}

}  // namespace

// Launchers (hipError_t of the launch). BF16 inputs of head dim d, with or
// without a cap and dropout.
hipError_t launch_pack_fwd_bf16(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s);
hipError_t launch_pack_fwd_f32(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s);
hipError_t launch_pack_dq_bf16(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s);
hipError_t launch_pack_dq_f32(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s);
hipError_t launch_pack_dkdv_bf16(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s);
hipError_t launch_pack_dkdv_f32(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s);
// The whole backward of a batch of short graphs but for the sum of the table gradient.
// blocks: of 32 rows that a graph has at most, 2, or 4 (d <= 32).
hipError_t launch_pack_short_bf16(const PackArgs& a, int d, int blocks, bool cap, bool drop, hipStream_t s);
hipError_t launch_pack_merge(const PackArgs& a, int d, bool bf16, hipStream_t s);
hipError_t launch_pack_dtable(const PackArgs& a, hipStream_t s);

}  // namespace gt
