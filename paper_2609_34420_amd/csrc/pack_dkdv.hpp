// dK, dV and the table gradient of packed attention (instantiated in
// pack_dkdv_*.hip).
//
// Key-stationary: a wave has 32 keys and streams the graph's queries through
// S = Q K^T and dP = dO V^T, so a lane owns one key and 16 queries of a block:
//   dV^T += dO^T (z P),   dK^T += Q^T dU,   dU = P (z dP / (1 - p) - D)(1 - tanh^2),
// with P and dU taken from registers (1 / (1 - p) and scale at the end).
//
// Dropout: a lane draws for one query and 16 keys, as the query-stationary kernels
// do (a draw serves 8 keys of one row); the kept pairs, a byte each, are transposed
// through LDS with the 8-bit transposing reads, as the distances are. In dS the
// 1 / (1 - p) of dP is left out: dS (1 - p) = P (z dP - D (1 - p)).
//
// Table gradient: dS is added into an LDS histogram in fixed point, 64-bit sums of
// round(dS 2^F) (float adds to LDS are some twenty times slower), in 32 copies
// (lane & 31) of 32, 64 or 128 buckets or 16 of 256. F comes from the largest
// |dS| that the dQ kernel met in this head, so that every term stays below 2^31
// and the rounding of 2^-31 of it is far below the sums in fp32; V's operand and
// the staged D carry it, so that dS arrives scaled. Each workgroup writes its
// sums; a last kernel adds them in a fixed order. Everything is bitwise
// reproducible.
//
// P and dU are rounded to bf16 as the operands of their products (2^-8 of a term).
//
// Bound: dependent chains (LDS reads, product, exponentials, product, LDS adds) at two
// waves per SIMD, which the registers leave at d = 64 (253 of 256): vector units busy
// 62 %, LDS 19 % (16384 nodes, H = 8, d = 64, cap: 1960 to 2100 us, 530 to 560 TFLOP/s;
// without the histogram's adds 1840); at three 74 % and 19 % (d <= 32). Two buffers of tiles
// spill: 2180 against 2115.
#pragma once
#include "pack.hpp"

namespace gt {

namespace {

// 32 x 32 bytes of a wave, 16 per lane row by row (lane l: row l / 2, from column
// 16 (l & 1) on, or row l & 31, from column 16 (l >> 5) on), to the lane's column
// (lane & 31), rows 16 g + 0 .. 15.
__device__ __forceinline__ void transpose_bytes(uint8_t* st, int at, uint4 v, const int (&off_tr8)[2], uint32_t (&b)[4]) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2* lds_i32x2;
  *reinterpret_cast<uint4*>(st + at) = v;
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)(void*)(st + off_tr8[hh]));
    b[2 * hh] = (uint32_t)x.x;
    b[2 * hh + 1] = (uint32_t)x.y;
  }
}

// Three waves per SIMD: bf16 at d <= 32 but for cap and dropout together, whose registers
// spill, with up to 64 buckets, more of which leave LDS for two workgroups. One buffer of
// tiles then, two where two workgroups run (512 graphs of 100 to 256 nodes, d = 8,
// dropout: 161 us with two waves, 142 with three; 16 graphs of up to 2400, d = 32, cap:
// 133 and 126; 64 of 50 to 1000 with cap and dropout: 92 and 95).
template <class M>
constexpr bool three_waves(bool cap, bool drop) { return M::BF16 && M::D == 32 && !(cap && drop); }

// BUCKETS: of the histogram's layout, up to 64, 128 or 256 (WIDE, which has an entry for
// every byte; a narrow one has one more bucket for the bytes past it).
template <class M, bool CAP, bool DROP, int BUCKETS>
__global__ __launch_bounds__(kPackThreads, (three_waves<M>(CAP, DROP) && BUCKETS == 64 ? 3 : (M::BF16 || M::D < 64 ? 2 : 1)))
void pack_dkdv_kernel(PackArgs a) {
  using T = typename M::T;
  constexpr int NA = M::NA;
  constexpr bool WIDE = BUCKETS == 256;
  constexpr int NB = M::BF16 && M::D == 32 && !(three_waves<M>(CAP, DROP) && BUCKETS == 64) ? 2 : 1;   // staged tiles
  constexpr int XCH = NA * 16 * 64 * 4 * 2;
  constexpr int STG = 2 * kPackWaves * M::TILE * (int)sizeof(T);
  constexpr int CPY = WIDE ? 16 : 32;
  // (LDS objects are placed by decreasing alignment: the table first, where a DS
  // immediate of 16 bits reaches it)
  extern __shared__ unsigned long long hist[];            // a.hist buckets of CPY copies
  __shared__ alignas(4096) float sTab[256];
  __shared__ alignas(1024) uint8_t sByte[kPackWaves][1024];
  __shared__ alignas(512) float sStat[NB][kPackWaves][64]; // per staged row: -LSE; D (1 - p) 2^F, negative without dropout
  __shared__ alignas(128) uint8_t sBuf0[STG > XCH ? STG : XCH];
  __shared__ alignas(128) uint8_t sBuf1[NB == 2 ? STG : 16];
  __shared__ float red[2][kPackWaves];
  __shared__ int bad[kPackWaves];

  const PackPlace pl(a, a.slots);
  if (pl.job >= a.slots) return;
  const int h = pl.h;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, col = lane & 31, g = lane >> 5;
  sTab[tid] = M::entry(tid < a.n_buckets ? a.table[(int64_t)h * a.n_buckets + tid] : 0.0f, a, false)
              + (M::BF16 && CAP ? a.cap * kLog2e : 0.0f);
  for (int t = tid; t < a.n_buckets * CPY / 2; t += kPackThreads)
    reinterpret_cast<uint4*>(hist)[t] = make_uint4(0u, 0u, 0u, 0u);
  {
    // (four loads in flight: one after the other they took a third of a short
    // workgroup's time)
    const float2* dm = a.dmax + (int64_t)h * a.njobs_dq;
    float x = 0.0f, y = 0.0f;
    for (int t = tid; t < a.njobs_dq; t += 4 * kPackThreads) {
      float2 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = t + k * kPackThreads;
        v[k] = dm[i < a.njobs_dq ? i : t];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x = fmaxf(x, v[k].x);
        y = fmaxf(y, v[k].y);
      }
    }
    x = wave_max(x);
    y = wave_max(y);
    if (lane == 0) {
      red[0][wave] = x;
      red[1][wave] = y;
    }
  }
  __syncthreads();
  // |dS| <= largest |dS| with D0 + largest correction (P <= 1), with 2 % for rounding
  float md = red[0][0], mc = red[1][0];
#pragma unroll
  for (int k = 1; k < kPackWaves; ++k) {
    md = fmaxf(md, red[0][k]);
    mc = fmaxf(mc, red[1][k]);
  }
  const float bound = 1.02f * (md + mc);
  int fexp = 0;
  if (bound > 0.0f && bound < INFINITY) {
    int e;
    frexpf(bound, &e);                                    // bound < 2^e
    fexp = 30 - e;
    fexp = fexp < 90 ? fexp : 90;                         // (at least -98; V 2^F is finite up to 2^37)
  }
  const float sF = ldexpf(1.0f, fexp);

  const ScoreConst sc = M::consts(a, CAP);
  // uncapped bf16: the score accumulator starts from -LSE log2 e / mul
  constexpr bool START = M::BF16 && !CAP;
  const float ml_mul = START ? 1.0f / sc.mul : 1.0f;
  const float d_mul = DROP ? sF : -sF;
  const Philox rng(a, h);
  const uint32_t below = (uint32_t)((a.thr - 1) & 0xffff) * 0x10001u;
  int off_tr8[2];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
    off_tr8[hh] = (16 * g + 8 * hh + ((lane & 15) >> 1)) * 32 + 16 * ((lane >> 4) & 1) + 8 * (lane & 1);

  const float rp = DROP ? a.rp : 1.0f;
  const float mk = a.scale * rp * ldexpf(1.0f, -fexp) * (CAP ? M::kSlope : 1.0f);
  bool any_bad = false;

  for (int job = pl.job; job < a.njobs; job += a.slots) {
    const PackWave gr = scalar_record(a.jobs + (int64_t)job * kPackWaves + wave);
    const int lw = gr.log2w, W = 1 << lw;
    const int grp = wave >> lw, gw = wave & (W - 1);
    const int off = gr.nk - gr.nq;
    const int jw = gr.row;                       // the wave's first key
    const int j = jw + col;
    const bool active = jw < gr.nk;
    const bool jok = j < gr.nk;
    const int jc = jok ? j : (active ? gr.nk - 1 : 0);
    // queries from the bound on see the key: the lane's, the wave's least and most
    const int jl = jw + 31 < gr.nk ? jw + 31 : gr.nk - 1;
    auto first = [&](int key) { return key < gr.prefix ? 0 : key - off; };
    const int lo = first(jc), lo0 = first(jw), lo1 = first(jl);
    const T* qh = rows_at<const T>(a.q, h, gr.q0);
    const T* oh = rows_at<const T>(a.d_o, h, gr.q0);
    const float* lseh = a.lse + h * a.ld_lse + gr.q0;
    const float* dlth = a.dlt + h * a.ld_dlt + gr.q0;
    typename M::Operand k, v;
    M::load_operand(rows_at<const T>(a.k, h, gr.k0 + jc), active, M::operand_mul(a, CAP), k);
    M::load_operand(rows_at<const T>(a.v, h, gr.k0 + jc), active, sF, v);
    uint4 rk0{}, rk1{};
    if constexpr (DROP) {
      rk0 = rng.keys((uint32_t)(jw + 16 * g) / 8u);
      rk1 = rng.keys((uint32_t)(jw + 16 * g) / 8u + 1u);
    }

    f32x16 dk[NA], dv[NA];
#pragma unroll
    for (int c = 0; c < NA; ++c) {
      dk[c] = zero_f32x16();
      dv[c] = zero_f32x16();
    }

    // spd bytes of a block: lane l loads 16 bytes of query row l / 2, from key
    // 16 (l & 1) of the wave's on, which are transposed through LDS. A block's first
    // row is a multiple of 32, so the lane's address mod 4 stays the same.
    const uint8_t* sbase = a.spd + gr.spd + (active ? jw : 0);
    const uint32_t srem = (uint32_t)(reinterpret_cast<uintptr_t>(sbase) & 15u);
    uint32_t svoff = (uint32_t)((lane >> 1) * (int64_t)gr.ld) + 16u * (uint32_t)(lane & 1) + srem;
    const uint32_t ssh = svoff & 3u;
    svoff -= ssh;
    auto fetch = [&](int i0, uint32_t (&w)[5]) {
      const int64_t n = gr.nq - i0 < 32 ? gr.nq - i0 : 32;
      const int64_t bytes = n > 0 && active ? (n - 1) * (int64_t)gr.ld + (gr.nk - jw) + srem + 3 : 0;
      load_spd5(make_rsrc_n(sbase - srem + (n > 0 ? (int64_t)i0 * gr.ld : 0), bytes & ~(int64_t)3), svoff, w);
    };
    uint32_t w[5];
    const int step = 32 << lw;
    float stat = 0.0f;
    auto load_stat = [&](int i0) {
      const int r = i0 + col < gr.nq ? i0 + col : gr.nq - 1;
      if (gr.nq > 0) stat = (g == 0 ? lseh : dlth)[r];
    };
    auto store_stat = [&](int i0, int buf) {
      float x = stat;
      opaque_f(x);
      const bool in = i0 + col < gr.nq;
      if (g == 0)
        x = in && x != -INFINITY ? -M::to_unit(x) * ml_mul : -INFINITY;
      else
        x = in ? x * d_mul : 0.0f;
      sStat[buf][wave][lane] = x;
    };

    // One block of 32 queries from i0 on, staged in qt and ot.
    auto block = [&](const T* qt, const T* ot, const float* st, int i0) {
      align_spd5(w, ssh);
      const uint4 w4 = make_uint4(w[0], w[1], w[2], w[3]);
      fetch(i0 + 32, w);
      if (i0 + 31 < lo0) return;                            // no query of the block sees a key (wave-uniform)
      uint32_t b[4];
      transpose_bytes(sByte[wave], 16 * lane, w4, off_tr8, b);
      f32x16 s, dp;
      float x[16], slope[16], ml[16], dl[16];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float4 y = *reinterpret_cast<const float4*>(st + 16 * g + 4 * u);
        const float4 z = *reinterpret_cast<const float4*>(st + 32 + 16 * g + 4 * u);
        ml[4 * u] = y.x; ml[4 * u + 1] = y.y; ml[4 * u + 2] = y.z; ml[4 * u + 3] = y.w;
        dl[4 * u] = z.x; dl[4 * u + 1] = z.y; dl[4 * u + 2] = z.z; dl[4 * u + 3] = z.w;
      }
      bias16(sTab, b, x);
      // (masks enter with the biases, so that the element work is one run of
      // instructions: 3 % at d = 64; with dropout after the exponential, 5 % at d = 8)
      if (!DROP && (i0 < lo1 || jw + 32 > gr.nk)) {
        const int r0 = jok ? lo - i0 - 16 * g : 16;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = r >= r0 ? x[r] : -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = START ? ml[r] : 0.0f;
        dp[r] = DROP ? 0.0f : dl[r];
      }
      M::rows(qt, k, s);
      M::rows(ot, v, dp);
      if constexpr (START) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = fmaf(s[r], sc.mul, x[r]);
      } else {
        M::template scores<CAP, true>(s, x, slope, sc);
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] += ml[r];
      }
      float p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = M::expo(x[r]);
      if (DROP && (i0 < lo1 || jw + 32 > gr.nk)) {
        const int r0 = jok ? lo - i0 - 16 * g : 16;
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = r >= r0 ? p[r] : 0.0f;
      }
      if constexpr (DROP) {
        uint32_t rw[8], z[4];
        const RowDraw rr = rng.row((uint32_t)(gr.q0 + i0 + col));
        rng.draw(rr, rk0, rw);
        rng.draw(rr, rk1, rw + 4);
        uint4 kb;
        kb.x = __builtin_amdgcn_perm(kept2(rw[1], below), kept2(rw[0], below), 0x06040200u) & 0x01010101u;
        kb.y = __builtin_amdgcn_perm(kept2(rw[3], below), kept2(rw[2], below), 0x06040200u) & 0x01010101u;
        kb.z = __builtin_amdgcn_perm(kept2(rw[5], below), kept2(rw[4], below), 0x06040200u) & 0x01010101u;
        kb.w = __builtin_amdgcn_perm(kept2(rw[7], below), kept2(rw[6], below), 0x06040200u) & 0x01010101u;
        transpose_bytes(sByte[wave], 32 * col + 16 * g, kb, off_tr8, z);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float pz = p[r] * (float)((z[r >> 2] >> (8 * (r & 3))) & 0xffu);
          x[r] = fmaf(pz, dp[r], -p[r] * dl[r]);
          p[r] = pz;
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = p[r] * dp[r];
      }
      if constexpr (!WIDE) {
        // bytes past the layout go to a bucket behind it
        const uint32_t past = (0x100u - (uint32_t)a.hist) * 0x01010101u;
        if (__any(((b[0] | b[1] | b[2] | b[3]) & past) != 0)) {
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              if ((b[u] & past) >> e & 0xffu) b[u] = (b[u] & ~(0xffu << e)) | (uint32_t)a.hist << e;
        }
      }
      const uint32_t copy = (uint32_t)(lane & (CPY - 1)) * 8u;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t at = WIDE ? ((((b[r >> 2] >> (8 * (r & 3))) & 0xffu) << 7) | copy)
                                 : __builtin_amdgcn_perm(b[r >> 2], copy, 0x0c0c0000u | ((4u + (r & 3)) << 8));
        unsigned long long* e = reinterpret_cast<unsigned long long*>(reinterpret_cast<uint8_t*>(hist) + at);
        if (r % 2 == 0)
          add_term<0>(e, x[r]);
        else
          add_term<1>(e, x[r]);
        if constexpr (CAP) x[r] *= slope[r];
      }
      M::cols(ot, p, dv);
      M::cols(qt, x, dk);
    };
    auto blocks = [&](const T* sQ, const T* sO, int buf, int t0) {
      if (!active) return;
      for (int ib = 0; ib < W; ++ib) {
        const int i0 = t0 + ib * 32, slot = (grp << lw) + ib;
        if (i0 >= gr.c1) break;
        block(sQ + slot * M::TILE, sO + slot * M::TILE, sStat[buf][slot], i0);
      }
    };

    int t0 = gr.c0;
    T* const sQ0 = reinterpret_cast<T*>(sBuf0);
    T* const sO0 = sQ0 + kPackWaves * M::TILE;
    if (gr.steps > 0) {
      load_stat(t0 + gw * 32);
      fetch(t0, w);
    }
    if constexpr (M::BF16) {
      const PackDma<M> cq(a.q.rs), co(a.d_o.rs);
      auto stage = [&](T* q, T* o, int buf, int t) {
        cq.load(qh, a.q.rs, t + gw * 32, gr.nq, q + wave * M::TILE);
        co.load(oh, a.d_o.rs, t + gw * 32, gr.nq, o + wave * M::TILE);
        store_stat(t + gw * 32, buf);
        load_stat(t + step + gw * 32);
      };
      if constexpr (NB == 2) {
        T* const sQ1 = reinterpret_cast<T*>(sBuf1);
        T* const sO1 = sQ1 + kPackWaves * M::TILE;
        if (gr.steps > 0) stage(sQ0, sO0, 0, t0);
        for (int t = 0; t < gr.steps; t += 2) {
          wait_vmcnt<0>();
          lds_barrier();
          if (t + 1 < gr.steps) stage(sQ1, sO1, 1, t0 + step);
          blocks(sQ0, sO0, 0, t0);
          t0 += step;
          if (t + 1 >= gr.steps) break;
          wait_vmcnt<0>();
          lds_barrier();
          if (t + 2 < gr.steps) stage(sQ0, sO0, 0, t0 + step);
          blocks(sQ1, sO1, 1, t0);
          t0 += step;
        }
      } else {
        for (int t = 0; t < gr.steps; ++t, t0 += step) {
          lds_barrier();
          stage(sQ0, sO0, 0, t0);
          wait_vmcnt<0>();
          lds_barrier();
          blocks(sQ0, sO0, 0, t0);
        }
      }
    } else {
      PackStage<M> tq, to;
      auto load = [&](int t) {
        tq.load(qh, a.q.rs, t + gw * 32, gr.nq);
        to.load(oh, a.d_o.rs, t + gw * 32, gr.nq);
      };
      if (gr.steps > 0) load(t0);
      for (int t = 0; t < gr.steps; ++t, t0 += step) {
        lds_barrier();
        tq.store(sQ0 + wave * M::TILE);
        to.store(sO0 + wave * M::TILE);
        store_stat(t0 + gw * 32, 0);
        lds_barrier();
        if (t + 1 < gr.steps) {
          load(t0 + step);
          load_stat(t0 + step + gw * 32);
        }
        blocks(sQ0, sO0, 0, t0);
      }
    }
    // a dS that is no number makes its key's dK so: the head's table gradient is
    // then NaN (the fixed-point sums cannot show it)
    bool ok = true;
#pragma unroll
    for (int r = 0; r < 16; ++r) ok = ok && fabsf(dk[0][r]) < INFINITY;
    any_bad = any_bad || __any(jok && !ok);
    if (gr.combine) {
      float* buf = reinterpret_cast<float*>(sBuf0);
      auto none = [](int) {};
      auto add = [](int, float& wa, float& wo) { wa = wo = 1.0f; };
      pack_combine(buf, lw, grp, gw, dk, none, add);
      pack_combine(buf, lw, grp, gw, dv, none, add);
    }
    if (jok && (!gr.combine || grp == 0)) {
      T* dkp = rows_at<T>(a.dk, h, gr.k0 + j);
      T* dvp = rows_at<T>(a.dv, h, gr.k0 + j);
      M::features(dk, [&](int f, float4 x) { M::store4(dkp + f, make_float4(x.x * mk, x.y * mk, x.z * mk, x.w * mk)); });
      M::features(dv, [&](int f, float4 x) { M::store4(dvp + f, make_float4(x.x * rp, x.y * rp, x.z * rp, x.w * rp)); });
    }
    lds_barrier();                                        // the next job stages over this one's tiles
  }
  if (lane == 0) bad[wave] = any_bad;
  __syncthreads();
  const double unscale = ldexp((double)rp, -fexp);
  const bool nan = bad[0] | bad[1] | bad[2] | bad[3];
  for (int b = tid; b < a.n_buckets; b += kPackThreads) {
    long long t = 0;
#pragma unroll
    for (int c = 0; c < CPY; ++c) t += (long long)hist[b * CPY + ((c + b) & (CPY - 1))];
    a.dtab_part[((int64_t)h * a.slots + pl.job) * a.n_buckets + b] = nan ? (double)NAN : (double)t * unscale;
  }
}

template <class M, bool CAP, bool DROP>
void launch_pack_dkdv_nb(PackArgs a, hipStream_t s) {
  const dim3 grid(pack_grid(a.slots, a.H)), block(kPackThreads);
  const int lds = hist_bytes(a.n_buckets);
  a.hist = hist_buckets(a.n_buckets);
  if (a.hist == 256) {
    hipLaunchKernelGGL((pack_dkdv_kernel<M, CAP, DROP, 256>), grid, block, lds, s, a);
    return;
  }
  if constexpr (three_waves<M>(CAP, DROP)) {
    if (a.hist <= 64) {
      hipLaunchKernelGGL((pack_dkdv_kernel<M, CAP, DROP, 64>), grid, block, lds, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((pack_dkdv_kernel<M, CAP, DROP, 128>), grid, block, lds, s, a);
}

template <class M>
hipError_t launch_pack_dkdv(const PackArgs& a, bool cap, bool drop, hipStream_t s) {
  if (cap && drop)
    launch_pack_dkdv_nb<M, true, true>(a, s);
  else if (cap)
    launch_pack_dkdv_nb<M, true, false>(a, s);
  else if (drop)
    launch_pack_dkdv_nb<M, false, true>(a, s);
  else
    launch_pack_dkdv_nb<M, false, false>(a, s);
  return hipGetLastError();
}

}  // namespace

}  // namespace gt
