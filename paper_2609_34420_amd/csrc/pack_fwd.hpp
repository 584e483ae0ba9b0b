// Forward of packed attention (instantiated in pack_fwd_*.hip).
//
// Query-stationary: a wave has 32 queries and computes S^T = K Q^T, so a lane
// owns one query and 16 keys of a 32-key block; the softmax is lane-local but
// for the two lane halves, and O^T += V^T P^T takes P from registers. One pass
// over the keys. Capped bf16 scores take a fixed reference where their range
// allows it (ScoreRef); the others a running reference m, which moves only when
// needed: while every lane's block sum stays at or below 256 the block is accepted
// as is (m is always a score the row attained, so the final sum is at least 1);
// else the block's maximum becomes the reference and the state is rescaled.
//
// P is summed in fp32 before it is rounded to bf16 for P V, so that the
// log-sum-exp is exact to fp32; dropped pairs stay in the sum. The rounding of P is
// the product's operand type, 2^-8 of each term at most.
//
// Tiles: 32 rows per wave of the workgroup, K and V; two buffers at d <= 32, one at
// d = 64, where four workgroups of one buffer hide a copy better than two of two
// (1224 against 1380 us at 16384 nodes).
//
// Bound: issue of the element work, some 10 vector instructions per pair and lane with
// a cap, 3 of them transcendental, against 8 products per block of 32 x 32 at d = 64:
// vector units busy 80 % (16384 nodes, H = 8, d = 64, cap: 988 us, 556 TFLOP/s), 98 %
// with dropout (512 graphs of 100 to 256 nodes, d = 8: 67 us), 87 to 89 % at d = 32 and 8
// with a cap; 63 % where 480 workgroups leave units with one (7651 nodes, dropout: 268 us);
// fp32: matrix cores 38 %, vector units 34 % at 1.8 waves per SIMD (6 graphs of 300 to 1200,
// H = 4, d = 32, cap: 40 us). 16 graphs'
// new node against all their keys: the bytes of K and V, 183 MB in 32 us.
#pragma once
#include "pack.hpp"

namespace gt {

namespace {

template <class M, bool CAP, bool DROP>
__global__ __launch_bounds__(kPackThreads, 2) void pack_fwd_kernel(PackArgs a) {
  using T = typename M::T;
  constexpr int NA = M::NA;
  constexpr int NB = M::BF16 && M::D == 32 ? 2 : 1;              // staged tiles
  constexpr int XCH = NA * 16 * 64 * 4 * 2 + 2 * 64 * 8;         // bytes of two waves' state
  constexpr int STG = 2 * kPackWaves * M::TILE * (int)sizeof(T);
  __shared__ alignas(128) uint8_t sBuf0[STG > XCH ? STG : XCH];
  __shared__ alignas(128) uint8_t sBuf1[NB == 2 ? STG : 16];
  __shared__ float sTab[256];
  __shared__ uint4 sKeys[DROP ? NB * kPackWaves * 4 : 1];        // KeyDraws of the staged keys

  const PackPlace pl(a, a.njobs);
  if (pl.job >= a.njobs) return;
  const int h = pl.h;
  const int wave = wave_id(), lane = threadIdx.x & 63, col = lane & 31, g = lane >> 5;
  const PackWave gr = scalar_record(a.jobs + (int64_t)pl.job * kPackWaves + wave);
  const int lw = gr.log2w, W = 1 << lw;
  const int grp = wave >> lw, gw = wave & (W - 1);
  constexpr bool START = M::BF16 && !CAP;              // the score accumulator starts from the bias
  ScoreRef fix{false, 0.0f};
  if constexpr (M::BF16 && CAP) {
    sTab[threadIdx.x] = capped_entry<M>(a, h, fix);
  } else {
    const int b = threadIdx.x;
    sTab[b] = M::entry(b < a.n_buckets ? a.table[(int64_t)h * a.n_buckets + b] : 0.0f, a, START);
  }

  const int off = gr.nk - gr.nq;
  const int iw = gr.row;                    // the wave's first query
  const int i = iw + col;
  const bool active = iw < gr.nq;
  const bool iok = i < gr.nq;
  const int ic = iok ? i : (active ? gr.nq - 1 : 0);
  // keys below the limit are visible: the lane's, the wave's least and most
  const int il = iw + 31 < gr.nq ? iw + 31 : gr.nq - 1;
  auto limit = [&](int row) {
    const int vis = row + off + 1 > gr.prefix ? row + off + 1 : gr.prefix;
    return vis < gr.c1 ? vis : gr.c1;
  };
  const int lim = limit(ic), lim0 = limit(iw), lim1 = active ? limit(il) : 0;
  const T* kh = rows_at<const T>(a.k, h, gr.k0);
  const T* vh = rows_at<const T>(a.v, h, gr.k0);
  typename M::Operand q;
  M::load_operand(rows_at<const T>(a.q, h, gr.q0 + ic), active, M::operand_mul(a, CAP), q);
  const ScoreConst sc = M::consts(a, CAP);
  const Philox rng(a, h);
  RowDraw rrow{};
  if constexpr (DROP) rrow = rng.row((uint32_t)(gr.q0 + i));
  const uint32_t below = (uint32_t)((a.thr - 1) & 0xffff) * 0x10001u;

  const PackSpdRow spd(a.spd + gr.spd + (int64_t)(active ? iw : 0) * gr.ld, gr.ld, active ? gr.nq - iw : 1,
                       active ? gr.nk : 0);
  f32x16 acc[NA];
#pragma unroll
  for (int c = 0; c < NA; ++c) acc[c] = zero_f32x16();
  float m = -INFINITY, mneg = 0.0f, l = 0.0f;
  uint32_t w[5];
  const int step = 32 << lw;

  // One 32-key block from key j0 on, staged in kt and vt.
  auto block = [&](const T* kt, const T* vt, const uint4* keys, int j0) {
    align_spd5(w, spd.sh);
    float x[16], slope[16];
    bias16(sTab, w, x);
    spd.fetch(j0 + 32, w);                             // (past the graph it reads zeros)
    f32x16 s = zero_f32x16();
    if constexpr (START) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = x[r];
    }
    M::rows(kt, q, s);
    if constexpr (START) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = fmaf(s[r], sc.mul, mneg);
    } else {
      M::template scores<CAP, false>(s, x, slope, sc);
      if (!fix.fixed) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] += mneg;
      }
    }
    if (j0 + 32 > lim0) keep_below(x, lim - j0 - 16 * g, -INFINITY);
    float p[16];
    float bs = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = M::expo(x[r]);
      bs += p[r];
    }
    if (!fix.fixed && __any(!(bs <= 256.0f) || m == -INFINITY)) {    // move the reference to the block's maximum
      float mx = x[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32)) - mneg;
      const float mn = fmaxf(m, mx);
      const float alpha = m == -INFINITY ? 0.0f : M::expo(m - mn);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < NA; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] *= alpha;
      m = mn;
      const float shift = (mn == -INFINITY ? 0.0f : -mn) - mneg;
      mneg += shift;
      bs = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] = M::expo(x[r] + shift);
        bs += p[r];
      }
    }
    l += bs;
    if constexpr (DROP) {
      uint32_t rw[8];
      rng.draw(rrow, keys[2 * g], rw);
      rng.draw(rrow, keys[2 * g + 1], rw + 4);
      M::cols_kept(vt, p, rw, below, a.thr, acc);
    } else {
      M::cols(vt, p, acc);
    }
  };
  // The wave's part of the tile from key t0 on: KeyDraws of its 32 staged keys.
  auto put_keys = [&](int t0, int buf) {
    if constexpr (DROP) {
      const uint4 k = rng.keys((uint32_t)(t0 + gw * 32) / 8u + (uint32_t)(lane & 3));
      if (lane < 4) sKeys[(buf * kPackWaves + wave) * 4 + lane] = k;
    }
  };
  auto blocks = [&](const T* sK, const T* sV, int buf, int t0) {
    for (int kb = 0; kb < W; ++kb) {
      const int j0 = t0 + kb * 32, slot = (grp << lw) + kb;
      if (j0 >= lim1) break;                           // no visible key from here on (wave-uniform)
      block(sK + slot * M::TILE, sV + slot * M::TILE, sKeys + (DROP ? (buf * kPackWaves + slot) * 4 : 0), j0);
    }
  };

  int t0 = gr.c0;                                      // the tile's first key
  T* const sK0 = reinterpret_cast<T*>(sBuf0);
  T* const sV0 = sK0 + kPackWaves * M::TILE;
  if (gr.steps > 0) spd.fetch(t0, w);
  if constexpr (M::BF16) {
    const PackDma<M> dk(a.k.rs), dv(a.v.rs);
    auto copy = [&](T* k, T* v, int t) {
      dk.load(kh, a.k.rs, t + gw * 32, gr.nk, k + wave * M::TILE);
      dv.load(vh, a.v.rs, t + gw * 32, gr.nk, v + wave * M::TILE);
    };
    if constexpr (NB == 1) {
      for (int t = 0; t < gr.steps; ++t, t0 += step) {
        lds_barrier();                                 // the last tile's reads are done
        copy(sK0, sV0, t0);
        put_keys(t0, 0);
        wait_vmcnt<0>();
        lds_barrier();                                 // the tile has landed
        blocks(sK0, sV0, 0, t0);
      }
    } else {
      T* const sK1 = reinterpret_cast<T*>(sBuf1);
      T* const sV1 = sK1 + kPackWaves * M::TILE;
      if (gr.steps > 0) {
        copy(sK0, sV0, t0);
        put_keys(t0, 0);
      }
      for (int t = 0; t < gr.steps; t += 2) {
        wait_vmcnt<0>();
        lds_barrier();                                 // the tile has landed, the last one's reads are done
        if (t + 1 < gr.steps) {
          copy(sK1, sV1, t0 + step);
          put_keys(t0 + step, 1);
        }
        blocks(sK0, sV0, 0, t0);
        t0 = uniform(t0 + step);
        if (t + 1 >= gr.steps) break;
        wait_vmcnt<0>();
        lds_barrier();
        if (t + 2 < gr.steps) {
          copy(sK0, sV0, t0 + step);
          put_keys(t0 + step, 0);
        }
        blocks(sK1, sV1, 1, t0);
        t0 = uniform(t0 + step);
      }
    }
  } else {
    PackStage<M> tk, tv;
    auto load = [&](int t) {
      tk.load(kh, a.k.rs, t + gw * 32, gr.nk);
      tv.load(vh, a.v.rs, t + gw * 32, gr.nk);
    };
    if (gr.steps > 0) load(t0);
    for (int t = 0; t < gr.steps; ++t, t0 += step) {
      lds_barrier();                                   // the last tile's reads are done
      tk.store(sK0 + wave * M::TILE);
      tv.store(sV0 + wave * M::TILE);
      put_keys(t0, 0);
      lds_barrier();
      if (t + 1 < gr.steps) load(t0 + step);
      blocks(sK0, sV0, 0, t0);
    }
  }
  l += __shfl_xor(l, 32);
  if (fix.fixed) m = l == 0.0f ? -INFINITY : fix.ref;
  if (gr.combine) {
    float2* stat = reinterpret_cast<float2*>(sBuf0 + NA * 16 * 64 * 4 * 2) + lane;
    pack_combine(
        reinterpret_cast<float*>(sBuf0), lw, grp, gw, acc, [&](int slot) { stat[slot * 64] = make_float2(m, l); },
        [&](int slot, float& wa, float& wo) {
          const float2 o = stat[slot * 64];
          const float mn = fmaxf(m, o.x);
          wa = m == -INFINITY ? 0.0f : M::expo(m - mn);
          wo = o.x == -INFINITY ? 0.0f : M::expo(o.x - mn);
          l = fmaf(l, wa, o.y * wo);
          m = mn;
        });
    if (grp != 0) return;
  }
  if (!iok) return;
  // O = acc rp / l; a row without a visible score has l = 0 and gets zeros
  // whatever V holds.
  const bool none = l == 0.0f;
  const float inv = (DROP ? a.rp : 1.0f) / l;
  const float lse = none ? -INFINITY : M::log_sum(m, l);
  auto value = [&](float4 v) {
    return none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
  };
  if (gr.part >= 0) {
    const int64_t row = ((int64_t)gr.part * a.H + h) * 32 + col;
    float* op = a.o_part + row * M::DS;
    M::features(acc, [&](int f, float4 v) { *reinterpret_cast<float4*>(op + f) = value(v); });
    if (g == 0) a.lse_part[row] = lse;
    return;
  }
  T* op = rows_at<T>(a.o, h, gr.q0 + i);
  M::features(acc, [&](int f, float4 v) { M::store4(op + f, value(v)); });
  if (g == 0) a.lse[h * a.ld_lse + gr.q0 + i] = lse;
}

template <class M>
hipError_t launch_pack_fwd(const PackArgs& a, bool cap, bool drop, hipStream_t s) {
  const dim3 grid(pack_grid(a.njobs, a.H)), block(kPackThreads);
  if (cap && drop)
    hipLaunchKernelGGL((pack_fwd_kernel<M, true, true>), grid, block, 0, s, a);
  else if (cap)
    hipLaunchKernelGGL((pack_fwd_kernel<M, true, false>), grid, block, 0, s, a);
  else if (drop)
    hipLaunchKernelGGL((pack_fwd_kernel<M, false, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((pack_fwd_kernel<M, false, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

}  // namespace gt
