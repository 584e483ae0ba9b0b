// dQ of packed attention (instantiated in pack_dq_*.hip), and the row sums
// that the dK / dV kernel (pack_dkdv.hpp), launched after it, takes.
//
// Query-stationary as the forward: S^T = K Q^T, dP^T = V dO^T, P = exp(S - LSE)
// at its own size before it meets dP (with the forward's reference of a head instead, and
// LSE at the end, rows far below it lose dS of 2^-45, and those near it overflow at 2^60),
//   dS = P (z dP / (1 - p) - D),   D_i = dO_i . O_i,
//   dU = dS (1 - tanh^2),   dQ^T += K^T dU^T, times scale at the end.
// D from a bf16 O is off by O's rounding: the table gradient, a sum in fp32, would
// show it, and dQ too where the softmax is peaked, since a row's error is the same
// for all of its keys (2.6 times the rounding of dQ itself for graphs of some
// thirty nodes, d = 8). The sum of a row's dS is zero with the exact D, so with
// D0 = dO . O the kernel's own sum of dS is D - D0. The row sum written for the
// dK / dV kernel is D0 plus it, and dQ is corrected by it times the sum of
// P (1 - tanh^2) K, which takes a second product per key tile.
//
// It also gives the largest |dS| of each job and the largest correction of D,
// from which the dK / dV kernel takes the scale of its fixed-point table gradient.
//
// dU is rounded to bf16 as the operand of its product. A row's terms of either sign
// largely cancel, so that rounding shows as much as that of dQ itself: 2.4e-3 to 2.6e-3
// in relative L2 where the best bf16 dQ is off by 1.7e-3. (dU as two bf16 terms would
// remove it for a second product and 24 conversions per block.)
//
// Bound: issue of the element work, 18 vector instructions per pair and lane with a
// cap (16384 nodes, H = 8, d = 64: 1545 us, 534 TFLOP/s without the correction's
// product; vector units busy 80 % of the cycles at two waves per SIMD, 87 to 91 % at
// three, d <= 32; fp32: matrix cores 45 %, vector units 31 %, 50 us for 6 graphs of 300 to
// 1200, H = 4, d = 32, cap). Two buffers of tiles at every d: at d = 64 the registers leave
// two workgroups per unit, and so does the LDS.
#pragma once
#include "pack.hpp"

namespace gt {

namespace {

// WPS: waves per SIMD that the registers are shared by.
template <class M, bool CAP, bool DROP, int WPS>
__global__ __launch_bounds__(kPackThreads, WPS) void pack_dq_kernel(PackArgs a) {
  using T = typename M::T;
  constexpr int NA = M::NA;
  constexpr int NB = M::BF16 ? 2 : 1;                            // staged tiles
  constexpr bool FIX = M::BF16;                                  // dQ is corrected for O's rounding
  constexpr int XCH = NA * 16 * 64 * 4 * 2 + 2 * 64 * 8;
  constexpr int STG = 2 * kPackWaves * M::TILE * (int)sizeof(T);
  __shared__ alignas(128) uint8_t sBuf0[STG > XCH ? STG : XCH];
  __shared__ alignas(128) uint8_t sBuf1[NB == 2 ? STG : 16];
  __shared__ float sTab[256];
  __shared__ float2 sMax[kPackWaves];
  __shared__ uint4 sKeys[DROP ? NB * kPackWaves * 4 : 1];

  const PackPlace pl(a, a.njobs);
  if (pl.job >= a.njobs) return;
  const int h = pl.h;
  const int wave = wave_id(), lane = threadIdx.x & 63, col = lane & 31, g = lane >> 5;
  const PackWave gr = scalar_record(a.jobs + (int64_t)pl.job * kPackWaves + wave);
  const int lw = gr.log2w, W = 1 << lw;
  const int grp = wave >> lw, gw = wave & (W - 1);
  constexpr bool START = M::BF16 && !CAP;
  {
    const int b = threadIdx.x;
    sTab[b] = M::entry(b < a.n_buckets ? a.table[(int64_t)h * a.n_buckets + b] : 0.0f, a, START)
              + (M::BF16 && CAP ? a.cap * kLog2e : 0.0f);
  }

  const int off = gr.nk - gr.nq;
  const int iw = gr.row;
  const int i = iw + col;
  const bool active = iw < gr.nq;
  const bool iok = i < gr.nq;
  const int ic = iok ? i : (active ? gr.nq - 1 : 0);
  const int il = iw + 31 < gr.nq ? iw + 31 : gr.nq - 1;
  auto limit = [&](int row) {
    const int vis = row + off + 1 > gr.prefix ? row + off + 1 : gr.prefix;
    return vis < gr.c1 ? vis : gr.c1;
  };
  const int lim = limit(ic), lim0 = limit(iw), lim1 = active ? limit(il) : 0;
  const T* kh = rows_at<const T>(a.k, h, gr.k0);
  const T* vh = rows_at<const T>(a.v, h, gr.k0);
  typename M::Operand q, d_o;
  M::load_operand(rows_at<const T>(a.q, h, gr.q0 + ic), active, M::operand_mul(a, CAP), q);
  M::load_operand(rows_at<const T>(a.d_o, h, gr.q0 + ic), active && iok, 1.0f, d_o);
  // D0 and -LSE (-inf: every P of the row is 0). With dropout the 1 / (1 - p) of dP is
  // left out up to the end: dS (1 - p) = P (z dP - D (1 - p)).
  const float rp = DROP ? a.rp : 1.0f;
  float dlt, mlse;
  {
    typename M::Operand o;
    M::load_operand(rows_at<const T>(a.o, h, gr.q0 + ic), active && iok, 1.0f, o);
    dlt = M::dot(o, d_o);
    dlt = (dlt + __shfl_xor(dlt, 32)) / rp;
    const float lse = active && iok ? a.lse[h * a.ld_lse + gr.q0 + ic] : -INFINITY;
    mlse = lse == -INFINITY ? -INFINITY : -M::to_unit(lse);
  }
  const ScoreConst sc = M::consts(a, CAP);
  const Philox rng(a, h);
  RowDraw rrow{};
  if constexpr (DROP) rrow = rng.row((uint32_t)(gr.q0 + i));
  const PackSpdRow spd(a.spd + gr.spd + (int64_t)(active ? iw : 0) * gr.ld, gr.ld, active ? gr.nq - iw : 1,
                       active ? gr.nk : 0);
  f32x16 acc[NA], fix[NA];
#pragma unroll
  for (int c = 0; c < NA; ++c) {
    acc[c] = zero_f32x16();
    fix[c] = zero_f32x16();
  }
  float dsum = 0.0f, dmax = 0.0f;
  uint32_t w[5];
  const int step = 32 << lw;

  auto block = [&](const T* kt, const T* vt, const uint4* keys, int j0) {
    align_spd5(w, spd.sh);
    float x[16], slope[16];
    bias16(sTab, w, x);
    spd.fetch(j0 + 32, w);
    f32x16 s = zero_f32x16(), dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if constexpr (START) s[r] = x[r];
      dp[r] = DROP ? 0.0f : -dlt;
    }
    M::rows(kt, q, s);
    M::rows(vt, d_o, dp);
    if constexpr (START) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = fmaf(s[r], sc.mul, mlse);
    } else {
      M::template scores<CAP, true>(s, x, slope, sc);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] += mlse;
    }
    if (j0 + 32 > lim0) keep_below(x, lim - j0 - 16 * g, -INFINITY);
    if constexpr (DROP) {
      uint32_t rw[8];
      rng.draw(rrow, keys[2 * g], rw);
      rng.draw(rrow, keys[2 * g + 1], rw + 4);
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] = (kept(rw, r, a.thr) ? dp[r] : 0.0f) - dlt;
    }
    float du[16];
    float bsum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
#pragma unroll
      for (int e = r; e < r + 2; ++e) {
        x[e] = M::expo(x[e]);
        const float ds = x[e] * dp[e];
        bsum += ds;
        if constexpr (CAP) x[e] *= slope[e];
        du[e] = CAP ? x[e] * dp[e] : ds;
        s[e] = ds;
      }
      dmax = fmaxf(fmaxf(dmax, fabsf(s[r])), fabsf(s[r + 1]));
    }
    dsum += bsum;
    if constexpr (FIX)
      M::cols2(kt, du, acc, x, fix);
    else
      M::cols(kt, du, acc);
  };
  auto put_keys = [&](int t0, int buf) {
    if constexpr (DROP) {
      const uint4 k = rng.keys((uint32_t)(t0 + gw * 32) / 8u + (uint32_t)(lane & 3));
      if (lane < 4) sKeys[(buf * kPackWaves + wave) * 4 + lane] = k;
    }
  };
  auto blocks = [&](const T* sK, const T* sV, int buf, int t0) {
    for (int kb = 0; kb < W; ++kb) {
      const int j0 = t0 + kb * 32, slot = (grp << lw) + kb;
      if (j0 >= lim1) break;
      block(sK + slot * M::TILE, sV + slot * M::TILE, sKeys + (DROP ? (buf * kPackWaves + slot) * 4 : 0), j0);
    }
  };

  int t0 = gr.c0;
  T* const sK0 = reinterpret_cast<T*>(sBuf0);
  T* const sV0 = sK0 + kPackWaves * M::TILE;
  if (gr.steps > 0) spd.fetch(t0, w);
  if constexpr (M::BF16) {
    T* const sK1 = reinterpret_cast<T*>(sBuf1);
    T* const sV1 = sK1 + kPackWaves * M::TILE;
    const PackDma<M> dk(a.k.rs), dv(a.v.rs);
    auto copy = [&](T* k, T* v, int t) {
      dk.load(kh, a.k.rs, t + gw * 32, gr.nk, k + wave * M::TILE);
      dv.load(vh, a.v.rs, t + gw * 32, gr.nk, v + wave * M::TILE);
    };
    if (gr.steps > 0) {
      copy(sK0, sV0, t0);
      put_keys(t0, 0);
    }
    for (int t = 0; t < gr.steps; t += 2) {
      wait_vmcnt<0>();
      lds_barrier();
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
  } else {
    PackStage<M> tk, tv;
    auto load = [&](int t) {
      tk.load(kh, a.k.rs, t + gw * 32, gr.nk);
      tv.load(vh, a.v.rs, t + gw * 32, gr.nk);
    };
    if (gr.steps > 0) load(t0);
    for (int t = 0; t < gr.steps; ++t, t0 += step) {
      lds_barrier();
      tk.store(sK0 + wave * M::TILE);
      tv.store(sV0 + wave * M::TILE);
      put_keys(t0, 0);
      lds_barrier();
      if (t + 1 < gr.steps) load(t0 + step);
      blocks(sK0, sV0, 0, t0);
    }
  }
  dsum += __shfl_xor(dsum, 32);
  dmax = wave_max(dmax);
  if (gr.combine) {
    float* stat = reinterpret_cast<float*>(sBuf0 + NA * 16 * 64 * 4 * 2) + lane;
    pack_combine(
        reinterpret_cast<float*>(sBuf0), lw, grp, gw, acc, [&](int slot) { stat[slot * 64] = dsum; },
        [&](int slot, float& wa, float& wo) {
          dsum += stat[slot * 64];
          wa = wo = 1.0f;
        });
    if constexpr (FIX)
      pack_combine(reinterpret_cast<float*>(sBuf0), lw, grp, gw, fix, [](int) {},
                   [](int, float& wa, float& wo) { wa = wo = 1.0f; });
  }
  const bool mine = !gr.combine || grp == 0;             // the wave holds its rows' results
  const float cmax = wave_max(mine ? fabsf(dsum) : 0.0f);
  if (lane == 0) sMax[wave] = make_float2(dmax, cmax);
  if (mine && iok) {
    const float mul = a.scale * rp * (CAP ? M::kSlope : 1.0f);
    if constexpr (FIX) {
#pragma unroll
      for (int c = 0; c < NA; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = fmaf(-dsum, fix[c][r], acc[c][r]);
    }
    T* out = rows_at<T>(a.dq, h, gr.q0 + i);
    M::features(acc, [&](int f, float4 v) {
      M::store4(out + f, make_float4(v.x * mul, v.y * mul, v.z * mul, v.w * mul));
    });
    if (g == 0) a.dlt[h * a.ld_dlt + gr.q0 + i] = dlt + dsum;    // D (1 - p)
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float2 m = sMax[0];
#pragma unroll
    for (int k = 1; k < kPackWaves; ++k) m = make_float2(fmaxf(m.x, sMax[k].x), fmaxf(m.y, sMax[k].y));
    a.dmax[(int64_t)h * a.njobs + pl.job] = make_float2(m.x * rp, m.y * rp);
  }
}

template <class M, int WPS>
hipError_t launch_pack_dq_wps(const PackArgs& a, bool cap, bool drop, hipStream_t s) {
  const dim3 grid(pack_grid(a.njobs, a.H)), block(kPackThreads);
  if (cap && drop)
    hipLaunchKernelGGL((pack_dq_kernel<M, true, true, WPS>), grid, block, 0, s, a);
  else if (cap)
    hipLaunchKernelGGL((pack_dq_kernel<M, true, false, WPS>), grid, block, 0, s, a);
  else if (drop)
    hipLaunchKernelGGL((pack_dq_kernel<M, false, true, WPS>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((pack_dq_kernel<M, false, false, WPS>), grid, block, 0, s, a);
  return hipGetLastError();
}

// At two waves per SIMD the fp32 kernel at d = 64 spills 19 to 31 registers. With a
// workgroup per compute unit or less there is nothing to share them with (2000 nodes,
// H = 4: 137 us, 90 with all registers); with more the second wave is worth it (8 graphs
// of 1000: 163 and 168).
template <class M>
hipError_t launch_pack_dq(const PackArgs& a, bool cap, bool drop, hipStream_t s) {
  if constexpr (!M::BF16 && M::D == 64)
    if ((int64_t)a.njobs * a.H <= 256) return launch_pack_dq_wps<M, 1>(a, cap, drop, s);
  return launch_pack_dq_wps<M, 2>(a, cap, drop, s);
}

}  // namespace

}  // namespace gt
