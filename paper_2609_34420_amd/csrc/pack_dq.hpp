// dQ of packed attention (instantiated in pack_dq_*.hip), and the row sums
// that the dK / dV kernel (pack_dkdv.hpp), launched after it, takes.
//
// Query-stationary as the forward: S^T = K Q^T, dP^T = V dO^T, P = exp(S - LSE),
//   dS = P (z dP / (1 - p) - D),   D_i = dO_i . O_i,
//   dU = dS (1 - tanh^2),   dQ^T += K^T dU^T, times scale at the end.
// D from the rounded O is off by O's rounding, which the table gradient, a sum in
// fp32, would show. The sum of a row's dS is zero with the exact D, so with
// D0 = dO . O the kernel's own sum of dS is D - D0: the row sum written for the
// dK / dV kernel is D0 plus it. (dQ itself is rounded as O is, and takes D0.)
//
// It also gives the largest |dS| of each wave and the largest correction of D,
// from which the dK / dV kernel takes the scale of its fixed-point table gradient.
#pragma once
#include "pack.hpp"

namespace gt {

namespace {

template <class M, bool CAP, bool DROP>
__global__ __launch_bounds__(kPackThreads, 2) void pack_dq_kernel(PackArgs a) {
  using T = typename M::T;
  constexpr int NA = M::NA;
  constexpr int XCH = NA * 16 * 64 * 4 * 2 + 2 * 64 * 8;
  constexpr int STG = 2 * kPackWaves * M::TILE * (int)sizeof(T);
  __shared__ alignas(128) uint8_t sBuf[STG > XCH ? STG : XCH];
  __shared__ float sTab[256];
  T* sK = reinterpret_cast<T*>(sBuf);
  T* sV = sK + kPackWaves * M::TILE;

  const PackPlace pl(a);
  if (pl.job >= a.njobs) return;
  const int h = pl.h;
  const PackJob jb = a.jobs[pl.job];
  const int wave = wave_id(), lane = threadIdx.x & 63, col = lane & 31, g = lane >> 5;
  const int lw = jb.log2w, W = 1 << lw;
  const int grp = wave >> lw, gw = wave & (W - 1);
  const PackGroup gr = a.groups[jb.group + grp];
  {
    const int b = threadIdx.x;
    sTab[b] = M::entry(b < a.n_buckets ? a.table[(int64_t)h * a.n_buckets + b] : 0.0f, a, CAP);
  }

  const int off = gr.nk - gr.nq;
  const int iw = gr.row0 + gw * 32;
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
  float dlt, mlse;                                     // D0 and -LSE (-inf: every P of the row is 0)
  {
    typename M::Operand o;
    M::load_operand(rows_at<const T>(a.o, h, gr.q0 + ic), active && iok, 1.0f, o);
    dlt = M::dot(o, d_o);
    dlt += __shfl_xor(dlt, 32);
    const float lse = active && iok ? a.lse[h * a.ld_lse + gr.q0 + ic] : -INFINITY;
    mlse = lse == -INFINITY ? -INFINITY : -M::to_unit(lse);
  }
  const ScoreConst sc = M::consts(a, CAP);
  const uint32_t roff = DROP ? a.offset + (a.offset_dev ? *a.offset_dev : 0u) : 0u;
  const PackSpdRow spd(a.spd + gr.spd + (int64_t)(active ? iw : 0) * gr.ld, gr.ld, active ? gr.nq - iw : 1,
                       active ? gr.nk : 0);
  f32x16 acc[NA];
#pragma unroll
  for (int c = 0; c < NA; ++c) acc[c] = zero_f32x16();
  float dsum = 0.0f, dmax = 0.0f;

  PackStage<M> tk, tv;
  uint32_t w[5];
  const int step = 32 << lw;
  int t0 = gr.c0;
  if (jb.steps > 0) {
    tk.load(kh, a.k.rs, t0 + gw * 32, gr.nk);
    tv.load(vh, a.v.rs, t0 + gw * 32, gr.nk);
    spd.fetch(t0, w);
  }
  for (int t = 0; t < jb.steps; ++t, t0 += step) {
    lds_barrier();
    tk.store(sK + wave * M::TILE);
    tv.store(sV + wave * M::TILE);
    lds_barrier();
    if (t + 1 < jb.steps) {
      tk.load(kh, a.k.rs, t0 + step + gw * 32, gr.nk);
      tv.load(vh, a.v.rs, t0 + step + gw * 32, gr.nk);
    }
    for (int kb = 0; kb < W; ++kb) {
      const int j0 = t0 + kb * 32;
      if (j0 >= lim1) break;
      const T* kt = sK + ((grp << lw) + kb) * M::TILE;
      const T* vt = sV + ((grp << lw) + kb) * M::TILE;
      align_spd5(w, spd.sh);
      float x[16], slope[16];
      bias16(sTab, w, x);
      spd.fetch(j0 + 32, w);
      f32x16 s = zero_f32x16(), dp = zero_f32x16();
      M::rows(kt, q, s);
      M::rows(vt, d_o, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = M::template score<CAP>(s[r], x[r], sc, slope[r]);
      if (j0 + 32 > lim0) {
        const int rem = lim - j0 - 16 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = r < rem ? x[r] : -INFINITY;
      }
      if constexpr (DROP) {
        uint32_t rw[8];
        draw16(a, roff, h, (uint32_t)(gr.q0 + i), j0 + 16 * g, rw);
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = kept(rw, r, a.thr) ? dp[r] * a.rp : 0.0f;
      }
      float bsum = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = M::expo(x[r], mlse) * (dp[r] - dlt);
        bsum += x[r];
        dmax = fmaxf(dmax, fabsf(x[r]));
        if constexpr (CAP) x[r] *= slope[r];
      }
      dsum += bsum;
      M::cols(kt, x, acc);
    }
  }
  dsum += __shfl_xor(dsum, 32);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) dmax = fmaxf(dmax, __shfl_xor(dmax, o));
  float2* dm = a.dmax + ((int64_t)h * a.njobs + pl.job) * kPackWaves + wave;
  if (jb.combine) {
    float* stat = reinterpret_cast<float*>(sBuf + NA * 16 * 64 * 4 * 2) + lane;
    pack_combine(
        reinterpret_cast<float*>(sBuf), lw, grp, gw, acc, [&](int slot) { stat[slot * 64] = dsum; },
        [&](int slot, float& wa, float& wo) {
          dsum += stat[slot * 64];
          wa = wo = 1.0f;
        });
    if (grp != 0) {
      if (lane == 0) *dm = make_float2(dmax, 0.0f);
      return;
    }
  }
  float cmax = fabsf(dsum);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) cmax = fmaxf(cmax, __shfl_xor(cmax, o));
  if (lane == 0) *dm = make_float2(dmax, cmax);
  if (!iok) return;
  const float mul = a.scale * (CAP ? M::kSlope : 1.0f);
  T* out = rows_at<T>(a.dq, h, gr.q0 + i);
  M::features(acc, [&](int f, float4 v) {
    M::store4(out + f, make_float4(v.x * mul, v.y * mul, v.z * mul, v.w * mul));
  });
  if (g == 0) a.dlt[h * a.ld_dlt + gr.q0 + i] = dlt + dsum;
}

template <class M>
hipError_t launch_pack_dq(const PackArgs& a, bool cap, bool drop, hipStream_t s) {
  const dim3 grid(pack_grid(a.njobs, a.H)), block(kPackThreads);
  if (cap && drop)
    hipLaunchKernelGGL((pack_dq_kernel<M, true, true>), grid, block, 0, s, a);
  else if (cap)
    hipLaunchKernelGGL((pack_dq_kernel<M, true, false>), grid, block, 0, s, a);
  else if (drop)
    hipLaunchKernelGGL((pack_dq_kernel<M, false, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((pack_dq_kernel<M, false, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

}  // namespace gt
