// Forward of packed attention (instantiated in pack_fwd_*.hip).
//
// Query-stationary: a wave has 32 queries and computes S^T = K Q^T, so a lane
// owns one query and 16 keys of a 32-key block; the softmax is lane-local but
// for the two lane halves, and O^T += V^T P^T takes P from registers. One pass
// over the keys with a running reference m and sum l. The reference moves only
// when needed: while every lane's block sum stays at or below 256 the block is
// accepted as is (m is always a score the row attained, so the final sum is at
// least 1); else the block's maximum becomes the reference and the state is
// rescaled.
//
// P is summed in fp32 before it is rounded to bf16 for P V, so that the
// log-sum-exp is exact to fp32; dropped pairs stay in the sum.
#pragma once
#include "pack.hpp"

namespace gt {

namespace {

template <class M, bool CAP, bool DROP>
__global__ __launch_bounds__(kPackThreads, 2) void pack_fwd_kernel(PackArgs a) {
  using T = typename M::T;
  constexpr int NA = M::NA;
  constexpr int XCH = NA * 16 * 64 * 4 * 2 + 2 * 64 * 8;         // bytes of two waves' state
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
  const int iw = gr.row0 + gw * 32;                    // the wave's first query
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
  const uint32_t roff = DROP ? a.offset + (a.offset_dev ? *a.offset_dev : 0u) : 0u;

  const PackSpdRow spd(a.spd + gr.spd + (int64_t)(active ? iw : 0) * gr.ld, gr.ld, active ? gr.nq - iw : 1,
                       active ? gr.nk : 0);
  f32x16 acc[NA];
#pragma unroll
  for (int c = 0; c < NA; ++c) acc[c] = zero_f32x16();
  float m = -INFINITY, mneg = 0.0f, l = 0.0f;

  PackStage<M> tk, tv;
  uint32_t w[5];
  const int step = 32 << lw;
  int t0 = gr.c0;                                      // the tile's first key
  if (jb.steps > 0) {
    tk.load(kh, a.k.rs, t0 + gw * 32, gr.nk);
    tv.load(vh, a.v.rs, t0 + gw * 32, gr.nk);
    spd.fetch(t0, w);
  }
  for (int t = 0; t < jb.steps; ++t, t0 += step) {
    lds_barrier();                                     // the last tile's reads are done
    tk.store(sK + wave * M::TILE);
    tv.store(sV + wave * M::TILE);
    lds_barrier();
    if (t + 1 < jb.steps) {
      tk.load(kh, a.k.rs, t0 + step + gw * 32, gr.nk);
      tv.load(vh, a.v.rs, t0 + step + gw * 32, gr.nk);
    }
    for (int kb = 0; kb < W; ++kb) {
      const int j0 = t0 + kb * 32;
      if (j0 >= lim1) break;                           // no visible key from here on (wave-uniform)
      const T* kt = sK + ((grp << lw) + kb) * M::TILE;
      const T* vt = sV + ((grp << lw) + kb) * M::TILE;
      align_spd5(w, spd.sh);
      float x[16];
      bias16(sTab, w, x);
      spd.fetch(j0 + 32, w);                           // (past the graph it reads zeros)
      f32x16 s = zero_f32x16();
      M::rows(kt, q, s);
      float slope;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = M::template score<CAP>(s[r], x[r], sc, slope);
      if (j0 + 32 > lim0) {
        const int rem = lim - j0 - 16 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = r < rem ? x[r] : -INFINITY;
      }
      float p[16];
      float bs = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] = M::expo(x[r], mneg);
        bs += p[r];
      }
      if (__any(!(bs <= 256.0f) || m == -INFINITY)) {  // move the reference to the block's maximum
        float mx = x[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mn = fmaxf(m, mx);
        const float alpha = m == -INFINITY ? 0.0f : M::expo(m, -mn);
        l *= alpha;
#pragma unroll
        for (int c = 0; c < NA; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[c][r] *= alpha;
        m = mn;
        mneg = mn == -INFINITY ? 0.0f : -mn;
        bs = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[r] = M::expo(x[r], mneg);
          bs += p[r];
        }
      }
      l += bs;
      if constexpr (DROP) {
        uint32_t rw[8];
        draw16(a, roff, h, (uint32_t)(gr.q0 + i), j0 + 16 * g, rw);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = kept(rw, r, a.thr) ? p[r] : 0.0f;
      }
      M::cols(vt, p, acc);
    }
  }
  l += __shfl_xor(l, 32);
  if (jb.combine) {
    float2* stat = reinterpret_cast<float2*>(sBuf + NA * 16 * 64 * 4 * 2) + lane;
    pack_combine(
        reinterpret_cast<float*>(sBuf), lw, grp, gw, acc, [&](int slot) { stat[slot * 64] = make_float2(m, l); },
        [&](int slot, float& wa, float& wo) {
          const float2 o = stat[slot * 64];
          const float mn = fmaxf(m, o.x);
          wa = m == -INFINITY ? 0.0f : M::expo(m, -mn);
          wo = o.x == -INFINITY ? 0.0f : M::expo(o.x, -mn);
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
