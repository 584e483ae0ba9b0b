// dK, dV and the table gradient of packed attention (instantiated in
// pack_dkdv_*.hip).
//
// Key-stationary: a wave has 32 keys and streams the graph's queries through
// S = Q K^T and dP = dO V^T, so a lane owns one key and 16 queries of a block:
//   dV^T += dO^T (z P),   dK^T += Q^T dU,   dU = P (z dP / (1 - p) - D)(1 - tanh^2),
// with P and dU taken from registers (1 / (1 - p) and scale at the end).
//
// Dropout: a lane draws for one query and 16 keys, as the query-stationary kernels
// do (a draw serves 8 keys of one row). The comparison of key e gives a ballot
// whose halves are the kept queries of keys e and 16 + e; written to those lanes
// and exchanged between the halves, each lane has its key's 32 queries as bits.
//
// Table gradient: dS is added into an LDS histogram in fixed point, 64-bit sums of
// round(dS 2^F) (float adds to LDS are some twenty times slower), in 32 copies
// (lane & 31) of up to 128 buckets or 16 of 256. F comes from the largest
// |dS| that the dQ kernel met in this head, so that every term stays below 2^31
// and the rounding of 2^-31 of it is far below the sums in fp32. Each workgroup
// writes its sums; a last kernel adds them in a fixed order. Everything is
// bitwise reproducible.
#pragma once
#include "pack.hpp"

namespace gt {

namespace {

constexpr int kPackHist = 4096;

// v_writelane_b32 (this compiler has the intrinsic, but no builtin for it): old
// with `lane` set to the wave-uniform val.
__device__ uint32_t write_lane(uint32_t val, uint32_t lane, uint32_t old) __asm("llvm.amdgcn.writelane.i32");

// Bits of the queries that keep the lane's key, from the draws of the lane's
// query (lane & 31) for keys 16 g .. + 15: bit r is query 16 g + r.
__device__ __forceinline__ uint32_t kept_queries(const uint32_t (&rw)[8], int thr) {
  const int lane = threadIdx.x & 63;
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const uint64_t b = __builtin_amdgcn_ballot_w64(kept(rw, e, thr));
    bits = write_lane((uint32_t)b, e, bits);
    bits = write_lane((uint32_t)(b >> 32), 16 + e, bits);
  }
  bits = __shfl(bits, lane & 31);
  return bits >> (16 * (lane >> 5));
}

template <class M, bool CAP, bool DROP>
__global__ __launch_bounds__(kPackThreads, 2) void pack_dkdv_kernel(PackArgs a) {
  using T = typename M::T;
  constexpr int NA = M::NA;
  constexpr int XCH = NA * 16 * 64 * 4 * 2;
  constexpr int STG = 2 * kPackWaves * M::TILE * (int)sizeof(T);
  __shared__ alignas(128) uint8_t sBuf[STG > XCH ? STG : XCH];
  __shared__ alignas(16) unsigned long long hist[kPackHist];
  __shared__ float sTab[256];
  __shared__ alignas(16) float sStat[kPackWaves][64];     // per staged row: -LSE; D
  __shared__ alignas(16) uint8_t sSpd[kPackWaves][1024];
  __shared__ float red[2][kPackWaves];
  __shared__ int bad[kPackWaves];
  T* sQ = reinterpret_cast<T*>(sBuf);
  T* sO = sQ + kPackWaves * M::TILE;

  const PackPlace pl(a);
  if (pl.job >= a.njobs) return;
  const int h = pl.h;
  const PackJob jb = a.jobs[pl.job];
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, col = lane & 31, g = lane >> 5;
  const int lw = jb.log2w, W = 1 << lw;
  const int grp = wave >> lw, gw = wave & (W - 1);
  const PackGroup gr = a.groups[jb.group + grp];
  const bool wide = a.n_buckets > 127;
  sTab[tid] = M::entry(tid < a.n_buckets ? a.table[(int64_t)h * a.n_buckets + tid] : 0.0f, a, CAP);
  for (int t = tid; t < kPackHist / 2; t += kPackThreads) reinterpret_cast<uint4*>(hist)[t] = make_uint4(0u, 0u, 0u, 0u);
  {
    const float2* dm = a.dmax + (int64_t)h * a.njobs_dq * kPackWaves;
    float x = 0.0f, y = 0.0f;
    for (int t = tid; t < a.njobs_dq * kPackWaves; t += kPackThreads) {
      const float2 v = dm[t];
      x = fmaxf(x, v.x);
      y = fmaxf(y, v.y);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      x = fmaxf(x, __shfl_xor(x, o));
      y = fmaxf(y, __shfl_xor(y, o));
    }
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
    fexp = fexp > 100 ? 100 : (fexp < -90 ? -90 : fexp);
  }
  const float sF = ldexpf(1.0f, fexp);

  const int off = gr.nk - gr.nq;
  const int jw = gr.row0 + gw * 32;                       // the wave's first key
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
  M::load_operand(rows_at<const T>(a.v, h, gr.k0 + jc), active, 1.0f, v);
  const ScoreConst sc = M::consts(a, CAP);
  const uint32_t roff = DROP ? a.offset + (a.offset_dev ? *a.offset_dev : 0u) : 0u;

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
  int off_tr8[2];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
    off_tr8[hh] = (16 * g + 8 * hh + ((lane & 15) >> 1)) * 32 + 16 * ((lane >> 4) & 1) + 8 * (lane & 1);

  PackStage<M> tq, to;
  float stat = 0.0f;
  uint32_t w[5];
  const int step = 32 << lw;
  int t0 = gr.c0;
  auto load = [&](int i0) {
    tq.load(qh, a.q.rs, i0, gr.nq);
    to.load(oh, a.d_o.rs, i0, gr.nq);
    const int r = i0 + col < gr.nq ? i0 + col : gr.nq - 1;
    if (gr.nq > 0) stat = (g == 0 ? lseh : dlth)[r];
  };
  auto store = [&](int i0) {
    tq.store(sQ + wave * M::TILE);
    to.store(sO + wave * M::TILE);
    float x = stat;
    opaque_f(x);
    const bool in = i0 + col < gr.nq;
    if (g == 0)
      x = in && x != -INFINITY ? -M::to_unit(x) : -INFINITY;
    else
      x = in ? x : 0.0f;
    sStat[wave][lane] = x;
  };
  if (jb.steps > 0) {
    load(t0 + gw * 32);
    fetch(t0, w);
  }
  for (int t = 0; t < jb.steps; ++t, t0 += step) {
    lds_barrier();
    store(t0 + gw * 32);
    lds_barrier();
    if (t + 1 < jb.steps) load(t0 + step + gw * 32);
    if (!active) continue;
    for (int ib = 0; ib < W; ++ib) {
      const int i0 = t0 + ib * 32;
      if (i0 >= gr.c1) break;
      const int slot = (grp << lw) + ib;
      align_spd5(w, ssh);
      uint4 w4 = make_uint4(w[0], w[1], w[2], w[3]);
      fetch(i0 + 32, w);
      if (i0 + 31 < lo0) continue;                        // no query of the block sees a key (wave-uniform)
      *reinterpret_cast<uint4*>(&sSpd[wave][16 * lane]) = w4;
      uint32_t b[4];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) i32x2* lds_i32x2;
        const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)(void*)&sSpd[wave][off_tr8[hh]]);
        b[2 * hh] = (uint32_t)x.x;
        b[2 * hh + 1] = (uint32_t)x.y;
      }
      f32x16 s = zero_f32x16(), dp = zero_f32x16();
      M::rows(sQ + slot * M::TILE, k, s);
      M::rows(sO + slot * M::TILE, v, dp);
      float x[16], slope[16], p[16], ml[16], dl[16];
      bias16(sTab, b, x);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float4 y = *reinterpret_cast<const float4*>(&sStat[slot][16 * g + 4 * u]);
        const float4 z = *reinterpret_cast<const float4*>(&sStat[slot][32 + 16 * g + 4 * u]);
        ml[4 * u] = y.x; ml[4 * u + 1] = y.y; ml[4 * u + 2] = y.z; ml[4 * u + 3] = y.w;
        dl[4 * u] = z.x; dl[4 * u + 1] = z.y; dl[4 * u + 2] = z.z; dl[4 * u + 3] = z.w;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = M::template score<CAP>(s[r], x[r], sc, slope[r]);
        p[r] = M::expo(x[r], ml[r]);
      }
      if (i0 < lo1 || jw + 32 > gr.nk) {
        const int r0 = lo - i0 - 16 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = jok && r >= r0 ? p[r] : 0.0f;
      }
      uint32_t keep = 0;
      if constexpr (DROP) {
        uint32_t rw[8];
        draw16(a, roff, h, (uint32_t)(gr.q0 + i0 + col), jw + 16 * g, rw);
        keep = kept_queries(rw, a.thr);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float d = dp[r];
        if constexpr (DROP) d = (keep >> r) & 1u ? d * a.rp : 0.0f;
        x[r] = p[r] * (d - dl[r]);
        if constexpr (DROP) p[r] = (keep >> r) & 1u ? p[r] : 0.0f;
      }
      if (!wide && __any(((b[0] | b[1] | b[2] | b[3]) & 0x80808080u) != 0)) {
        // the narrow layout ends at 127, which is past its buckets
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t hi = (b[u] >> 7) & 0x01010101u;
          b[u] = (b[u] | hi * 0x7fu) & 0x7f7f7f7fu;
        }
      }
      const int sh = wide ? 7 : 8;
      const uint32_t copy = (uint32_t)(lane & (wide ? 15 : 31)) * 8u;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t at = (((b[r >> 2] >> (8 * (r & 3))) & 0xffu) << sh) | copy;
        atomicAdd(reinterpret_cast<unsigned long long*>(reinterpret_cast<uint8_t*>(hist) + at),
                  (unsigned long long)(long long)__float2int_rn(x[r] * sF));
        if constexpr (CAP) x[r] *= slope[r];
      }
      M::cols(sO + slot * M::TILE, p, dv);
      M::cols(sQ + slot * M::TILE, x, dk);
    }
  }
  {
    // a dS that is no number makes its key's dK so: the head's table gradient is
    // then NaN (the fixed-point sums cannot show it)
    bool ok = true;
#pragma unroll
    for (int r = 0; r < 16; ++r) ok = ok && fabsf(dk[0][r]) < INFINITY;
    const bool any_bad = __any(jok && !ok);
    if (lane == 0) bad[wave] = any_bad;
  }
  if (jb.combine) {
    float* buf = reinterpret_cast<float*>(sBuf);
    auto none = [](int) {};
    auto add = [](int, float& wa, float& wo) { wa = wo = 1.0f; };
    pack_combine(buf, lw, grp, gw, dk, none, add);
    pack_combine(buf, lw, grp, gw, dv, none, add);
  }
  if (jok && (!jb.combine || grp == 0)) {
    const float mk = a.scale * (CAP ? M::kSlope : 1.0f), mv = DROP ? a.rp : 1.0f;
    T* dkp = rows_at<T>(a.dk, h, gr.k0 + j);
    T* dvp = rows_at<T>(a.dv, h, gr.k0 + j);
    M::features(dk, [&](int f, float4 x) { M::store4(dkp + f, make_float4(x.x * mk, x.y * mk, x.z * mk, x.w * mk)); });
    M::features(dv, [&](int f, float4 x) { M::store4(dvp + f, make_float4(x.x * mv, x.y * mv, x.z * mv, x.w * mv)); });
  }
  __syncthreads();
  const int cpy = wide ? 16 : 32;
  const double unscale = ldexp(1.0, -fexp);
  const bool nan = bad[0] | bad[1] | bad[2] | bad[3];
  for (int b = tid; b < a.n_buckets; b += kPackThreads) {
    long long t = 0;
    for (int c = 0; c < cpy; ++c) t += (long long)hist[b * cpy + ((c + b) & (cpy - 1))];
    a.dtab_part[((int64_t)h * a.njobs + pl.job) * a.n_buckets + b] = nan ? (double)NAN : (double)t * unscale;
  }
}

template <class M>
hipError_t launch_pack_dkdv(const PackArgs& a, bool cap, bool drop, hipStream_t s) {
  const dim3 grid(pack_grid(a.njobs, a.H)), block(kPackThreads);
  if (cap && drop)
    hipLaunchKernelGGL((pack_dkdv_kernel<M, true, true>), grid, block, 0, s, a);
  else if (cap)
    hipLaunchKernelGGL((pack_dkdv_kernel<M, true, false>), grid, block, 0, s, a);
  else if (drop)
    hipLaunchKernelGGL((pack_dkdv_kernel<M, false, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((pack_dkdv_kernel<M, false, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

}  // namespace gt
