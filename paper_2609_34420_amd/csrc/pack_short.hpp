// Backward of packed batches whose graphs have at most 64 (NK = 2) or 128 (NK = 4)
// queries and keys, bf16 (instantiated in pack_short.hip): dQ, dK, dV and the table
// gradient in one pass.
//
// A wave has 32 queries and all the keys of its graph, up to NK blocks of 32, so a
// row's P and dP stay in registers until its sum D = sum_j P z dP is whole: D is
// exact, O is not needed, and each score is formed once.
//   S^T = K Q^T, dP^T = V dO^T, dS = P (z dP / (1 - p) - D), dU = dS (1 - tanh^2),
//   dQ^T = K^T dU^T from registers; P and dU then go to LDS as bf16 tiles, queries as
//   rows, and the wave that has the key block takes dV^T = dO^T P and dK^T = Q^T dU,
//   both operands read transposed.
// K, Q and dO are staged (their products run down the rows), V's operand comes
// straight from global memory.
//
// Table gradient: as in pack_dkdv.hpp, in an LDS histogram that lives through all jobs
// of the workgroup. Its scale 2^F follows the largest |dS| met so far: it only
// falls, and the sums are shifted when it does. The workgroups take job after job and
// give one sum each.
//
// P and dU are rounded to bf16 as the operands of their products (2^-8 of a term); the
// cap's slope waits in fp16, two to a register (2^-11 of dU; 1 - tanh^2 comes out of
// fp32 with an error of 2^-22 at least, fp16's step at the low end).
//
// Bound: set-up and latency of jobs of one or two blocks, and issue (vector units busy
// 74 %, with a third or half of the lanes past their graph): 1024 graphs of 9 to 60
// nodes, H = 8, d = 8, cap: 31 us. The whole backward, for that of two passes: those 41 for
// 63; 4000 of 50 to 64: 172 for 269; 2048 of 16 to 40 at d = 64, 256 buckets: 185 for 238;
// 2048 of 85 to 92 at d = 16, cap: 296 for 348. Longer graphs keep the two passes: their
// P and dP do not fit a wave's registers, and D from O is not exact enough for the table
// gradient. A job's record read a job ahead gained 1 %.
#pragma once
#include "pack.hpp"

namespace gt {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// NK: blocks of 32 keys that a graph has at most (2 or 4).
template <class M, int NK, bool CAP, bool DROP, bool WIDE>
__global__ __launch_bounds__(kPackThreads, NK == 2 && M::D == 32 && !(CAP && DROP) ? 3 : 2) void pack_short_kernel(PackArgs a) {
  constexpr int NA = M::NA, D = M::D;
  constexpr int CPY = WIDE ? 16 : 32;
  constexpr int PT = 32 * 32;                               // elements of a tile of P or dU
  extern __shared__ unsigned long long hist[];              // a.hist buckets of CPY copies
  __shared__ alignas(4096) float sTab[256];
  __shared__ alignas(128) uint16_t sK[kPackWaves][M::TILE], sQ[kPackWaves][M::TILE], sO[kPackWaves][M::TILE];
  __shared__ alignas(128) uint16_t sX[kPackWaves][NK][PT];
  __shared__ float red[kPackWaves];
  __shared__ int bad[kPackWaves];
  static_assert(sizeof sTab + 3 * sizeof sK + sizeof sX + sizeof red + sizeof bad == short_lds(D, NK));

  const PackPlace pl(a, a.slots);
  if (pl.job >= a.slots) return;
  const int h = pl.h;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, col = lane & 31, g = lane >> 5;
  constexpr bool START = !CAP;
  sTab[tid] = M::entry(tid < a.n_buckets ? a.table[(int64_t)h * a.n_buckets + tid] : 0.0f, a, START)
              + (CAP ? a.cap * kLog2e : 0.0f);
  for (int t = tid; t < a.n_buckets * CPY / 2; t += kPackThreads)
    reinterpret_cast<uint4*>(hist)[t] = make_uint4(0u, 0u, 0u, 0u);
  const ScoreConst sc = M::consts(a, CAP);
  const Philox rng(a, h);
  const float rp = DROP ? a.rp : 1.0f;
  const PackDma<M> cq(a.q.rs), ck(a.k.rs), co(a.d_o.rs);
  const float mk = a.scale * rp * (CAP ? M::kSlope : 1.0f);
  const uint32_t copy = (uint32_t)(lane & (CPY - 1)) * 8u;
  const int p0 = tr_operand_off<32>(0, 0), p1 = tr_operand_off<32>(1, 0);
  int fexp = 90;
  bool any_bad = false;

  for (int job = pl.job; job < a.njobs; job += a.slots) {
    const PackWave gr = scalar_record(a.jobs + (int64_t)job * kPackWaves + wave);
    const int lw = gr.log2w, W = 1 << lw;
    const int grp = wave >> lw, gw = wave & (W - 1);
    const int iw = gr.row, i = iw + col;                   // the wave's first query and key, the lane's
    const bool active = iw < gr.nq, iok = i < gr.nq, jok = i < gr.nk;
    const int ic = iok ? i : (active ? gr.nq - 1 : 0);
    const int vis = ic + gr.nk - gr.nq + 1 > gr.prefix ? ic + gr.nk - gr.nq + 1 : gr.prefix;
    const int lim = iok ? (vis < gr.nk ? vis : gr.nk) : 0;    // visible keys of the lane's query

    const int il = iw + 31 < gr.nq ? iw + 31 : gr.nq - 1;
    const int vl = il + gr.nk - gr.nq + 1 > gr.prefix ? il + gr.nk - gr.nq + 1 : gr.prefix;
    const int lim1 = active ? (vl < gr.nk ? vl : gr.nk) : 0;  // of the wave's queries

    lds_barrier();                                          // the last job's tiles are read, the table is written
    cq.load(rows_at<const uint16_t>(a.q, h, gr.q0), a.q.rs, iw, gr.nq, sQ[wave]);
    co.load(rows_at<const uint16_t>(a.d_o, h, gr.q0), a.d_o.rs, iw, gr.nq, sO[wave]);
    ck.load(rows_at<const uint16_t>(a.k, h, gr.k0), a.k.rs, iw, gr.nk, sK[wave]);
    typename M::Operand q, d_o, v[2];
    M::load_operand(rows_at<const uint16_t>(a.q, h, gr.q0 + ic), active, 1.0f, q);
    M::load_operand(rows_at<const uint16_t>(a.d_o, h, gr.q0 + ic), iok, 1.0f, d_o);
    const uint16_t* vh = rows_at<const uint16_t>(a.v, h, gr.k0);
    const PackSpdRow spd(a.spd + gr.spd + (int64_t)(active ? iw : 0) * gr.ld, gr.ld, active ? gr.nq - iw : 1,
                         active ? gr.nk : 0);
    uint32_t w[NK][5];
    auto load_v = [&](int kb) {
      const int j = kb * 32 + perm32(col);
      M::load_operand(vh + (j < gr.nk ? j : 0) * a.v.rs, j < gr.nk, 1.0f, v[kb & 1]);
    };
#pragma unroll
    for (int kb = 0; kb < NK; ++kb) {
      if (kb < 2) load_v(kb);
      spd.fetch(kb * 32, w[kb]);
    }
    const float lse = iok ? a.lse[h * a.ld_lse + gr.q0 + ic] : -INFINITY;
    const float mlse = lse == -INFINITY ? -INFINITY : -M::to_unit(lse);
    RowDraw rrow{};
    if constexpr (DROP) rrow = rng.row((uint32_t)(gr.q0 + i));
    wait_vmcnt<0>();
    lds_barrier();                                          // the tiles have landed

    // tile: queries as rows, the lane's row from key 16 g on
    auto put = [&](uint16_t* tile, const float (&y)[16]) {
      *reinterpret_cast<bf16x8*>(tile + col * 32 + swz_tile<32>(col, 2 * g) * 8) = cvt_bf16x8(y);
      *reinterpret_cast<bf16x8*>(tile + col * 32 + swz_tile<32>(col, 2 * g + 1) * 8) = cvt_bf16x8(y + 8);
    };
    // P (in x), z dP (in dp) and the slope of both key blocks, z P into its tile; the
    // sum of P z dP
    float x[NK][16], dp[NK][16];
    f16x2 slope[NK][8];
    float dsum = 0.0f;
#pragma unroll
    for (int kb = 0; kb < NK; ++kb) {
      if (kb * 32 >= lim1) {                                // no visible key (wave-uniform)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[kb][r] = dp[kb][r] = 0.0f;
        put(sX[wave][kb], x[kb]);
        continue;
      }
      align_spd5(w[kb], spd.sh);
      bias16(sTab, w[kb], x[kb]);
      f32x16 s = zero_f32x16(), t = zero_f32x16();
      if constexpr (START) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = x[kb][r];
      }
      M::rows(sK[(grp << lw) + kb], q, s);
#pragma unroll
      for (int kc = 0; kc < (M::DS + 15) / 16; ++kc) t = mfma32(v[kb & 1].f[kc], d_o.f[kc], t);
      if (kb + 2 < NK) load_v(kb + 2);
      if constexpr (START) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[kb][r] = fmaf(s[r], sc.mul, mlse);
      } else {
        float sl[16];
        M::template scores<CAP, true>(s, x[kb], sl, sc);
#pragma unroll
        for (int r = 0; r < 16; r += 2) slope[kb][r / 2] = f16x2{(_Float16)sl[r], (_Float16)sl[r + 1]};
#pragma unroll
        for (int r = 0; r < 16; ++r) x[kb][r] += mlse;
      }
      keep_below(x[kb], lim - kb * 32 - 16 * g, -INFINITY);
      uint32_t rw[8];
      if constexpr (DROP) {
        rng.draw(rrow, rng.keys((uint32_t)(kb * 32 + 16 * g) / 8u), rw);
        rng.draw(rrow, rng.keys((uint32_t)(kb * 32 + 16 * g) / 8u + 1u), rw + 4);
      }
      float zp[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[kb][r] = M::expo(x[kb][r]);
        dp[kb][r] = t[r];
        zp[r] = x[kb][r];
        if constexpr (DROP) {
          const bool keep = kept(rw, r, a.thr);
          dp[kb][r] = keep ? dp[kb][r] : 0.0f;
          zp[r] = keep ? zp[r] : 0.0f;
        }
        dsum = fmaf(x[kb][r], dp[kb][r], dsum);
      }
      put(sX[wave][kb], zp);
    }
    dsum += __shfl_xor(dsum, 32);                           // D (1 - p)
    float dmax = 0.0f;
#pragma unroll
    for (int kb = 0; kb < NK; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[kb][r] *= dp[kb][r] - dsum;                       // dS (1 - p)
        dmax = fmaxf(dmax, fabsf(x[kb][r]));
      }
    dmax = wave_max(dmax);
    if (lane == 0) red[wave] = dmax;
    lds_barrier();
    const float top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    if (top > 0.0f && top < INFINITY) {
      int e;
      frexpf(top, &e);                                      // top < 2^e
      if (30 - e < fexp) {
        const int down = fexp - (30 - e);
        fexp = 30 - e;
        for (int t = tid; t < a.n_buckets * CPY; t += kPackThreads) {
          const long long y = (long long)hist[t];
          hist[t] = (unsigned long long)(down < 63 ? (y + (1ll << (down - 1))) >> down : 0ll);
        }
        lds_barrier();
      }
    }
    const float sF = ldexpf(1.0f, fexp);
    f32x16 acc[NA];
#pragma unroll
    for (int c = 0; c < NA; ++c) acc[c] = zero_f32x16();
#pragma unroll
    for (int kb = 0; kb < NK; ++kb) {
      if (kb * 32 >= lim1) continue;
      uint32_t (&b)[5] = w[kb];
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
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t at = WIDE ? ((((b[r >> 2] >> (8 * (r & 3))) & 0xffu) << 7) | copy)
                                 : __builtin_amdgcn_perm(b[r >> 2], copy, 0x0c0c0000u | ((4u + (r & 3)) << 8));
        unsigned long long* e = reinterpret_cast<unsigned long long*>(reinterpret_cast<uint8_t*>(hist) + at);
        if (r % 2 == 0)
          add_term<0>(e, x[kb][r] * sF);
        else
          add_term<1>(e, x[kb][r] * sF);
        if constexpr (CAP) x[kb][r] *= (float)slope[kb][r / 2][r & 1];
      }
      M::cols(sK[(grp << lw) + kb], x[kb], acc);
    }
    if (iok) {
      uint16_t* out = rows_at<uint16_t>(a.dq, h, gr.q0 + i);
      M::features(acc, [&](int f, float4 y) {
        M::store4(out + f, make_float4(y.x * mk, y.y * mk, y.z * mk, y.w * mk));
      });
    }
    // a dS that is no number makes its row's dQ so
    bool ok = true;
#pragma unroll
    for (int r = 0; r < 16; ++r) ok = ok && fabsf(acc[0][r]) < INFINITY;
    any_bad = any_bad || __any(iok && !ok);

    auto product = [&](const uint16_t* rows, const uint16_t* tile, f32x16 (&y)[NA]) {
      M::cols(rows, lds_tr_operand(tile, p0, p1), lds_tr_operand(tile + 8 * 32, p0, p1), y);
    };
    auto store = [&](const PackTensor& t, const f32x16 (&y)[NA], float mul) {
      if (!jok) return;
      uint16_t* out = rows_at<uint16_t>(t, h, gr.k0 + i);
      M::features(y, [&](int f, float4 z) {
        M::store4(out + f, make_float4(z.x * mul, z.y * mul, z.z * mul, z.w * mul));
      });
    };
#pragma unroll
    for (int c = 0; c < NA; ++c) acc[c] = zero_f32x16();
    f32x16 acc2[NA];
#pragma unroll
    for (int c = 0; c < NA; ++c) acc2[c] = zero_f32x16();
    if (lw == 0) {
      put(sX[wave][1], x[0]);
      lds_barrier();
      product(sO[wave], sX[wave][0], acc);
      product(sQ[wave], sX[wave][1], acc2);
    } else {
      const int nqb = (gr.nq + 31) / 32;
      for (int qb = 0; qb < nqb; ++qb) product(sO[(grp << lw) + qb], sX[(grp << lw) + qb][gw], acc);
      lds_barrier();
#pragma unroll
      for (int kb = 0; kb < NK; ++kb) put(sX[wave][kb], x[kb]);
      lds_barrier();
      for (int qb = 0; qb < nqb; ++qb) product(sQ[(grp << lw) + qb], sX[(grp << lw) + qb][gw], acc2);
    }
    store(a.dv, acc, rp);
    store(a.dk, acc2, mk);
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

template <class M, int NK, bool CAP, bool DROP>
void launch_pack_short_nb(PackArgs a, hipStream_t s) {
  const dim3 grid(pack_grid(a.slots, a.H)), block(kPackThreads);
  const int lds = hist_bytes(a.n_buckets);
  a.hist = hist_buckets(a.n_buckets);
  if constexpr (NK == 2) {
    if (a.hist == 256) {
      hipLaunchKernelGGL((pack_short_kernel<M, NK, CAP, DROP, true>), grid, block, lds, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((pack_short_kernel<M, NK, CAP, DROP, false>), grid, block, lds, s, a);
}

// (NK = 4: without both cap and dropout and with up to 64 buckets, as its caller sees to)
template <class M, int NK>
hipError_t launch_pack_short(const PackArgs& a, bool cap, bool drop, hipStream_t s) {
  if (NK == 4 && ((cap && drop) || a.n_buckets > 64)) return hipErrorInvalidValue;
  if (cap && drop) {
    if constexpr (NK == 2) launch_pack_short_nb<M, NK, true, true>(a, s);
  } else if (cap) {
    launch_pack_short_nb<M, NK, true, false>(a, s);
  } else if (drop) {
    launch_pack_short_nb<M, NK, false, true>(a, s);
  } else {
    launch_pack_short_nb<M, NK, false, false>(a, s);
  }
  return hipGetLastError();
}

}  // namespace

}  // namespace gt
