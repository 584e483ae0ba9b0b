// Sums of the packed kernels' partial results: the forward's key parts, and the
// workgroups' table gradients.
#include "pack.hpp"

namespace gt {

namespace {

// A row's parts, in their order: LSE = log sum_p exp(LSE_p), O = sum_p
// exp(LSE_p - LSE) O_p. One workgroup per merged item and head, 4 features per thread.
// A launch and one pass of latency: 4.8 us for the new nodes of 16 graphs (7.8
// with one load in flight).
template <bool BF16>
__global__ __launch_bounds__(256) void pack_merge_kernel(PackArgs a, int d) {
  const PackMerge mg = a.merges[blockIdx.x / a.H];
  const int h = blockIdx.x % a.H;
  const int cpr = d / 4;
  for (int t = threadIdx.x; t < mg.rows * cpr; t += 256) {
    const int row = t / cpr, f = t % cpr * 4;
    const auto at = [&](int p) { return ((int64_t)(mg.part + p) * a.H + h) * 32 + row; };
    // one pass with a running maximum, 8 parts' loads in flight
    float m = -INFINITY, tot = 0.0f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < mg.parts; p0 += 8) {
      float l[8];
      float4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t x = at(p0 + k < mg.parts ? p0 + k : p0);
        l[k] = a.lse_part[x];
        v[k] = *reinterpret_cast<const float4*>(a.o_part + x * d + f);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (p0 + k >= mg.parts || l[k] == -INFINITY) continue;
        const float mn = l[k] > m || isnan(l[k]) ? l[k] : m;
        const float wo = m == -INFINITY ? 0.0f : expf(m - mn), w = expf(l[k] - mn);
        m = mn;
        tot = fmaf(tot, wo, w);
        o.x = fmaf(o.x, wo, w * v[k].x);
        o.y = fmaf(o.y, wo, w * v[k].y);
        o.z = fmaf(o.z, wo, w * v[k].z);
        o.w = fmaf(o.w, wo, w * v[k].w);
      }
    }
    float lse = -INFINITY;
    if (m != -INFINITY) {
      const float inv = 1.0f / tot;
      o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
      lse = m + logf(tot);
    }
    const int64_t r = mg.row + row;
    if constexpr (BF16)
      Bf16Pack<32, 32>::store4(rows_at<uint16_t>(a.o, h, r) + f, o);
    else
      *reinterpret_cast<float4*>(rows_at<float>(a.o, h, r) + f) = o;
    if (f == 0) a.lse[h * a.ld_lse + r] = lse;
  }
}

// dtable[h, b]: the workgroups' sums in a fixed order, 16 threads per bucket. A launch
// and one pass of latency: 4.5 us at every size.
__global__ __launch_bounds__(256) void pack_dtable_kernel(PackArgs a) {
  __shared__ double red[256];
  const int h = blockIdx.y, b = blockIdx.x * 16 + threadIdx.x % 16;
  double s = 0.0;
  if (b < a.n_buckets)
    for (int j = threadIdx.x / 16; j < a.slots; j += 16 * 8) {
      double v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = j + 16 * k < a.slots ? a.dtab_part[((int64_t)h * a.slots + j + 16 * k) * a.n_buckets + b] : 0.0;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
  red[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 16 && b < a.n_buckets) {
    for (int k = 1; k < 16; ++k) s += red[k * 16 + threadIdx.x];
    a.dtable[(int64_t)h * a.n_buckets + b] = (float)s;
  }
}

}  // namespace

hipError_t launch_pack_merge(const PackArgs& a, int d, bool bf16, hipStream_t s) {
  const dim3 grid((unsigned)a.nmerges * (unsigned)a.H);
  if (bf16)
    hipLaunchKernelGGL(pack_merge_kernel<true>, grid, dim3(256), 0, s, a, d);
  else
    hipLaunchKernelGGL(pack_merge_kernel<false>, grid, dim3(256), 0, s, a, d);
  return hipGetLastError();
}

hipError_t launch_pack_dtable(const PackArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.n_buckets + 15) / 16, (unsigned)a.H);
  hipLaunchKernelGGL(pack_dtable_kernel, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace gt
