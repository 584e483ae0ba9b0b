// Sums of the packed kernels' partial results: the forward's key parts, and the
// workgroups' table gradients.
#include "pack.hpp"

namespace gt {

namespace {

// A row's parts, in their order: LSE = log sum_p exp(LSE_p), O = sum_p
// exp(LSE_p - LSE) O_p. One workgroup per merged item and head, 4 features per thread.
template <bool BF16>
__global__ __launch_bounds__(256) void pack_merge_kernel(PackArgs a, int d) {
  const PackMerge mg = a.merges[blockIdx.x / a.H];
  const int h = blockIdx.x % a.H;
  const int cpr = d / 4;
  for (int t = threadIdx.x; t < mg.rows * cpr; t += 256) {
    const int row = t / cpr, f = t % cpr * 4;
    const auto at = [&](int p) { return ((int64_t)(mg.part + p) * a.H + h) * 32 + row; };
    float m = -INFINITY;
    for (int p = 0; p < mg.parts; ++p) {
      const float l = a.lse_part[at(p)];
      m = l > m || isnan(l) ? l : m;
    }
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float lse = -INFINITY;
    if (m != -INFINITY) {
      float tot = 0.0f;
      for (int p = 0; p < mg.parts; ++p) {
        const float lp = a.lse_part[at(p)];
        if (lp == -INFINITY) continue;
        const float w = expf(lp - m);
        const float4 v = *reinterpret_cast<const float4*>(a.o_part + at(p) * d + f);
        tot += w;
        o.x = fmaf(w, v.x, o.x);
        o.y = fmaf(w, v.y, o.y);
        o.z = fmaf(w, v.z, o.z);
        o.w = fmaf(w, v.w, o.w);
      }
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

// dtable[h, b]: the workgroups' sums in a fixed order, 16 threads per bucket.
__global__ __launch_bounds__(256) void pack_dtable_kernel(PackArgs a) {
  __shared__ double red[256];
  const int h = blockIdx.y, b = blockIdx.x * 16 + threadIdx.x % 16;
  double s = 0.0;
  if (b < a.n_buckets)
    for (int j = threadIdx.x / 16; j < a.slots; j += 16)
      s += a.dtab_part[((int64_t)h * a.slots + j) * a.n_buckets + b];
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
