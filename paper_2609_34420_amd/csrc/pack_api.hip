// C ABI of the packed calls: host-side validation, then stream-ordered launches.
#include <cmath>
#include <cstdint>

#include "../../include/gt_attn.h"
#include "pack.hpp"

namespace gt {
namespace {

constexpr int64_t kMaxRowStride = 1LL << 23;     // 32 rows of a tile stay below 2^30 bytes
constexpr float kMinCap = 1.0f / 1024, kMaxCap = 1024.0f;
// Products of scale, its inverse, caps and biases stay finite.
constexpr float kMinScale = 0x1p-64f, kMaxScale = 0x1p64f;

inline size_t pad256(size_t x) { return (x + 255) / 256 * 256; }
inline bool aligned(const void* p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool pack_ok(const gt_attn_pack_t* p) {
  if (!p || p->H < 1 || p->n_graphs < 1 || p->total_q < 0 || p->total_k < 0 || p->spd_bytes < 0) return false;
  for (int i = 0; i < 3; ++i)
    if (p->jobs[i] < 0 || p->job_off[i] < 0) return false;
  return p->merges >= 0 && p->parts >= 0 && p->merge_off >= 0 && p->slots >= 0 && p->slots <= p->slots3 &&
         p->slots3 <= p->jobs[2] &&
         p->short_jobs >= 0 && p->short_off >= 0 && p->short_slots >= 0 && p->short_slots <= p->short_jobs &&
         (p->short_blocks == 2 || p->short_blocks == 4);
}

bool rows_ok(const gt_attn_rows_t* t, int64_t rows, int32_t d, gt_dtype_t dtype) {
  if (!t || t->head_stride < 0) return false;
  if (rows == 0) return true;
  const int64_t q = dtype == GT_BF16 ? 8 : 4;
  return t->p && aligned(t->p, 16) && t->head_stride % q == 0 && t->row_stride % q == 0 && t->row_stride >= d &&
         t->row_stride <= kMaxRowStride;
}

PackTensor tensor(const gt_attn_rows_t* t) { return {t->p, t->head_stride, t->row_stride}; }

// What both calls take.
gt_status_t common(const gt_attn_pack_t* pack, const void* plan, const gt_attn_rows_t* q, const gt_attn_rows_t* k,
                   const gt_attn_rows_t* v, const uint8_t* spd, const float* table, int32_t n_buckets,
                   const gt_attn_rows_t* o, const float* lse, int64_t ld_lse, int32_t d, gt_dtype_t dtype,
                   float scale, float cap, const gt_attn_dropout_t* dropout, PackArgs& a) {
  if (dtype != GT_F32 && dtype != GT_BF16) return GT_ERR_UNSUPPORTED;
  if (d != 8 && d != 16 && d != 32 && d != 64) return GT_ERR_UNSUPPORTED;
  if (!pack_ok(pack)) return GT_ERR_INVALID;
  if (n_buckets < 1 || n_buckets > 256 || !(scale >= kMinScale && scale <= kMaxScale)) return GT_ERR_INVALID;
  if (cap != 0.0f && !(cap >= kMinCap && cap <= kMaxCap)) return GT_ERR_INVALID;
  if (!rows_ok(q, pack->total_q, d, dtype) || !rows_ok(o, pack->total_q, d, dtype) ||
      !rows_ok(k, pack->total_k, d, dtype) || !rows_ok(v, pack->total_k, d, dtype))
    return GT_ERR_INVALID;
  if (!table || (pack->spd_bytes > 0 && !spd)) return GT_ERR_INVALID;
  if (pack->total_q > 0 && (!lse || ld_lse < pack->total_q)) return GT_ERR_INVALID;
  if (pack->plan_bytes > 0 && (!plan || !aligned(plan, 16))) return GT_ERR_INVALID;
  a.rp = 1.0f;
  if (dropout) {
    if (!(dropout->p >= 0.0) || !(dropout->p < 1.0)) return GT_ERR_INVALID;
    const long t = std::lround(dropout->p * 65536.0);
    if (t > 65535) return GT_ERR_INVALID;
    a.thr = (int32_t)t - 32768;
    a.rp = (float)(65536.0 / (65536.0 - (double)t));
    a.seed0 = (uint32_t)dropout->seed;
    a.seed1 = (uint32_t)(dropout->seed >> 32);
    a.offset = dropout->offset;
    a.offset_dev = dropout->offset_dev;
    if (!aligned(a.offset_dev, 4)) return GT_ERR_INVALID;
  } else {
    a.thr = -32768;
  }
  a.q = tensor(q); a.k = tensor(k); a.v = tensor(v); a.o = tensor(o);
  a.lse = const_cast<float*>(lse);
  a.ld_lse = ld_lse;
  a.spd = spd;
  a.table = table;
  a.n_buckets = n_buckets;
  a.H = pack->H;
  a.scale = scale;
  a.cap = cap;
  a.merges = reinterpret_cast<const PackMerge*>(static_cast<const uint8_t*>(plan) + pack->merge_off);
  a.nmerges = pack->merges;
  return GT_OK;
}

// The work list of stage i (0 forward, 1 dQ, 2 dK / dV).
void stage(const gt_attn_pack_t* pack, const void* plan, int i, PackArgs& a) {
  a.jobs = reinterpret_cast<const PackWave*>(static_cast<const uint8_t*>(plan) + pack->job_off[i]);
  a.njobs = pack->jobs[i];
}

// The one-pass backward: faster than two passes wherever it was measured (H = 8, the whole
// call, one pass and two). With up to two blocks of keys 1024 graphs of 9 to 60 nodes, d = 8,
// cap: 41 and 63 us; 300 of 40 to 64, d = 64, cap and dropout: 43 and 79; 2048 of 16 to 40,
// d = 64, 256 buckets, of which one workgroup fits a compute unit: 185 and 238. With up to
// four where two workgroups fit, up to 64 buckets: of 156 batches of 65 to 128 nodes or with
// one such graph the least gain is 2048 of 65 to 96, d = 8, 64 buckets: 233 and 252; 1024 of
// 100 to 128, d = 32, cap: 222 and 293. One workgroup of those to a unit lost (512 of 65 to
// 128, d = 8: 136 and 125), and a cap and dropout together, which take registers, gained
// nothing (2048 of 85 to 92: 466 and 470).
bool short_applies(const gt_attn_pack_t* p, int32_t d, bool cap, bool drop, int32_t n_buckets) {
  return p->short_jobs > 0 &&
         (p->short_blocks == 2 ||
          (d < 64 && !(cap && drop) && short_resident(d, p->short_blocks, cap, drop, n_buckets) == 2));
}

struct FwdParts { size_t lse, bytes; };
FwdParts fwd_parts(const gt_attn_pack_t* p, int32_t d) {
  const size_t rows = (size_t)p->parts * (size_t)p->H * 32;
  const size_t o = pad256(rows * (size_t)d * sizeof(float));
  return {o, o + pad256(rows * sizeof(float))};
}
struct BwdParts { size_t dmax, dtab, bytes; };
BwdParts bwd_parts(const gt_attn_pack_t* p, int32_t n_buckets) {
  const size_t H = (size_t)p->H;
  BwdParts b;
  b.dmax = pad256(H * (size_t)p->total_q * sizeof(float));
  b.dtab = b.dmax + pad256(H * (size_t)p->jobs[1] * sizeof(float2));
  const size_t slots = (size_t)(p->slots3 > p->short_slots ? p->slots3 : p->short_slots);
  b.bytes = b.dtab + pad256(H * slots * (size_t)n_buckets * sizeof(double));
  return b;
}

}  // namespace
}  // namespace gt

extern "C" {

size_t gt_attn_pack_fwd_workspace_size(const gt_attn_pack_t* pack, int32_t d) {
  return gt::pack_ok(pack) && d > 0 ? gt::fwd_parts(pack, d).bytes : 0;
}

size_t gt_attn_pack_bwd_workspace_size(const gt_attn_pack_t* pack, int32_t n_buckets) {
  return gt::pack_ok(pack) && n_buckets > 0 ? gt::bwd_parts(pack, n_buckets).bytes : 0;
}

gt_status_t gt_attn_pack_fwd(const gt_attn_pack_t* pack, const void* plan, const gt_attn_rows_t* q,
                             const gt_attn_rows_t* k, const gt_attn_rows_t* v, const uint8_t* spd,
                             const float* table, int32_t n_buckets, const gt_attn_rows_t* o, float* lse,
                             int64_t ld_lse, void* workspace, size_t workspace_bytes, int32_t d,
                             gt_dtype_t dtype, float scale, float cap, const gt_attn_dropout_t* dropout,
                             void* stream) {
  gt::PackArgs a{};
  const gt_status_t st = gt::common(pack, plan, q, k, v, spd, table, n_buckets, o, lse, ld_lse, d, dtype, scale, cap,
                                    dropout, a);
  if (st != GT_OK) return st;
  const gt::FwdParts ws = gt::fwd_parts(pack, d);
  if (ws.bytes > 0) {
    if (!workspace || workspace_bytes < ws.bytes || !gt::aligned(workspace, 256)) return GT_ERR_WORKSPACE;
    a.o_part = static_cast<float*>(workspace);
    a.lse_part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + ws.lse);
  }
  gt::stage(pack, plan, 0, a);
  if (a.njobs == 0) return GT_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool drop = a.thr > -32768;
  hipError_t e = dtype == GT_BF16 ? gt::launch_pack_fwd_bf16(a, d, cap > 0.0f, drop, s)
                                  : gt::launch_pack_fwd_f32(a, d, cap > 0.0f, drop, s);
  if (e == hipSuccess && a.nmerges > 0) e = gt::launch_pack_merge(a, d, dtype == GT_BF16, s);
  return e == hipSuccess ? GT_OK : GT_ERR_LAUNCH;
}

gt_status_t gt_attn_pack_bwd(const gt_attn_pack_t* pack, const void* plan, const gt_attn_rows_t* q,
                             const gt_attn_rows_t* k, const gt_attn_rows_t* v, const uint8_t* spd,
                             const float* table, int32_t n_buckets, const gt_attn_rows_t* o,
                             const float* lse, int64_t ld_lse, const gt_attn_rows_t* d_o,
                             const gt_attn_rows_t* dq, const gt_attn_rows_t* dk, const gt_attn_rows_t* dv,
                             float* dtable, void* workspace, size_t workspace_bytes, int32_t d,
                             gt_dtype_t dtype, float scale, float cap, const gt_attn_dropout_t* dropout,
                             void* stream) {
  gt::PackArgs a{};
  const gt_status_t st = gt::common(pack, plan, q, k, v, spd, table, n_buckets, o, lse, ld_lse, d, dtype, scale, cap,
                                    dropout, a);
  if (st != GT_OK) return st;
  if (!pack->backward) return GT_ERR_INVALID;
  if (!gt::rows_ok(d_o, pack->total_q, d, dtype) || !gt::rows_ok(dq, pack->total_q, d, dtype) ||
      !gt::rows_ok(dk, pack->total_k, d, dtype) || !gt::rows_ok(dv, pack->total_k, d, dtype) || !dtable)
    return GT_ERR_INVALID;
  const gt::BwdParts ws = gt::bwd_parts(pack, n_buckets);
  if (ws.bytes > 0) {
    if (!workspace || workspace_bytes < ws.bytes || !gt::aligned(workspace, 256)) return GT_ERR_WORKSPACE;
    uint8_t* w = static_cast<uint8_t*>(workspace);
    a.dlt = reinterpret_cast<float*>(w);
    a.dmax = reinterpret_cast<float2*>(w + ws.dmax);
    a.dtab_part = reinterpret_cast<double*>(w + ws.dtab);
  }
  a.ld_dlt = pack->total_q;
  a.d_o = gt::tensor(d_o); a.dq = gt::tensor(dq); a.dk = gt::tensor(dk); a.dv = gt::tensor(dv);
  a.dtable = dtable;
  a.njobs_dq = pack->jobs[1];
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = dtype == GT_BF16, c = cap > 0.0f, drop = a.thr > -32768;
  a.slots = bf16 && gt::dkdv_resident(d, c, drop, n_buckets) == 3 ? pack->slots3 : pack->slots;
  hipError_t e = hipSuccess;
  if (bf16 && gt::short_applies(pack, d, c, drop, n_buckets)) {
    a.jobs = reinterpret_cast<const gt::PackWave*>(static_cast<const uint8_t*>(plan) + pack->short_off);
    a.njobs = pack->short_jobs;
    const int32_t fit = (gt::short_resident(d, pack->short_blocks, c, drop, n_buckets) * 256 + a.H - 1) / a.H;
    a.slots = fit < pack->short_slots ? fit : pack->short_slots;
    e = gt::launch_pack_short_bf16(a, d, pack->short_blocks, c, drop, s);
    if (e == hipSuccess) e = gt::launch_pack_dtable(a, s);
    return e == hipSuccess ? GT_OK : GT_ERR_LAUNCH;
  }
  gt::stage(pack, plan, 1, a);
  if (a.njobs > 0) e = bf16 ? gt::launch_pack_dq_bf16(a, d, c, drop, s) : gt::launch_pack_dq_f32(a, d, c, drop, s);
  if (e != hipSuccess) return GT_ERR_LAUNCH;
  gt::stage(pack, plan, 2, a);
  if (a.njobs > 0) e = bf16 ? gt::launch_pack_dkdv_bf16(a, d, c, drop, s) : gt::launch_pack_dkdv_f32(a, d, c, drop, s);
  if (e == hipSuccess) e = gt::launch_pack_dtable(a, s);
  return e == hipSuccess ? GT_OK : GT_ERR_LAUNCH;
}

}  // extern "C"
