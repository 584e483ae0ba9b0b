// Plan of a packed batch of graphs: which rows and columns each workgroup of
// the packed kernels takes. Host code only; the plan depends on the sizes, the
// prefixes and the number of heads.
//
// Rows are dealt out in blocks of 32 per wave. Where the batch fills the chip, a
// graph gives workgroups of 128 rows, and remainders of up to 64 rows (small graphs
// are nothing else) share a workgroup, 2 or 4 of them, those with the most alike
// numbers of columns together, since a workgroup's waves meet at every tile (512
// graphs of 100 to 256 nodes, d = 8, with their remainders in workgroups of their own:
// forward 80 us and 71 so, dQ 103 and 91, dK / dV 182 and 157). Where it does
// not, 2 or 4 groups of waves take the same rows and a part of the columns each,
// and in the forward with few rows against many keys several workgroups do, whose
// partial results are merged by a kernel of its own.
#include <algorithm>
#include <cstring>
#include <limits>
#include <vector>

#include "../../include/gt_attn.h"
#include "pack_plan.hpp"

namespace gt {
namespace {

constexpr int64_t kMaxNodes = (1LL << 25) - 16;   // 32 rows of distances stay below 2^31 bytes
constexpr int kSlots = 512;                       // workgroups that run at a time: two per compute unit

// Longest graph of the one-pass backward: P and dP of 128 keys are 128 registers.
constexpr int32_t kShortRows = 128;

enum Stage { kForward, kDq, kDkdv };

struct Graph {
  int32_t q0, nq, k0, nk, prefix, ld;
  int64_t spd;
};

// A group of a job before its waves are written out.
struct Group {
  int32_t graph, row0, c0, c1, part;
};
struct Job {
  int32_t group;       // first of its 4 / W groups
  int32_t log2w, combine, steps;
  int32_t cost;        // 32 x 32 blocks of its longest wave
};

struct Plan {
  std::vector<Group> groups;
  std::vector<Job> jobs;
  std::vector<PackMerge> merges;
  int32_t parts = 0;
};

int32_t clamp32(int64_t x, int64_t lo, int64_t hi) { return (int32_t)std::min(std::max(x, lo), hi); }

// Columns that rows [row0, row0 + rows) of a graph meet.
void columns(const Graph& g, Stage st, int32_t row0, int32_t rows, int32_t& c0, int32_t& c1) {
  const int64_t off = (int64_t)g.nk - g.nq;
  if (st != kDkdv) {
    const int64_t last = std::min<int64_t>(g.nq, (int64_t)row0 + rows) - 1;
    c0 = 0;
    c1 = clamp32(std::max<int64_t>(g.prefix, last + off + 1), 0, g.nk);
  } else {
    c0 = row0 < g.prefix ? 0 : clamp32(row0 - off, 0, g.nq) / 32 * 32;
    c1 = g.nq;
  }
}

struct Item {
  Group g;
  int32_t cost;       // blocks per wave
};

// The jobs of one stage with 128 / s rows per workgroup (s = 1, 2, 4).
Plan build(const std::vector<Graph>& graphs, int32_t H, Stage st, int s) {
  Plan p;
  std::vector<std::vector<Item>> whole(3);         // by log2w: groups that share a workgroup with others
  std::vector<std::pair<Item, int>> split;         // combined: item, log2w
  for (size_t gi = 0; gi < graphs.size(); ++gi) {
    const Graph& g = graphs[gi];
    const int32_t rows = st == kDkdv ? g.nk : g.nq;
    int32_t step;
    for (int32_t r = 0; r < rows; r += step) {
      int lw = s == 1 ? 2 : (s == 2 ? 1 : 0);
      while (lw > 0 && rows - r <= (32 << (lw - 1))) --lw;
      step = 32 << lw;
      Item it{{(int32_t)gi, r, 0, 0, -1}, 0};
      columns(g, st, r, step, it.g.c0, it.g.c1);
      it.cost = (it.g.c1 - it.g.c0 + 31) / 32;
      if (s == 1)
        whole[lw].push_back(it);
      else
        split.push_back({it, lw});
    }
  }
  for (int lw = 0; lw < 3; ++lw) {
    auto& w = whole[lw];
    std::stable_sort(w.begin(), w.end(), [](const Item& a, const Item& b) { return a.cost > b.cost; });
    const int n = kPackWaves >> lw;
    for (size_t i = 0; i < w.size(); i += n) {
      const Job j{(int32_t)p.groups.size(), lw, 0, (w[i].cost + (1 << lw) - 1) >> lw, w[i].cost};
      for (int k = 0; k < n; ++k)
        p.groups.push_back(i + k < w.size() ? w[i + k].g : Group{-1, 0, 0, 0, -1});
      p.jobs.push_back(j);
    }
  }
  // Parts: with 32-row workgroups that still leave the chip empty, as many per
  // item as make all about equally long.
  int32_t target = std::numeric_limits<int32_t>::max();
  if (st == kForward && s == 4) {
    int64_t sum = 0;
    int32_t top = 0;
    for (auto& it : split) {
      sum += it.first.cost;
      top = std::max(top, it.first.cost);
    }
    const int64_t even = std::max<int64_t>(16, (sum * H + kSlots - 1) / kSlots);
    // (a merge costs a launch, about 8 blocks: 4 waves share an item's blocks)
    if ((int64_t)split.size() * H < kSlots && top / 4 > even / 4 + 8) target = (int32_t)even;
  }
  for (auto& e : split) {
    const Item& it = e.first;
    const int lw = e.second, n = kPackWaves >> lw;
    const int32_t unit = n * (32 << lw);             // columns per step of a combined workgroup
    const int32_t cols = it.g.c1 - it.g.c0;
    int32_t parts = 1;
    if (it.cost > target) parts = std::min((it.cost + target - 1) / target, (cols + unit - 1) / unit);
    int32_t per_part = (cols + parts - 1) / std::max(parts, 1);
    per_part = (per_part + unit - 1) / unit * unit;
    parts = per_part > 0 ? std::max(1, (cols + per_part - 1) / per_part) : 1;
    if (parts > 1) {
      const Graph& g = graphs[it.g.graph];
      p.merges.push_back({g.q0 + it.g.row0, std::min(32 << lw, g.nq - it.g.row0), p.parts, parts});
    }
    for (int32_t k = 0; k < parts; ++k) {
      const int32_t a = it.g.c0 + k * per_part, b = parts == 1 ? it.g.c1 : std::min(it.g.c1, a + per_part);
      const int32_t per = ((b - a + n - 1) / n + (32 << lw) - 1) / (32 << lw) * (32 << lw);
      const Job j{(int32_t)p.groups.size(), lw, n > 1 ? 1 : 0, per / (32 << lw), per / 32};
      for (int i = 0; i < n; ++i) {
        Group g = it.g;
        g.c0 = (int32_t)std::min<int64_t>(a + (int64_t)i * per, b > a ? (b + 31) / 32 * 32 : a);
        g.c1 = (int32_t)std::max<int64_t>(g.c0, std::min<int64_t>(a + (int64_t)(i + 1) * per, b));
        g.part = parts > 1 ? p.parts : -1;
        p.groups.push_back(g);
      }
      if (parts > 1) ++p.parts;
      p.jobs.push_back(j);
    }
  }
  std::stable_sort(p.jobs.begin(), p.jobs.end(), [](const Job& a, const Job& b) { return a.cost > b.cost; });
  return p;
}

std::vector<PackWave> waves(const std::vector<Graph>& graphs, const Plan& p) {
  std::vector<PackWave> out;
  out.reserve(p.jobs.size() * kPackWaves);
  for (const Job& j : p.jobs)
    for (int w = 0; w < kPackWaves; ++w) {
      const Group& g = p.groups[j.group + (w >> j.log2w)];
      const Graph x = g.graph >= 0 ? graphs[g.graph] : Graph{};
      out.push_back({x.q0, x.nq, x.k0, x.nk, g.row0 + (w & ((1 << j.log2w) - 1)) * 32, g.c0, g.c1, x.prefix, x.spd,
                     x.ld, g.part, j.log2w, j.combine, j.steps, 0});
    }
  return out;
}

// How long a plan takes, in 32 x 32 blocks of a workgroup alone on its compute unit:
// its longest workgroup, or the work over what the chip does with two on every unit
// (1.4 times one; each then runs at 0.7, and in the forward, of which a unit takes
// four, at 0.53: 16 causal graphs of up to 2400 nodes 85 us unsplit, 71 with two
// groups). Sharing rows between groups of waves costs
// more copies and barriers per block (1, 1.05 and 1.2 with 1, 2 and 4 groups) and
// the addition of their results. Forward and backward over 20 batches of 500 to
// 16384 nodes, bf16 and fp32, head dims 16 to 64: within 5 % of the best of the three
// nearly everywhere (7651 nodes, d = 64, bf16, backward: 888 / 947 / 1099 us with 1 / 2 /
// 4; 1000 nodes 99 / 64 / 49; 16 graphs of 300: 59 / 71 / 80).
// full: the work bounds it, which a further split only adds to.
double span(const Plan& p, int32_t H, Stage st, int s, bool& full) {
  const double per_block = s == 1 ? 1.0 : (s == 2 ? 1.05 : 1.2);
  double sum = 0.0, top = 0.0;
  for (const Job& j : p.jobs) {
    const double c = j.cost * per_block + (j.combine ? 5.0 : 3.0);
    sum += c;
    top = std::max(top, c);
  }
  const double wgs = (double)p.jobs.size() * H;
  double slower = wgs <= 256.0 ? 1.0 : 1 / 0.7;
  if (st == kForward && wgs > 512.0) slower += 0.235 * (std::min(wgs / 256, 4.0) - 2.0);
  const double work = sum * H / (256 * 1.4);
  full = work >= top * slower;
  return std::max(work, top * slower) + (p.parts ? 8.0 : 0.0);
}

// The plans of the three stages. dQ's are the forward's where that has no parts, and
// dK / dV's are dQ's in a batch without prefixes whose graphs have as many queries as
// keys: each is built once, and lies in the plan once.
class Plans {
 public:
  Plans(const std::vector<Graph>& graphs, int32_t H) : graphs_(graphs), H_(H) {
    for (const Graph& g : graphs)
      square_ = square_ && g.nq == g.nk && g.prefix == std::numeric_limits<int32_t>::max();
  }
  const Plan* best(Stage st) {
    const Plan* best = nullptr;
    double cost = 0.0;
    bool full = false;
    for (int i = 0; i < 3 && !full; ++i) {
      const Plan& p = get(st, i);
      const double c = span(p, H_, st, 1 << i, full);
      if (!best || c < 0.97 * cost) {
        cost = c;
        best = &p;
      }
    }
    return best;
  }

 private:
  const Plan& get(Stage st, int i) {
    if (st == kDkdv && square_) st = kDq;
    if (st == kDq && made_[kForward][i] && plans_[kForward][i].parts == 0) st = kForward;
    if (!made_[st][i]) {
      plans_[st][i] = build(graphs_, H_, st, 1 << i);
      made_[st][i] = true;
    }
    return plans_[st][i];
  }
  const std::vector<Graph>& graphs_;
  const int32_t H_;
  bool square_ = true, made_[3][3] = {};
  Plan plans_[3][3];
};

// Workgroups per head of the key-stationary kernel, which take one job after the
// other: the table, the histogram and its sums cost about as much as 16 blocks,
// so short jobs share a workgroup as long as the chip stays full. Long ones get one
// each, dealt out longest first as workgroups end.
int32_t slots(const Plan& p, int32_t H, int resident) {
  const int64_t n = (int64_t)p.jobs.size();
  int64_t sum = 0;
  for (const Job& j : p.jobs) sum += j.cost;
  const int64_t by_work = (sum + 15) / 16;
  const int64_t full = (256 * resident + H - 1) / H;
  return (int32_t)std::min(n, std::max(by_work, full));
}

// The list of the one-pass backward, and the blocks of 32 rows that a graph has at most:
// one group per graph, of the waves that its longer side takes. Empty if a graph is
// longer.
std::vector<PackWave> short_list(const std::vector<Graph>& graphs, int32_t& blocks) {
  std::vector<PackWave> out;
  int32_t top = 0;
  for (const Graph& g : graphs) top = std::max(top, std::max(g.nq, g.nk));
  blocks = top <= 64 ? 2 : 4;
  if (top > kShortRows) return out;
  for (int32_t lw = 2; lw >= 0; --lw) {
    for (const Graph& g : graphs) {
      const int32_t n = std::max(g.nq, g.nk);
      if (n == 0 || (n > 64 ? 2 : (n > 32 ? 1 : 0)) != lw) continue;
      for (int32_t w = 0; w < 1 << lw; ++w)
        out.push_back({g.q0, g.nq, g.k0, g.nk, w * 32, 0, g.nk, g.prefix, g.spd, g.ld, -1, lw, 0, 1, 0});
    }
    while (out.size() % kPackWaves) out.push_back({0, 0, 0, 0, 0, 0, 0, 0, 0, 0, -1, lw, 0, 1, 0});
  }
  return out;
}

template <typename T>
int64_t place(size_t& at, const std::vector<T>& v, uint8_t* buf) {
  const size_t off = at;
  const size_t n = v.size() * sizeof(T);
  if (buf && n) std::memcpy(buf + off, v.data(), n);
  at = (off + n + 255) / 256 * 256;
  return (int64_t)off;
}

gt_status_t make(int32_t G, int32_t H, const int32_t* n_q, const int32_t* n_k, const int32_t* prefix,
                 const int64_t* spd_off, const int64_t* spd_ld, bool backward, void* plan, size_t plan_bytes,
                 gt_attn_pack_t* out) {
  std::vector<Graph> graphs;
  graphs.reserve(G);
  gt_attn_pack_t info{};
  int64_t behind = 0;                    // byte behind the graphs so far, one behind the other
  for (int32_t g = 0; g < G; ++g) {
    const int32_t a = n_q[g], b = n_k[g];
    if (a < 0 || b < 0) return GT_ERR_INVALID;
    if (a > kMaxNodes || b > kMaxNodes) return GT_ERR_UNSUPPORTED;
    if (prefix && prefix[g] < 0) return GT_ERR_INVALID;
    const int64_t ld = spd_ld ? spd_ld[g] : b;
    const int64_t off = spd_off ? spd_off[g] : behind;
    if (ld < b || off < 0) return GT_ERR_INVALID;
    if (ld > kMaxNodes) return GT_ERR_UNSUPPORTED;
    behind += (int64_t)a * ld;
    if (a > 0 && b > 0) {
      const int64_t last = (int64_t)(a - 1) * ld + b;
      if (off > std::numeric_limits<int64_t>::max() - last) return GT_ERR_INVALID;
      info.spd_bytes = std::max(info.spd_bytes, off + last);
    }
    // (a graph without pairs has no distances: the place and stride given for it, checked
    // against no buffer, stay out of the records)
    const bool pairs = a > 0 && b > 0;
    graphs.push_back({(int32_t)info.total_q, a, (int32_t)info.total_k, b,
                      prefix ? prefix[g] : std::numeric_limits<int32_t>::max(), pairs ? (int32_t)ld : b,
                      pairs || !(spd_off || spd_ld) ? off : 0});
    info.total_q += a;
    info.total_k += b;
    if (info.total_q > std::numeric_limits<int32_t>::max() || info.total_k > std::numeric_limits<int32_t>::max())
      return GT_ERR_UNSUPPORTED;
  }
  info.n_graphs = G;
  info.H = H;
  info.backward = backward;
  Plans plans(graphs, H);
  const Plan* chosen[3] = {};
  std::vector<PackWave> lists[3];
  const Stage stages[3] = {kForward, kDq, kDkdv};
  for (int i = 0; i < (backward ? 3 : 1); ++i) {
    chosen[i] = plans.best(stages[i]);
    const Plan& p = *chosen[i];
    // (a launch counts its threads in 32 bits)
    if (((int64_t)p.jobs.size() + 8) * H * kPackWaves * 64 > std::numeric_limits<uint32_t>::max())
      return GT_ERR_UNSUPPORTED;
    if (std::find(chosen, chosen + i, &p) == chosen + i) lists[i] = waves(graphs, p);
    info.jobs[i] = (int32_t)p.jobs.size();
    if (i == kForward) {
      info.merges = (int32_t)p.merges.size();
      info.parts = p.parts;
    }
    if (i == kDkdv) {
      info.slots = slots(p, H, 2);
      info.slots3 = slots(p, H, 3);
    }
  }
  std::vector<PackWave> shorts;
  info.short_blocks = 2;
  if (backward) shorts = short_list(graphs, info.short_blocks);
  info.short_jobs = (int32_t)(shorts.size() / kPackWaves);
  info.short_slots = std::min(info.short_jobs, (3 * 256 + H - 1) / H);
  auto lay_out = [&](uint8_t* buf) {
    size_t at = 0;
    for (int i = 0; i < 3; ++i) {
      const int same = (int)(std::find(chosen, chosen + i, chosen[i]) - chosen);
      info.job_off[i] = same < i ? info.job_off[same] : place(at, lists[i], buf);
    }
    info.merge_off = place(at, chosen[kForward]->merges, buf);
    info.short_off = place(at, shorts, buf);
    info.plan_bytes = (int64_t)at;
  };
  lay_out(nullptr);
  *out = info;
  if (plan) {
    if (plan_bytes < (size_t)info.plan_bytes) return GT_ERR_WORKSPACE;
    std::memset(plan, 0, (size_t)info.plan_bytes);
    lay_out(static_cast<uint8_t*>(plan));
  }
  return GT_OK;
}

}  // namespace
}  // namespace gt

extern "C" gt_status_t gt_attn_pack_plan(int32_t n_graphs, int32_t H, const int32_t* n_q, const int32_t* n_k,
                                         const int32_t* prefix, const int64_t* spd_off, const int64_t* spd_ld,
                                         int32_t backward, void* plan, size_t plan_bytes, gt_attn_pack_t* info) {
  if (n_graphs < 1 || H < 1 || H > 65535 || !n_q || !n_k || !info) return GT_ERR_INVALID;
  try {
    return gt::make(n_graphs, H, n_q, n_k, prefix, spd_off, spd_ld, backward != 0, plan, plan_bytes, info);
  } catch (...) {     // out of host memory
    return GT_ERR_WORKSPACE;
  }
}
