// Records of a packed batch's plan (built on the host by pack_plan.hip, read
// by the pack_*.hip kernels).
#pragma once
#include <stdint.h>

namespace gt {

// A workgroup of a packed kernel has 4 waves, each with 32 stationary rows
// (queries, or keys in the key-stationary kernel), and streams the rows of the
// other side as columns, 32 staged rows per wave at a time. Its waves form
// 4 / W groups of W waves (W = 1 << log2w); a group has up to 32 W rows of one
// graph and a range of columns. A job is what a workgroup takes at a time: 4
// records, one per wave, so that a wave knows its work after one read.
constexpr int kPackWaves = 4;

struct PackWave {
  int32_t q0, nq;      // the graph's first packed query row, and its query rows
  int32_t k0, nk;      // the same of its keys
  int32_t row;         // the wave's first stationary row, counted in the graph
  int32_t c0, c1;      // its group's columns [c0, c1), counted in the graph; c0 a multiple of 32
  int32_t prefix;      // key j is visible to query i if j < prefix or j <= i + nk - nq
  int64_t spd;         // byte offset of the graph's distances
  int32_t ld;          // their row stride (nk in a graph without pairs)
  int32_t part;        // slot of a partial result, or -1
  int32_t log2w;
  int32_t combine;     // 1: the job's groups have the same rows; their results are added up
  int32_t steps;       // tiles of 32 W columns that the job's longest group takes
  int32_t pad;
};

// Rows whose partial results (slots part .. part + parts - 1) are merged.
struct PackMerge {
  int32_t row, rows, part, parts;
};

}  // namespace gt
