// Sizes of the beam selection's passes and its workspace.  Host code alone (no HIP), so that a
// test can evaluate them.
#pragma once
#include <cstddef>
#include <cstdint>

namespace wici {

constexpr int kMostBeams = 64, kMostChosen = 64;
constexpr int kMostVocab = 1 << 24;
constexpr int kMostRows = 65535;    // searches x beams: a grid's second dimension
constexpr int kLoads = 2;           // 16-byte loads of a lane at a time (8: 35.3 us for 33.0)
constexpr int kMostGroups = 1024;   // whose maxima one workgroup takes, one a work-item

// A row of `vocab` logits as 16-byte blocks from its first one on: the blocks of 64 lanes are one load,
// `per_group` loads (a power of two) one group, whose maximum is kept, and `per_unit` of them, whole
// groups, one wavefront's unit.  Counted is up to one block more than a row has (it holds nothing): as
// many as a row of any alignment has of aligned ones, for which programs keep workspaces.
struct BeamPlan {
  int in_block;   // elements of a block
  int per_group, per_unit;
  int groups, units;
};
inline BeamPlan beam_plan(int vocab, bool bf16) {
  BeamPlan p;
  p.in_block = bf16 ? 8 : 4;
  const int64_t blocks = ((int64_t)vocab + 2 * (p.in_block - 1)) / p.in_block;
  const int64_t loads = (blocks + 63) / 64;
  p.per_group = 1;
  while ((loads + p.per_group - 1) / p.per_group > kMostGroups) p.per_group *= 2;
  p.per_unit = p.per_group > kLoads ? p.per_group : kLoads;
  p.groups = (int)((loads + p.per_group - 1) / p.per_group);
  p.units = (int)((loads + p.per_unit - 1) / p.per_unit);
  return p;
}

// The workspace: byte offsets, each array a multiple of 16 bytes apart.
struct BeamSpace {
  size_t sum, lse;        // double [rows][units], [rows]
  size_t top, group;      // float [rows][units], [rows][groups]
  size_t row_top;         // float [rows]
  size_t z, index;        // float, int32 [rows][k]
  size_t bytes;
};
inline BeamSpace beam_space(const BeamPlan& p, int64_t rows, int k) {
  BeamSpace s;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 15) / 16 * 16;
    return here;
  };
  s.sum = take(8 * (size_t)rows * p.units);
  s.lse = take(8 * (size_t)rows);
  s.top = take(4 * (size_t)rows * p.units);
  s.group = take(4 * (size_t)rows * p.groups);
  s.row_top = take(4 * (size_t)rows);
  s.z = take(4 * (size_t)rows * k);
  s.index = take(4 * (size_t)rows * k);
  s.bytes = at;
  return s;
}

}  // namespace wici
