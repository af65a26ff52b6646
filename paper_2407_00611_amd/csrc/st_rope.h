// Norms and rotations of queries and keys: what the entry points hand to the kernels (st_rope.hip).
#pragma once

#include "st_internal.h"

namespace st {

struct RopeArgs {
  int32_t B, S, Hq, Hkv, D, rot;
  int32_t next;              // 1: the pairs are neighbours, 0: half the rotated values apart
  int32_t norm;
  float eps;
  int32_t n_axes, axis_pairs[ST_ROPE_MAX_AXES];
  int64_t offset, offset2;   // positions without a table: runs of rows, as a shard has them
  int32_t seg;
  View q, k, q_out, k_out;   // backward: the outputs are dx
  View dq, dk;               // backward
  const float *q_weight, *k_weight;
  const double* freq;        // [rot / 2], radians per position
  const int32_t* positions;  // nullable, [n_axes, B, S]
  float* dw_parts;           // backward, nullable: [min(kRopeBlocksMost, B S)][2][D]
};

constexpr int kRopeBlocksMost = 1024;    // workgroups of the backward, each with sums of its own: so many, or one a token
hipError_t launch_rope_fwd(const RopeArgs& g, bool bf16, hipStream_t stream);
hipError_t launch_rope_bwd(const RopeArgs& g, bool bf16, bool d_bf16, float* dwq, float* dwk, bool assign, hipStream_t stream);

}  // namespace st
