// vc_norm.h -- plan and host launchers of the normed rotations.  Internal.
#pragma once
#include "vc_q8.h"

namespace vc {

struct NormPlan {
  RowsDesc qi, ki, qo, ko;  // rows in and out
  RowsDesc qg, kg;          // gradient: the outputs' gradients
  const void *qw, *kw;      // weights [L][d]
  const int32_t *pos;       // [3][B][n]
  const int32_t *count;     // tokens per sequence; null: n
  int32_t B, L, Hq, Hkv, d, n;  // Hq (Hkv) is 0 where there are no queries (keys)
  int32_t fp32, w_fp32;
  float eps;
  int32_t groups;  // gradient: workgroups of each layer
  float *part;     // gradient: [L][groups][2][d] sums of each workgroup
  float *dqw, *dkw;  // gradient: [L][d]
  RopeTable t;       // gradient: of the rotation back
};

hipError_t launch_norm_rope(const NormPlan &p, hipStream_t st);
hipError_t launch_norm_rope_grad(const NormPlan &p, hipStream_t st);

}  // namespace vc
