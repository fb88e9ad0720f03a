// vc_norm_api.cpp -- the C ABI of the normed rotations (include/viscache.h): argument
// checks and the gradient's workspace.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "../../include/viscache.h"
#include "vc_host.h"
#include "vc_norm.h"

using namespace vc;

namespace {

// Workgroups of a layer's gradient: enough for the card to hold four on each CU over
// all layers, and none without a token for its four waves.
int32_t grad_groups(const vc_decode_shape *s, int32_t n) {
  const int64_t toks = (int64_t)s->B * n;
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>((toks + 3) / 4, 1024 / s->L));
}

bool tokens_ok(const vc_decode_shape *s, int32_t n) { return (int64_t)s->L * s->B * n < (int64_t(1) << 24); }
// The gradient's second launch: 2 L d / 16 workgroups of 1024 threads.
bool grad_ok(const vc_decode_shape *s, int32_t n) { return tokens_ok(s, n) && s->L < (1 << 17); }

// What both directions check, and their plan.
vc_status norm_plan(const vc_decode_shape *s, const vc_rope *r, const vc_norm *nm, int32_t n, NormPlan &p) {
  const vc_status st = check_shape(s);
  if (st != VC_OK) return st;
  if (!r || !nm || n < 0) return VC_ERR_ARG;
  p = NormPlan{};
  if (rope_table(r, s->d, p.t) != VC_OK) return VC_ERR_ARG;
  if (!(nm->eps >= std::numeric_limits<float>::min()) || !std::isfinite(nm->eps)) return VC_ERR_ARG;
  if (nm->weight_fp32 != 0 && nm->weight_fp32 != 1) return VC_ERR_ARG;
  p.B = s->B; p.L = s->L; p.d = s->d; p.n = n;
  p.fp32 = r->fp32;
  p.w_fp32 = nm->weight_fp32;
  p.eps = nm->eps;
  p.qw = nm->q_weight;
  p.kw = nm->k_weight;
  return VC_OK;
}

bool weight_ok(const void *w) { return w && reinterpret_cast<uintptr_t>(w) % 16 == 0; }

}  // namespace

extern "C" {

vc_status viscache_norm_rope(const vc_decode_shape *s, const vc_rope *r, const vc_norm *nm, int32_t n,
                             const int32_t *pos, const int32_t *count, const vc_rows *q_in, const vc_rows *q_out,
                             const vc_rows *k_in, const vc_rows *k_out, void *stream) {
  NormPlan p;
  const vc_status st = norm_plan(s, r, nm, n, p);
  if (st != VC_OK) return st;
  if (!q_in != !q_out || !k_in != !k_out || (!q_in && !k_in)) return VC_ERR_ARG;
  if (n == 0) return VC_OK;
  if (!pos || (q_in && !weight_ok(nm->q_weight)) || (k_in && !weight_ok(nm->k_weight))) return VC_ERR_ARG;
  const int es = r->fp32 ? 4 : 2;
  if (q_in && (!rows_ok(q_in, es, s->L, s->B, n, s->Hq, s->d, false, false) ||
               !rows_ok(q_out, es, s->L, s->B, n, s->Hq, s->d, true, false)))
    return VC_ERR_ARG;
  if (k_in && (!rows_ok(k_in, es, s->L, s->B, n, s->Hkv, s->d, false, false) ||
               !rows_ok(k_out, es, s->L, s->B, n, s->Hkv, s->d, true, false)))
    return VC_ERR_ARG;
  if (!tokens_ok(s, n)) return VC_ERR_UNSUPPORTED;
  if (q_in) {
    p.qi = desc(q_in);
    p.qo = desc(q_out);
    p.Hq = s->Hq;
  } else {
    p.qw = nullptr;
  }
  if (k_in) {
    p.ki = desc(k_in);
    p.ko = desc(k_out);
    p.Hkv = s->Hkv;
  } else {
    p.kw = nullptr;
  }
  p.pos = pos;
  p.count = count;
  return launch_norm_rope(p, static_cast<hipStream_t>(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

size_t viscache_norm_rope_grad_workspace_bytes(const vc_decode_shape *s, int32_t n) {
  if (check_shape(s) != VC_OK || n < 0 || !grad_ok(s, n)) return 0;
  return align_up(sizeof(float) * 2 * (size_t)s->d * (size_t)s->L * (size_t)grad_groups(s, n));
}

vc_status viscache_norm_rope_grad(const vc_decode_shape *s, const vc_rope *r, const vc_norm *nm, int32_t n,
                                  const int32_t *pos, const int32_t *count, const vc_rows *q, const vc_rows *q_dout,
                                  const vc_rows *q_din, float *q_dweight, const vc_rows *k, const vc_rows *k_dout,
                                  const vc_rows *k_din, float *k_dweight, void *workspace, size_t workspace_bytes,
                                  void *stream) {
  NormPlan p;
  const vc_status st = norm_plan(s, r, nm, n, p);
  if (st != VC_OK) return st;
  if (!q != !q_dout || !q != !q_din || !q != !q_dweight || !k != !k_dout || !k != !k_din || !k != !k_dweight ||
      (!q && !k))
    return VC_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(q_dweight) | reinterpret_cast<uintptr_t>(k_dweight)) % 4 != 0) return VC_ERR_ARG;
  if ((q && !weight_ok(nm->q_weight)) || (k && !weight_ok(nm->k_weight))) return VC_ERR_ARG;
  if (n > 0) {  // (without tokens the weights' gradients are zeros)
    if (!pos) return VC_ERR_ARG;
    const int es = r->fp32 ? 4 : 2;
    auto side_ok = [&](const vc_rows *x, const vc_rows *g, const vc_rows *o, int32_t H) {
      return rows_ok(x, es, s->L, s->B, n, H, s->d, false, false) && rows_ok(g, es, s->L, s->B, n, H, s->d, false, false) &&
             rows_ok(o, es, s->L, s->B, n, H, s->d, true, false);
    };
    if ((q && !side_ok(q, q_dout, q_din, s->Hq)) || (k && !side_ok(k, k_dout, k_din, s->Hkv))) return VC_ERR_ARG;
  }
  if (!grad_ok(s, n)) return VC_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < viscache_norm_rope_grad_workspace_bytes(s, n) ||
      reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
    return VC_ERR_WORKSPACE;
  if (q) {
    if (n > 0) p.qi = desc(q), p.qg = desc(q_dout), p.qo = desc(q_din);
    p.Hq = s->Hq;
  } else {
    p.qw = nullptr;
  }
  if (k) {
    if (n > 0) p.ki = desc(k), p.kg = desc(k_dout), p.ko = desc(k_din);
    p.Hkv = s->Hkv;
  } else {
    p.kw = nullptr;
  }
  p.t.sgn = -p.t.sgn;  // the outputs' gradients turn back
  p.pos = pos;
  p.count = count;
  p.groups = grad_groups(s, n);
  p.part = static_cast<float *>(workspace);
  p.dqw = q_dweight;
  p.dkw = k_dweight;
  return launch_norm_rope_grad(p, static_cast<hipStream_t>(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

}  // extern "C"
