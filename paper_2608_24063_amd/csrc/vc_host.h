// vc_host.h -- argument checks that the entry points over strided rows share: shapes,
// row descriptors, rotations.  Host only, internal.
#pragma once
#include <cmath>

#include "../../include/viscache.h"
#include "vc_q8.h"

namespace vc {

constexpr size_t kAlign = 256;                // workspaces and their parts
constexpr int64_t kMaxWg = int64_t(1) << 23;  // 512 threads each: a launch holds fewer than 2^32
inline size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }

inline vc_status check_shape(const vc_decode_shape *s) {
  if (!s) return VC_ERR_ARG;
  if (s->B < 1 || s->L < 1 || s->Hq < 1 || s->Hkv < 1) return VC_ERR_SHAPE;
  if (s->Hq % s->Hkv != 0) return VC_ERR_SHAPE;
  // Products of the first three factors stay below 2^62, so none overflows.
  if ((int64_t)s->L * s->B > INT32_MAX || (int64_t)s->L * s->B * s->Hq > INT32_MAX) return VC_ERR_SHAPE;
  if (s->Hq / s->Hkv > 16) return VC_ERR_UNSUPPORTED;
  if (s->d != 64 && s->d != 128) return VC_ERR_UNSUPPORTED;
  return VC_OK;
}

// A strided tensor of elements of `es` bytes over dims L, B, n, H.  `by_unit`:
// only the token stride is used.  An output's rows must not fall on each other
// along any one dimension.
inline bool rows_ok(const vc_rows *r, int es, int64_t L, int64_t B, int64_t n, int64_t H, int64_t d, bool out, bool by_unit) {
  if (!r || !r->data || reinterpret_cast<uintptr_t>(r->data) % 16 != 0) return false;
  const int64_t st[4] = {by_unit ? 0 : r->layer, by_unit ? 0 : r->seq, r->token, by_unit ? 0 : r->head};
  const int64_t n_[4] = {by_unit ? 1 : L, by_unit ? 1 : B, n, by_unit ? 1 : H};
  __int128 last = 0;
  for (int i = 0; i < 4; ++i) {
    if (n_[i] == 1) continue;  // never multiplied by more than 0
    if (st[i] < 0 || st[i] % (16 / es) != 0) return false;
    if (out && st[i] < d) return false;
    last += (__int128)st[i] * (n_[i] - 1);
  }
  return last < ((__int128)1 << 60);
}

inline RowsDesc desc(const vc_rows *r) {
  return RowsDesc{(uint64_t) reinterpret_cast<uintptr_t>(r->data), r->layer, r->seq, r->token, r->head};
}

// The rotation as the kernels take it.
inline vc_status rope_table(const vc_rope *r, int32_t d, RopeTable &t) {
  if (r->rot < 16 || r->rot % 16 != 0 || r->rot > d) return VC_ERR_ARG;
  for (int i = 0; i < 3; ++i)
    if (r->sections[i] < 0 || r->sections[i] > r->rot / 2) return VC_ERR_ARG;
  if (r->sections[0] + r->sections[1] + r->sections[2] != r->rot / 2) return VC_ERR_ARG;
  if ((r->layout != VC_ROPE_SECTIONED && r->layout != VC_ROPE_INTERLEAVED) ||
      (r->pairing != VC_ROPE_HALVES && r->pairing != VC_ROPE_ADJACENT) || (r->fp32 != 0 && r->fp32 != 1) ||
      (r->inverse != 0 && r->inverse != 1) || !std::isfinite(r->scale))
    return VC_ERR_ARG;
  if (!r->inv_freq && !(r->theta > 0.0 && std::isfinite(r->theta))) return VC_ERR_ARG;
  t = RopeTable{};
  for (int i = 0; i < r->rot / 2; ++i) {
    const double f = r->inv_freq ? r->inv_freq[i] : std::pow(r->theta, -2.0 * i / r->rot);
    if (!std::isfinite(f)) return VC_ERR_ARG;
    t.turns[i] = f / 6.283185307179586476925286766559;
    int axis;
    if (r->layout == VC_ROPE_SECTIONED)
      axis = (i >= r->sections[0]) + (i >= r->sections[0] + r->sections[1]);
    else
      axis = i % 3 == 1 && i < 3 * r->sections[1] ? 1 : i % 3 == 2 && i < 3 * r->sections[2] ? 2 : 0;
    t.axis1 |= (uint64_t)(axis == 1) << i;
    t.axis2 |= (uint64_t)(axis == 2) << i;
  }
  t.rot = r->rot;
  t.adjacent = r->pairing == VC_ROPE_ADJACENT;
  t.scale = r->scale;
  t.sgn = r->inverse ? -1.f : 1.f;
  return VC_OK;
}

}  // namespace vc
