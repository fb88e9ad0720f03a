// vc_q8_api.cpp -- the C ABI of the 8-bit cache and of the rotary positions
// (include/viscache.h): argument checks, frequencies, workspace layout and how
// an attention call is cut into workgroups.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/viscache.h"
#include "vc_q8.h"

using namespace vc;

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxWg = int64_t(1) << 23;  // 512 threads each: a launch holds fewer than 2^32
constexpr int kCols = 16;                     // columns of the single-token kernel
size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }

vc_status check_shape(const vc_decode_shape *s) {
  if (!s) return VC_ERR_ARG;
  if (s->B < 1 || s->L < 1 || s->Hq < 1 || s->Hkv < 1) return VC_ERR_SHAPE;
  if (s->Hq % s->Hkv != 0) return VC_ERR_SHAPE;
  // Products of the first three factors stay below 2^62, so none overflows.
  if ((int64_t)s->L * s->B > INT32_MAX || (int64_t)s->L * s->B * s->Hq > INT32_MAX) return VC_ERR_SHAPE;
  if (s->Hq / s->Hkv > 16) return VC_ERR_UNSUPPORTED;
  if (s->d != 64 && s->d != 128) return VC_ERR_UNSUPPORTED;
  return VC_OK;
}

vc_status check_cache(const vc_q8cache *c) {
  if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->row_off ||
      !c->cap || !c->len)
    return VC_ERR_ARG;
  if (c->format != VC_Q8_INT8 && c->format != VC_Q8_E4M3) return VC_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k_codes) | reinterpret_cast<uintptr_t>(c->v_codes) |
       reinterpret_cast<uintptr_t>(c->k_tail) | reinterpret_cast<uintptr_t>(c->v_tail)) %
          16 !=
      0)
    return VC_ERR_ARG;
  return VC_OK;
}

// A strided tensor of elements of `es` bytes over dims L, B, n, H.  `by_unit`:
// only the token stride is used.  An output's rows must not fall on each other
// along any one dimension.
bool rows_ok(const vc_rows *r, int es, int64_t L, int64_t B, int64_t n, int64_t H, int64_t d, bool out, bool by_unit) {
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

RowsDesc desc(const vc_rows *r) {
  return RowsDesc{(uint64_t) reinterpret_cast<uintptr_t>(r->data), r->layer, r->seq, r->token, r->head};
}

Q8Cache bind(const vc_q8cache *c) {
  return Q8Cache{static_cast<uint8_t *>(c->k_codes), static_cast<uint8_t *>(c->v_codes), c->k_scale, c->v_scale,
                 static_cast<uint16_t *>(c->k_tail), static_cast<uint16_t *>(c->v_tail), c->row_off, c->cap, c->len,
                 c->order};
}

// How an attention call is cut, and what it needs of the workspace: partial O,
// (max, sum), and the units' pieces of a step.
struct Cut {
  int32_t piece = 0, npmax = 1, qcols = 0, nqt = 0, ns = 1;
  int64_t wgs = 0, slots = 0;  // workgroups; columns of partial results
  size_t ml = 0, np = 0, total = 0;
};

bool attend_cut(const vc_decode_shape *s, int32_t n, int32_t max_rows, Cut &c) {
  const int64_t units = (int64_t)s->L * s->B * s->Hkv;
  const int64_t G = s->Hq / s->Hkv, cols = n * G;
  if (cols > (int64_t(1) << 24)) return false;
  const int64_t nt = std::max<int64_t>(1, ((int64_t)max_rows + kQ8Block - 1) / kQ8Block);
  if (cols <= kCols) {
    // Units are cut into pieces of a multiple of four blocks (one per wave and
    // turn), as many as make about 256 workgroups, one a CU, and not where that
    // were two a unit or three short ones, which save less than the join costs.
    // (us: 4 units of 12544 rows in pieces of 4, 8, 16, 48 blocks 12.4, 13.3, 15.7,
    // 26.1; 32 of 2300 to 5800 rows in 4, 8, 12, 24: 21.1, 19.2, 16.4, 19.7; 112 of
    // 620 to 1490 in 12 and uncut 17.1, 16.2; 160 of 800 to 1900 in 20 and uncut
    // 19.7, 18.5; 896 of 2300 to 5800 in 24, 48 and uncut 199, 198, 188; 8 of 9, 12,
    // 16, 20 blocks in 4 10.3, 11.3, 11.3, 11.4, uncut 9.7, 10.8, 12.1, 13.4; 32 of
    // them in 4 10.7, 11.6, 12.1, 12.7, uncut 9.8, 11.0, 12.2, 14.3.  Far longer units
    // would gain from two even pieces, by what the cut makes of them now and in two:
    // 128 of 4000, 8000, 16000, 32000 rows 31.2 30.7, 50.5 48.2, 108 100, 220 191; 112 of
    // 3000, 8000, 32000 26.0 23.9, 43.3 41.9, 173 161; but 160 of 8000, 32000 62.8 72.9, 232
    // 280 and 200 of them 77.2 87.0, 280 303.)
    const int64_t want = units * nt / 256;
    c.qcols = kCols;
    c.piece = (int32_t)std::min<int64_t>(std::max<int64_t>(4, (want + 3) / 4 * 4), int64_t(1) << 26);
    if (nt <= std::max<int64_t>(2 * (int64_t)c.piece, 12)) c.piece = (int32_t)nt;
    c.npmax = (int32_t)((nt + c.piece - 1) / c.piece);
    c.wgs = units * c.npmax;
    c.slots = c.npmax > 1 ? c.wgs * kCols : 0;
  } else {
    c.qcols = cols > 128 ? 256 : 128;
    const int64_t nqt = (cols + c.qcols - 1) / c.qcols;
    const int64_t tiles = units * nqt;
    if (tiles >= kMaxWg) return false;
    const int64_t resident = c.qcols == 256 ? 256 : 512;
    c.nqt = (int32_t)nqt;
    // Workgroups that the card holds at once share the tiles' rows where that
    // is two a tile or more.  (us, whole tiles and shared ones: 132, 152 and 168 tiles of
    // 12544 rows 334 340, 301 346, 324 341; 136 and 152 of 23040 540 604, 546 617: shares
    // of one tile each are whole tiles with a join.  Sequences of unlike lengths would
    // gain, four of 2250 to 9000 rows in 144 tiles 220 144, but their lengths are not
    // known here.  Whole tiles leave the more workgroups idle the fewer they are, 124 of
    // 256 at 132.)
    c.ns = tiles * 2 <= resident && nt >= 2 * kQ8SplitBlocks ? 2 : 1;
    c.wgs = c.ns > 1 ? std::min(resident, tiles * (nt / kQ8SplitBlocks)) : tiles;
    c.slots = c.ns > 1 ? c.wgs * c.qcols : 0;
  }
  if (c.wgs >= kMaxWg || (c.slots && units * cols >= 2 * kMaxWg)) return false;  // (the join: 256 threads a column)
  c.ml = align_up(sizeof(float) * (size_t)c.slots * (size_t)s->d);
  c.np = c.ml + align_up(sizeof(float2) * (size_t)c.slots);
  const int64_t words = cols <= kCols ? units : c.ns > 1 ? 2 * units * c.nqt : 0;
  c.total = std::max(c.np + align_up(sizeof(int32_t) * (size_t)words), kAlign);
  return true;
}

// The rotation as the kernels take it.
vc_status rope_table(const vc_rope *r, int32_t d, RopeTable &t) {
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

// Workgroups a unit of an append: one where its blocks are few, which then also
// advances the length; else a block each, and the lengths in a launch of their own.
// (us, keys and values of 128 channels in int8, one workgroup and a block each: 8 units of
// 64, 128, 200, 256, 400 rows 2.5 4.3, 5.7 5.6, 8.0 6.2, 9.0 5.5, 13.3 6.0; 112 of 128,
// 200, 256, 400, 640 rows 6.3 7.4, 8.9 9.5, 10.3 9.5, 14.3 12.6, 22.4 14.1; 896 of 128,
// 256, 400, 640 rows 16.3 19.8, 26.6 30.8, 38.0 53.0, 83.1 66.8.  They meet at 128 rows of
// few units and between 400 and 640 of many; 256 lies between.)
int64_t append_groups(int64_t n) {
  return n <= 4 * kQ8Block ? 1 : (n + kQ8Block - 1) / kQ8Block + 1;
}

// The checks and the plan of an attention call (n = 0: the checks that apply).
vc_status attend_plan(const vc_decode_shape *s, const vc_q8cache *c, const vc_rows *q, const vc_rows *out, int32_t n,
                      const int32_t *count, int32_t causal, int32_t out_fp32, float scale, int32_t max_rows,
                      void *workspace, size_t workspace_bytes, Q8Attn &p) {
  vc_status st = check_shape(s);
  if (st != VC_OK) return st;
  if ((st = check_cache(c)) != VC_OK) return st;
  if (n < 0 || max_rows < 0 || (causal != 0 && causal != 1) || (out_fp32 != 0 && out_fp32 != 1)) return VC_ERR_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) return VC_ERR_ARG;
  if (n == 0) return VC_OK;
  if (!rows_ok(q, 2, s->L, s->B, n, s->Hq, s->d, false, false) ||
      !rows_ok(out, out_fp32 ? 4 : 2, s->L, s->B, n, s->Hq, s->d, true, false))
    return VC_ERR_ARG;
  Cut cut;
  if (!attend_cut(s, n, max_rows, cut)) return VC_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < cut.total || reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
    return VC_ERR_WORKSPACE;
  p = Q8Attn{};
  p.c = bind(c);
  p.q = desc(q);
  p.out = desc(out);
  p.count = count;
  p.L = s->L; p.B = s->B; p.Hq = s->Hq; p.Hkv = s->Hkv; p.G = s->Hq / s->Hkv; p.d = s->d;
  p.units = s->L * s->B * s->Hkv;
  p.n = n;
  p.cols = n * p.G;
  p.causal = causal;
  p.fp32 = out_fp32;
  p.max_rows = max_rows;
  p.sc = scale * 1.4426950408889634f;
  p.wgs = (int32_t)cut.wgs;
  p.piece = cut.piece; p.npmax = cut.npmax;
  p.qcols = cut.qcols; p.nqt = cut.nqt; p.ns = cut.ns;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  p.part_o = reinterpret_cast<float *>(ws);
  p.part_ml = reinterpret_cast<float2 *>(ws + cut.ml);
  p.np = reinterpret_cast<int32_t *>(ws + cut.np);
  return VC_OK;
}

}  // namespace

extern "C" {

vc_status viscache_q8_append(const vc_decode_shape *s, const vc_q8cache *c, const vc_rows *k, const vc_rows *v,
                             int32_t n, const int32_t *count, const int64_t *unit_off, void *stream) {
  vc_status st = check_shape(s);
  if (st != VC_OK) return st;
  if ((st = check_cache(c)) != VC_OK) return st;
  if (n < 0) return VC_ERR_ARG;
  if (n == 0) return VC_OK;
  const bool by_unit = unit_off != nullptr;
  if (!rows_ok(k, 2, s->L, s->B, n, s->Hkv, s->d, false, by_unit) ||
      !rows_ok(v, 2, s->L, s->B, n, s->Hkv, s->d, false, by_unit))
    return VC_ERR_ARG;
  Q8Rows p{};
  p.c = bind(c);
  p.k = desc(k);
  p.v = desc(v);
  p.unit_off = unit_off;
  p.count = count;
  p.B = s->B; p.Hkv = s->Hkv; p.d = s->d;
  p.units = s->L * s->B * s->Hkv;
  p.n = n;
  const int64_t nj = append_groups(n);
  if (nj * p.units >= kMaxWg) return VC_ERR_UNSUPPORTED;
  p.nj = (int32_t)nj;
  return launch_q8_append(p, c->format, static_cast<hipStream_t>(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

vc_status viscache_q8_read(const vc_decode_shape *s, const vc_q8cache *c, int32_t max_rows, const vc_rows *k,
                           const vc_rows *v, const int64_t *unit_off, int32_t out_fp32, void *stream) {
  vc_status st = check_shape(s);
  if (st != VC_OK) return st;
  if ((st = check_cache(c)) != VC_OK) return st;
  if (max_rows < 0 || (out_fp32 != 0 && out_fp32 != 1)) return VC_ERR_ARG;
  if (max_rows == 0) return VC_OK;
  const bool by_unit = unit_off != nullptr;
  const int es = out_fp32 ? 4 : 2;
  if (!rows_ok(k, es, s->L, s->B, max_rows, s->Hkv, s->d, true, by_unit) ||
      !rows_ok(v, es, s->L, s->B, max_rows, s->Hkv, s->d, true, by_unit))
    return VC_ERR_ARG;
  Q8Rows p{};
  p.c = bind(c);
  p.k = desc(k);
  p.v = desc(v);
  p.unit_off = unit_off;
  p.B = s->B; p.Hkv = s->Hkv; p.d = s->d;
  p.units = s->L * s->B * s->Hkv;
  p.n = max_rows;
  p.fp32 = out_fp32;
  const int64_t nj = ((int64_t)max_rows + kQ8Block - 1) / kQ8Block;
  if (nj * p.units >= kMaxWg) return VC_ERR_UNSUPPORTED;
  p.nj = (int32_t)nj;
  return launch_q8_read(p, c->format, static_cast<hipStream_t>(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

size_t viscache_q8_attend_workspace_bytes(const vc_decode_shape *s, int32_t n, int32_t max_rows) {
  if (check_shape(s) != VC_OK || n < 0 || max_rows < 0) return 0;
  Cut c;
  return attend_cut(s, n, max_rows, c) ? c.total : 0;
}

vc_status viscache_q8_attend(const vc_decode_shape *s, const vc_q8cache *c, const vc_rows *q, const vc_rows *out,
                             int32_t n, const int32_t *count, int32_t causal, int32_t out_fp32, float scale,
                             int32_t max_rows, void *workspace, size_t workspace_bytes, void *stream) {
  Q8Attn p;
  const vc_status st =
      attend_plan(s, c, q, out, n, count, causal, out_fp32, scale, max_rows, workspace, workspace_bytes, p);
  if (st != VC_OK || n == 0) return st;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const hipError_t e = p.cols <= kCols ? launch_q8_decode(p, c->format, hs) : launch_q8_prompt(p, c->format, hs);
  return e == hipSuccess ? VC_OK : VC_ERR_HIP;
}

vc_status viscache_q8_step(const vc_decode_shape *s, const vc_q8cache *c, const vc_rope *rope, const int32_t *pos,
                           const vc_rows *q, const vc_rows *k, const vc_rows *v, const vc_rows *out, int32_t out_fp32,
                           float scale, int32_t max_rows, void *workspace, size_t workspace_bytes, void *stream) {
  Q8Attn p;
  vc_status st = attend_plan(s, c, q, out, 1, nullptr, 1, out_fp32, scale, max_rows, workspace, workspace_bytes, p);
  if (st != VC_OK) return st;
  if (!rows_ok(k, 2, s->L, s->B, 1, s->Hkv, s->d, false, false) ||
      !rows_ok(v, 2, s->L, s->B, 1, s->Hkv, s->d, false, false))
    return VC_ERR_ARG;
  if (rope) {
    if (rope->fp32 || !pos) return VC_ERR_ARG;
    if ((st = rope_table(rope, s->d, p.rope)) != VC_OK) return st;
  }
  p.step = 1;
  p.k = desc(k);
  p.v = desc(v);
  p.pos = pos;
  return launch_q8_decode(p, c->format, static_cast<hipStream_t>(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

vc_status viscache_rope(const vc_decode_shape *s, const vc_rope *r, int32_t n, const int32_t *pos,
                        const int32_t *count, const vc_rows *q_in, const vc_rows *q_out, const vc_rows *k_in,
                        const vc_rows *k_out, void *stream) {
  vc_status st = check_shape(s);
  if (st != VC_OK) return st;
  if (!r || n < 0) return VC_ERR_ARG;
  RopePlan p{};
  if ((st = rope_table(r, s->d, p.t)) != VC_OK) return st;
  if (!q_in != !q_out || !k_in != !k_out || (!q_in && !k_in)) return VC_ERR_ARG;
  if (n == 0) return VC_OK;
  if (!pos) return VC_ERR_ARG;
  const int es = r->fp32 ? 4 : 2;
  if (q_in && (!rows_ok(q_in, es, s->L, s->B, n, s->Hq, s->d, false, false) ||
               !rows_ok(q_out, es, s->L, s->B, n, s->Hq, s->d, true, false)))
    return VC_ERR_ARG;
  if (k_in && (!rows_ok(k_in, es, s->L, s->B, n, s->Hkv, s->d, false, false) ||
               !rows_ok(k_out, es, s->L, s->B, n, s->Hkv, s->d, true, false)))
    return VC_ERR_ARG;
  if ((int64_t)s->L * s->B * n >= (int64_t(1) << 24)) return VC_ERR_UNSUPPORTED;
  if (q_in) {
    p.qi = desc(q_in);
    p.qo = desc(q_out);
    p.Hq = s->Hq;
  }
  if (k_in) {
    p.ki = desc(k_in);
    p.ko = desc(k_out);
    p.Hkv = s->Hkv;
  }
  p.pos = pos;
  p.count = count;
  p.B = s->B; p.L = s->L; p.d = s->d; p.n = n;
  p.fp32 = r->fp32;
  return launch_rope(p, static_cast<hipStream_t>(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

}  // extern "C"
