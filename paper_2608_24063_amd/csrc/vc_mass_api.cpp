// vc_mass_api.cpp -- the C ABI of the cache that keeps its rows' attention weight
// (include/viscache.h): argument checks, workspace layout and how a call is cut into
// workgroups.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/viscache.h"
#include "vc_host.h"
#include "vc_mass.h"

using namespace vc;

namespace {

constexpr int kTokenCols = 16;  // columns of the single-token kernel

vc_status check_cache(const vc_mass_cache *c) {
  if (!c || !c->k_pool || !c->v_pool || !c->mass || !c->row_off || !c->cap || !c->len) return VC_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k_pool) | reinterpret_cast<uintptr_t>(c->v_pool)) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(c->mass) % 4 != 0)
    return VC_ERR_ARG;
  return VC_OK;
}

MassPool bind(const vc_mass_cache *c) {
  return MassPool{static_cast<uint16_t *>(c->k_pool), static_cast<uint16_t *>(c->v_pool), c->mass, c->row_off, c->cap,
                  c->len};
}

// How an attention call is cut, and the parts of its workspace.
struct Cut {
  int32_t waves = 0, piece = 0, npmax = 1, here = 0, ldr = 0, finish = 0, finish_wgs = 0, qcols = 0, nqt = 0, ns = 1, ktiles = 1, csplit = 1;
  int64_t wgs = 0, slots = 0;  // workgroups; columns of partial results
  size_t ml = 0, stat = 0, state = 0, np = 0, logits = 0, mass = 0, total = 0;
};

bool attend_cut(const vc_decode_shape *s, int32_t n, int32_t max_rows, Cut &c) {
  const int64_t units = (int64_t)s->L * s->B * s->Hkv;
  const int64_t G = s->Hq / s->Hkv, cols = n * G;
  max_rows = std::min(max_rows, kMassMaxRows);  // no unit holds more
  if (cols > (int64_t(1) << 24)) return false;
  if (cols <= kTokenCols) {
    const int64_t nt = std::max<int64_t>(1, ((int64_t)max_rows + kMassTile - 1) / kMassTile);
    // Units are cut into pieces of a multiple of four tiles (one per wave and turn), as
    // many as make about 256 workgroups, one a CU, but no more than 24 a unit, which the
    // second launch has to join; not where the rows that a piece saves cost less than
    // that launch, nor where the units fill the chip by themselves.  A CU reads 51 GB/s, however
    // many its waves.  (us, 7 columns and 128 channels, in pieces of 4, 8, 16, 32 tiles and
    // whole: 4 units of 1000 rows 11.3 12.7 14.7 15.9 15.9, of 4000 13.2 12.1 13.5 17.8 45,
    // of 12000 21.7 15.7 15.6 19.1 124; 32 of 1000 11.4 12.7 14.8 16.0 16.2, of 4000 25.7
    // 20.8 19.4 20.3 46.5; 64 of 1000 15.4 14.2 16.3 16.8 17.2, of 4000 39.8 31.3 28.8 28.6
    // 47.0; 112 of 1000 24.3 21.1 19.7 17.8 18.1, of 2000 37.1 30.8 27.6 26.9 28.5, of 12000
    // 217 188 179 175 199.  A unit of 400 rows takes 10.7 whole.)  Units so long that the
    // pieces of 1024 workgroups are, too, even out better in as many (256 and 1024
    // workgroups: 112 units of 12000 rows 181 173, of 23000 341 320, of 4000 to 12000 132 127,
    // of 4000 47 47; 32 of 23000 97 100, 64 of 4000 29 31).
    const auto fours = [](int64_t x) { return (x + 3) / 4 * 4; };
    c.qcols = kTokenCols;
    const int64_t want = units * nt > 32768 ? 1024 : 256;
    c.piece = (int32_t)std::max<int64_t>({4, fours((units * nt + want - 1) / want), fours((nt + 23) / 24)});
    if (nt <= 12 || units > 128 || (units > 96 && nt <= 48)) c.piece = (int32_t)nt;
    c.npmax = (int32_t)((nt + c.piece - 1) / c.piece);
    c.wgs = units * c.npmax;
    c.slots = c.npmax > 1 ? c.wgs * kTokenCols : 0;
    // Eight waves where four would leave more than a third of a whole unit's logits to the
    // workspace.  (us, four and eight waves: 896 units of 200 rows and 7 columns 23.2 36.4,
    // of 1000 74 87, of 1500 110 120; 640 of 1000 rows and 8 columns 46 55, of 3000 175 157;
    // 320 of 3000 104 87; 2000 of 2500 rows, 4 columns and 64 channels 208 215.)
    const int64_t pitch = cols | 1;
    c.waves = c.npmax == 1 && nt * kMassTile * pitch > kMassHeld4 * 3 / 2 ? 8 : 4;
    const int64_t room = (c.waves == 8 ? kMassHeld8 : kMassHeld4) / pitch / kMassTile * kMassTile;
    c.here = (int32_t)(c.npmax > 1 ? 0 : std::min(room, nt * kMassTile));
    c.ldr = (int32_t)(nt * kMassTile - c.here);
    // The second launch's workgroups (of 1024 threads).  Four rows a thread where one would take
    // more than the 512 workgroups that the card holds.  (us of both launches, one and four rows:
    // 112 units of 23000 319 309, of 12000 172.5 168.5, of 4000 47.5 48.6; 64 of 12000 98.4
    // 96.4, of 4000 29.0 32.4; 4 of 12000 15.6 17.5.)
    if (c.npmax > 1) {
      const int64_t chunks = ((int64_t)max_rows + kMassChunk - 1) / kMassChunk;
      c.finish = units * chunks > 512 ? 4 : 1;
      const int64_t wgs = units * ((chunks + c.finish - 1) / c.finish);
      if (wgs >= kMaxWg / 2) return false;
      c.finish_wgs = (int32_t)wgs;
    }
  } else {
    const int64_t nt = std::max<int64_t>(1, ((int64_t)max_rows + kQ8Block - 1) / kQ8Block);
    // Two workgroups of 128 columns hide each other's start, which counts where rows are few,
    // and make more parts where all work is little.  (us of a call, 256 and 128 columns: 640
    // units, 300 rows and 2400 columns 668 626, 595 and 2840 1075 1032, 600 and 4800 1424
    // 1435; 112 units, 500 and 2100 145.4 140.6, 900 and 2100 219 222, 1065 and 455 81.4 86.5,
    // 3300 and 2100 657 701; 4 units, 600 and 4200 50.8 46.7, 1040 and 280 37.3 32.7; 8 of
    // 1100 and 800 47.9 43.0; 20 of 1564 and 512 52.5 53.8; 12 of 4065 and 455 57.8 58.3.)
    const int64_t wide = units * ((cols + 255) / 256);
    const bool few = nt <= 8 || (wide <= 768 && wide * nt <= 768);
    c.qcols = cols > 128 && !few ? 256 : 128;
    const int64_t nqt = (cols + c.qcols - 1) / c.qcols, tiles = units * nqt;
    if (tiles >= kMaxWg) return false;
    const int64_t resident = c.qcols == 256 ? 256 : 512;
    c.nqt = (int32_t)nqt;
    // Workgroups that the card holds at once share the tiles' rows where that is two
    // a tile or more (attention over the 8-bit cache was measured on both sides of it).
    c.ns = tiles * 2 <= resident && nt >= 2 * kQ8SplitBlocks ? 2 : 1;
    c.wgs = c.ns > 1 ? std::min(resident, tiles * (nt / kQ8SplitBlocks)) : tiles;
    c.slots = c.ns > 1 ? c.wgs * c.qcols : 0;
    // The other launches' workgroups: the append's, the join's, the masses'.
    c.ktiles = (int32_t)std::max<int64_t>(1, ((int64_t)max_rows + kMassKeys - 1) / kMassKeys);
    const int64_t key_tiles = units * c.ktiles;
    if (units * (((int64_t)n * s->d + 2047) / 2048) >= kMaxWg || (c.slots && units * cols >= 2 * kMaxWg) ||
        key_tiles >= kMaxWg)
      return false;
    // A row tile's columns are split over workgroups (the card holds 512 of them) until
    // there are 2048, eight blocks of columns at least together: tiles of later rows are
    // seen by fewer columns, and many small workgroups even that out.  (us of the masses,
    // columns in 1, 2 and 5 parts: 8 units of 25088 rows and 16384 columns 883 850 874; 12
    // units of 9000 to 12900 rows and 455 columns, which stay whole, 35 38 50.)  Down to a
    // block each where tiles are so few that this makes no more than 256, one a CU.  (us of a
    // call, whole and split: 455 columns, 4 units of 3000 rows 50.3 43.6, of 12000 58.6 60.1
    // in two parts; 280 columns, 4 units of 1000 40.8 36.8; 1400 columns, 4 units of 3000
    // 63.1 54.9; 800 columns and 64 channels, a unit of 2000 39.8 29.6.)
    const int64_t blocks = (cols + 63) / 64;
    c.csplit = (int32_t)std::max<int64_t>({1, std::min<int64_t>(blocks / 8, (2048 + key_tiles - 1) / key_tiles),
                                           std::min<int64_t>(blocks, 256 / key_tiles)});
    if (key_tiles * c.csplit >= kMaxWg) c.csplit = 1;
  }
  if (c.wgs >= kMaxWg) return false;
  const bool token = cols <= kTokenCols;
  c.ml = align_up(sizeof(float) * (size_t)c.slots * (size_t)s->d);
  c.stat = c.ml + align_up(sizeof(float2) * (size_t)c.slots);
  c.state = c.stat + (token ? 0 : align_up(sizeof(float2) * (size_t)(units * cols)));
  c.np = c.state + align_up(sizeof(int4) * (size_t)units);
  c.logits = c.np + (token || c.ns == 1 ? 0 : align_up(sizeof(int32_t) * 2 * (size_t)(units * c.nqt)));
  c.mass = c.logits + (token ? align_up(sizeof(float) * (size_t)(units * cols) * (size_t)c.ldr) : 0);
  c.total = c.mass;
  if (c.csplit > 1)
    c.total += align_up(sizeof(float) * (size_t)units * (size_t)c.ktiles * (size_t)c.csplit * kMassKeys);
  return true;
}

// The parts of an eviction's workspace.
struct EvictCut {
  int32_t chunks = 0, ldl = 0;
  size_t count = 0, flags = 0, ticket = 0, total = 0;
};

bool evict_cut(const vc_decode_shape *s, int32_t max_rows, EvictCut &c) {
  max_rows = std::min(max_rows, kMassMaxRows);
  const int64_t units = (int64_t)s->L * s->B * s->Hkv, rows = kEvictBytes / (2 * s->d);
  c.chunks = (int32_t)((max_rows + rows - 1) / rows);
  if (units * c.chunks >= kMaxWg || units >= kMaxWg / 2) return false;  // (1024 threads a unit)
  c.ldl = (int32_t)(c.chunks * rows);
  c.count = align_up(sizeof(int32_t) * (size_t)units * (size_t)c.ldl);
  c.flags = c.count + align_up(sizeof(int32_t) * (size_t)units);
  c.ticket = c.flags + align_up(sizeof(uint32_t) * (size_t)units * (size_t)c.chunks);
  c.total = c.ticket + align_up(sizeof(uint32_t) * (size_t)units);
  return true;
}

}  // namespace

extern "C" {

size_t viscache_mass_attend_workspace_bytes(const vc_decode_shape *s, int32_t n, int32_t max_rows) {
  if (check_shape(s) != VC_OK || n < 0 || max_rows < 0) return 0;
  Cut c;
  return attend_cut(s, std::max(n, 1), max_rows, c) ? c.total : 0;
}

vc_status viscache_mass_attend(const vc_decode_shape *s, const vc_mass_cache *c, const vc_rows *k, const vc_rows *v,
                               const vc_rows *q, const vc_rows *out, int32_t n, const int32_t *count, int32_t out_fp32,
                               float scale, float decay, int32_t max_rows, void *workspace, size_t workspace_bytes,
                               void *stream) {
  vc_status st = check_shape(s);
  if (st != VC_OK) return st;
  if ((st = check_cache(c)) != VC_OK) return st;
  if (n < 0 || max_rows < 0 || (out_fp32 != 0 && out_fp32 != 1) || !k != !v) return VC_ERR_ARG;
  const float sc = scale * 1.4426950408889634f;  // logits in powers of two
  if (!(scale > 0.f) || !std::isfinite(sc) || !(decay >= 0.f) || !std::isfinite(decay)) return VC_ERR_ARG;
  if (n == 0) return VC_OK;
  if (!rows_ok(q, 2, s->L, s->B, n, s->Hq, s->d, false, false) ||
      !rows_ok(out, out_fp32 ? 4 : 2, s->L, s->B, n, s->Hq, s->d, true, false))
    return VC_ERR_ARG;
  if (k && (!rows_ok(k, 2, s->L, s->B, n, s->Hkv, s->d, false, false) ||
            !rows_ok(v, 2, s->L, s->B, n, s->Hkv, s->d, false, false)))
    return VC_ERR_ARG;
  Cut cut;
  if (!attend_cut(s, n, max_rows, cut)) return VC_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < cut.total || reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
    return VC_ERR_WORKSPACE;
  MassAttn p{};
  p.c = bind(c);
  p.q = desc(q);
  p.out = desc(out);
  if (k) {
    p.k = desc(k);
    p.v = desc(v);
    if (n == 1) p.k.token = p.v.token = 0;  // (not checked)
  }
  p.count = count;
  p.L = s->L; p.B = s->B; p.Hq = s->Hq; p.Hkv = s->Hkv; p.G = s->Hq / s->Hkv; p.d = s->d;
  p.units = s->L * s->B * s->Hkv;
  p.wgs = (int32_t)cut.wgs;
  p.n = n;
  p.cols = n * p.G;
  p.append = k != nullptr;
  p.fp32 = out_fp32;
  p.causal = 1;
  p.max_rows = std::min(max_rows, kMassMaxRows);
  p.sc = sc;
  p.decay = decay;
  p.order = c->order;
  p.waves = cut.waves; p.piece = cut.piece; p.npmax = cut.npmax; p.here = cut.here; p.ldr = cut.ldr;
  p.finish = cut.finish; p.finish_wgs = cut.finish_wgs;
  p.qcols = cut.qcols; p.nqt = cut.nqt; p.ns = cut.ns;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  p.part_o = reinterpret_cast<float *>(ws);
  p.part_ml = reinterpret_cast<float2 *>(ws + cut.ml);
  p.stat = reinterpret_cast<float2 *>(ws + cut.stat);
  p.state = reinterpret_cast<int4 *>(ws + cut.state);
  p.np = reinterpret_cast<int32_t *>(ws + cut.np);
  p.logits = reinterpret_cast<float *>(ws + cut.logits);
  p.ktiles = cut.ktiles; p.csplit = cut.csplit;
  p.part_mass = reinterpret_cast<float *>(ws + cut.mass);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const hipError_t e = p.cols <= kTokenCols ? launch_mass_token(p, hs) : launch_mass_prompt(p, hs);
  return e == hipSuccess ? VC_OK : VC_ERR_HIP;
}

size_t viscache_mass_evict_workspace_bytes(const vc_decode_shape *s, int32_t max_rows) {
  if (check_shape(s) != VC_OK || max_rows < 0) return 0;
  EvictCut c;
  return evict_cut(s, max_rows, c) ? c.total : 0;
}

vc_status viscache_mass_evict(const vc_decode_shape *s, const vc_mass_cache *c, const vc_mass_cache *to,
                              const int32_t *keep, int32_t sinks, int32_t recent, int32_t max_rows, int32_t *index,
                              int32_t index_rows, void *workspace, size_t workspace_bytes, void *stream) {
  vc_status st = check_shape(s);
  if (st != VC_OK) return st;
  if ((st = check_cache(c)) != VC_OK) return st;
  if (to) {
    if ((st = check_cache(to)) != VC_OK) return st;
    if (to->k_pool == c->k_pool || to->v_pool == c->v_pool || to->mass == c->mass || to->len == c->len)
      return VC_ERR_ARG;
  }
  if (!keep || sinks < 0 || recent < 0 || max_rows < 0 || index_rows < 0 || (index_rows > 0 && !index))
    return VC_ERR_ARG;
  EvictCut cut;
  if (!evict_cut(s, max_rows, cut)) return VC_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < cut.total || reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
    return VC_ERR_WORKSPACE;
  EvictPlan p{};
  p.c = bind(c);
  if (to) p.to = bind(to);
  p.keep = keep;
  p.units = s->L * s->B * s->Hkv;
  p.d = s->d;
  p.inplace = to == nullptr;
  p.sinks = sinks;
  p.recent = recent;
  p.max_rows = std::min(max_rows, kMassMaxRows);
  p.chunks = cut.chunks;
  p.ldl = cut.ldl;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  p.list = reinterpret_cast<int32_t *>(ws);
  p.count = reinterpret_cast<int32_t *>(ws + cut.count);
  p.flags = reinterpret_cast<uint32_t *>(ws + cut.flags);
  p.ticket = reinterpret_cast<uint32_t *>(ws + cut.ticket);
  p.index = index_rows > 0 ? index : nullptr;
  p.index_rows = index_rows;
  return launch_mass_evict(p, static_cast<hipStream_t>(stream)) == hipSuccess ? VC_OK : VC_ERR_HIP;
}

}  // extern "C"
