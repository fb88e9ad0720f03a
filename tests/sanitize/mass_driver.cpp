// mass_driver.cpp -- the host side of the normed rotations and of the cache with masses
// (argument checks, cuts, workspace layout) under the sanitizers, without a GPU: the
// launchers are stand-ins that hold every plan against what its kernels take for granted,
// then report a failed launch.  Any call must end in a status, whatever its arguments.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <limits>

#include "../../include/viscache.h"
#include "../../paper_2608_24063_amd/csrc/vc_mass.h"
#include "../../paper_2608_24063_amd/csrc/vc_norm.h"

static const char *g_case = "";
static long g_plans = 0, g_calls = 0;
#define CHECK(x)                                                  \
  do {                                                            \
    if (!(x)) {                                                   \
      std::printf("%s: %s (line %d)\n", g_case, #x, __LINE__);    \
      std::exit(1);                                               \
    }                                                             \
  } while (0)

static uint8_t g_ws[256] __attribute__((aligned(256)));  // stands for any workspace: only its address is used
static size_t g_bytes;

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// A launch holds fewer than 2^32 threads.
static void launch(int64_t wgs, int64_t threads) { CHECK(wgs >= 1 && wgs < ((int64_t)1 << 31) && wgs * threads < ((int64_t)1 << 32)); }
// [at, at + bytes) is inside the workspace, aligned, and begins at or behind `from`.
static const uint8_t *part(const void *at_, int64_t bytes, const uint8_t *from) {
  const uint8_t *at = static_cast<const uint8_t *>(at_);
  CHECK(at >= from && (at - g_ws) % 256 == 0 && bytes >= 0 && (uint64_t)(at - g_ws) + (uint64_t)bytes <= g_bytes);
  return at + bytes;
}

namespace vc {

static void attention(const MassAttn &p) {
  ++g_plans;
  const int64_t units = (int64_t)p.L * p.B * p.Hkv;
  CHECK(units == p.units && p.G >= 1 && p.G <= 16 && p.G * p.Hkv == p.Hq && p.cols == (int64_t)p.n * p.G);
  CHECK(p.max_rows >= 0 && p.max_rows <= kMassMaxRows && std::isfinite(p.sc) && p.decay >= 0.f && p.causal == 1);
}

hipError_t launch_mass_token(const MassAttn &p, hipStream_t) {
  attention(p);
  CHECK(p.cols <= 16 && (p.waves == 4 || p.waves == 8));
  const int64_t tiles = ceil_div(p.max_rows, kMassTile);
  CHECK(p.piece >= 1 && p.npmax >= 1 && (int64_t)p.piece * p.npmax >= tiles && p.wgs == (int64_t)p.units * p.npmax);
  launch(p.wgs, 64 * p.waves);
  // Rows' logits: in LDS whole tiles that fit there, behind them the workspace, 16 bytes aligned.
  CHECK(p.here % kMassTile == 0 && p.ldr % kMassTile == 0 && (int64_t)p.here + p.ldr >= p.max_rows);
  CHECK((int64_t)p.here * (p.cols | 1) <= (p.waves == 8 ? kMassHeld8 : kMassHeld4));
  const uint8_t *at = g_ws;
  if (p.npmax > 1) {
    CHECK(p.here == 0 && p.waves == 4);
    launch(p.units * ceil_div(p.max_rows, kMassChunk), kMassChunk);
    at = part(p.part_o, (int64_t)p.wgs * 16 * p.d * 4, at);
    at = part(p.part_ml, (int64_t)p.wgs * 16 * 8, at);
  }
  at = part(p.state, (int64_t)p.units * 16, at);
  part(p.logits, (int64_t)p.units * p.cols * p.ldr * 4, at);
  return hipErrorInvalidValue;
}

hipError_t launch_mass_prompt(const MassAttn &p, hipStream_t) {
  attention(p);
  CHECK(p.cols > 16 && (p.qcols == 128 || p.qcols == 256));
  CHECK((int64_t)p.nqt * p.qcols >= p.cols && (int64_t)(p.nqt - 1) * p.qcols < p.cols);
  const int64_t tiles = (int64_t)p.units * p.nqt;
  if (p.ns == 1) {
    CHECK(p.wgs == tiles);
  } else {
    CHECK(tiles <= kQ8SplitTiles && p.wgs >= 2 * tiles);  // a wave's registers hold the tiles
    launch(ceil_div((int64_t)p.units * p.cols, 1024 / p.d), 256);
  }
  launch(p.wgs, p.qcols * 2);
  if (p.append) launch(p.units * ceil_div(p.n, 2048 / p.d), 256);
  CHECK(p.csplit >= 1 && p.ktiles >= 1 && (int64_t)p.ktiles * kMassKeys >= p.max_rows);
  launch((int64_t)p.units * p.ktiles * p.csplit, kMassKeys);
  const uint8_t *at = g_ws;
  if (p.ns > 1) {
    at = part(p.part_o, (int64_t)p.wgs * p.qcols * p.d * 4, at);
    at = part(p.part_ml, (int64_t)p.wgs * p.qcols * 8, at);
  }
  at = part(p.stat, (int64_t)p.units * p.cols * 8, at);
  at = part(p.state, (int64_t)p.units * 16, at);
  if (p.ns > 1) at = part(p.np, tiles * 8, at);
  if (p.csplit > 1) {
    launch((int64_t)p.units * p.ktiles, kMassKeys);
    part(p.part_mass, (int64_t)p.units * p.ktiles * p.csplit * kMassKeys * 4, at);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_mass_evict(const EvictPlan &p, hipStream_t) {
  ++g_plans;
  CHECK(p.units >= 1 && p.sinks >= 0 && p.recent >= 0 && p.max_rows >= 0 && p.max_rows <= kMassMaxRows);
  launch(p.units, 1024);
  CHECK(p.ldl >= p.max_rows && (int64_t)p.chunks * (kEvictBytes / (2 * p.d)) >= p.max_rows);
  if (p.chunks) launch((int64_t)p.units * p.chunks, 512);
  CHECK(p.index ? p.index_rows > 0 : true);
  const uint8_t *at = part(p.list, (int64_t)p.units * p.ldl * 4, g_ws);
  at = part(p.count, (int64_t)p.units * 4, at);
  at = part(p.flags, (int64_t)p.units * p.chunks * 4, at);
  part(p.ticket, (int64_t)p.units * 4, at);
  return hipErrorInvalidValue;
}

static void norm(const NormPlan &p) {
  ++g_plans;
  CHECK((int64_t)p.L * p.B * p.n < 1 << 24 && p.t.rot >= 16 && p.t.rot <= p.d && p.t.rot % 16 == 0 && p.eps > 0.f);
  CHECK((p.Hq > 0) == (p.qw != nullptr) && (p.Hkv > 0) == (p.kw != nullptr) && p.Hq + p.Hkv > 0);
}
hipError_t launch_norm_rope(const NormPlan &p, hipStream_t) {
  norm(p);
  launch((int64_t)p.L * p.B * p.n, 256);
  return hipErrorInvalidValue;
}
hipError_t launch_norm_rope_grad(const NormPlan &p, hipStream_t) {
  norm(p);
  CHECK(p.groups >= 1 && (p.dqw != nullptr) == (p.qw != nullptr) && (p.dkw != nullptr) == (p.kw != nullptr));
  launch((int64_t)p.L * p.groups, 256);
  launch((int64_t)p.L * 2 * (p.d / 16), 1024);
  part(p.part, (int64_t)p.L * p.groups * 2 * p.d * 4, g_ws);
  return hipErrorInvalidValue;
}

}  // namespace vc

static bool known(vc_status s) { return s >= VC_OK && s <= VC_ERR_HIP; }

int main() {
  const int32_t big = std::numeric_limits<int32_t>::max(), low = std::numeric_limits<int32_t>::min();
  const int64_t far = std::numeric_limits<int64_t>::max();
  void *dev = reinterpret_cast<void *>(uintptr_t(0x700000000000));  // addresses that are never read
  void *dev2 = reinterpret_cast<void *>(uintptr_t(0x710000000000));
  const vc_mass_cache cache{dev, dev, (float *)dev, (int64_t *)dev, (int32_t *)dev, (int32_t *)dev, nullptr};
  const vc_mass_cache other{dev2, dev2, (float *)dev2, (int64_t *)dev2, (int32_t *)dev2, (int32_t *)dev2, (int32_t *)dev2};
  const vc_decode_shape shapes[] = {
      {1, 1, 1, 1, 64},        {1, 28, 28, 4, 128},    {8, 28, 28, 4, 128},  {3, 1, 28, 4, 128},  {130, 1, 4, 1, 64},
      {70, 2, 14, 2, 64},      {1, 1, 16, 1, 128},     {2, 80, 64, 8, 128},  {256, 1, 2, 1, 64},  {257, 1, 2, 1, 64},
      {big, 1, 1, 1, 64},      {46341, 46341, 1, 1, 64}, {big, big, big, big, 128}, {1, 1, 17, 1, 64}, {1, 1, 3, 2, 64},
      {0, 1, 1, 1, 64},        {low, 1, 1, 1, 64},     {1, 1, 4, 4, 96},     {1 << 20, 7, 16, 1, 128}, {1 << 19, 1, 4, 1, 64},
      {1, 1 << 18, 1, 1, 64},  {1, 97, 7, 1, 128},     {1, 128, 8, 1, 128},
  };
  const int32_t ns[] = {low, -1, 0, 1, 2, 4, 5, 16, 17, 64, 65, 256, 257, 1000, 1 << 20, 1 << 24, big};
  const int32_t mr[] = {low, -1, 0, 1, 31, 32, 33, 511, 512, 513, 1500, 5000, 23040, 1 << 20, big - 1023, big};
  char name[256];
  for (const auto &s : shapes) {
    const int64_t d = s.d, H = s.Hq > 0 && s.Hq < 1 << 20 ? s.Hq : 1;
    for (int32_t rows : mr)
      for (int32_t x : {low, -1, 0, 4, big}) {
        std::snprintf(name, sizeof name, "evict B %d L %d Hkv %d d %d rows %d sinks %d", s.B, s.L, s.Hkv, s.d, rows, x);
        g_case = name;
        const size_t need = viscache_mass_evict_workspace_bytes(&s, rows);
        for (int k = 0; k < 4; ++k) {
          g_bytes = need - (k == 3 && need ? 1 : 0);
          const vc_status st = viscache_mass_evict(&s, &cache, k == 1 ? &other : nullptr, (int32_t *)dev, x, x, rows,
                                                   (int32_t *)dev, k == 2 ? x : 1, g_ws, g_bytes, nullptr);
          CHECK(known(st) && (st != VC_ERR_HIP || need > 0));
          if (k == 3) CHECK(st != VC_ERR_HIP);  // a byte too few
          ++g_calls;
        }
      }
    for (int32_t n : ns) {
      const int64_t N = n > 0 ? n : 1, B = s.B > 0 ? s.B : 1;
      // token, head, sequence, layer from the innermost; and strides that overflow.
      const vc_rows t{dev, H * d * N <= far / 64 / B ? B * N * H * d : 0, N * H * d, H * d, d};
      const vc_rows wild[] = {t, {dev, far, far, far, far}, {dev, -8, 0, d, d}, {nullptr, 0, 0, 0, 0}, {dev, 0, 0, 0, 0}};
      for (const auto &r : wild) {
        for (int32_t rows : mr) {
          const size_t need = viscache_mass_attend_workspace_bytes(&s, n, rows);
          std::snprintf(name, sizeof name, "B %d L %d Hq %d Hkv %d d %d n %d rows %d strides %lld %lld %lld %lld", s.B, s.L,
                        s.Hq, s.Hkv, s.d, n, rows, (long long)r.layer, (long long)r.seq, (long long)r.token,
                        (long long)r.head);
          g_case = name;
          for (int k = 0; k < 3; ++k) {
            g_bytes = need - (k == 2 && need ? 1 : 0);
            const vc_status st = viscache_mass_attend(&s, &cache, k ? &r : nullptr, k ? &r : nullptr, &r, &r, n, nullptr, k == 1,
                                                      0.1f, 0.5f, rows, g_ws, g_bytes, nullptr);
            CHECK(known(st) && (st != VC_ERR_HIP || need > 0));
            if (k == 2) CHECK(st != VC_ERR_HIP);
            ++g_calls;
          }
        }
        const vc_rope ropes[] = {
            {s.d, {s.d / 2, 0, 0}, 0, 0, 0, 0, 1.f, 1e6, nullptr}, {s.d, {s.d / 2 - 16, 8, 8}, 1, 1, 1, 1, 1.f, 1e-300, nullptr},
            {big, {big, big, big}, 0, 0, 0, 0, 1.f, 1e6, nullptr}, {low, {low, low, low}, 0, 0, 0, 0, 1.f, 1e6, nullptr}};
        for (const auto &rope : ropes)
          for (float eps : {1e-6f, 0.f, -1.f, 1e38f, std::numeric_limits<float>::quiet_NaN()}) {
            const vc_norm nm{eps, rope.fp32, dev, dev};
            const int32_t *pos = (int32_t *)dev;
            float *w = (float *)dev;
            CHECK(known(viscache_norm_rope(&s, &rope, &nm, n, pos, nullptr, &r, &r, &r, &r, nullptr)));
            CHECK(known(viscache_norm_rope(&s, &rope, &nm, n, pos, nullptr, nullptr, nullptr, &r, &r, nullptr)));
            const size_t need = viscache_norm_rope_grad_workspace_bytes(&s, n);
            for (int k = 0; k < 2; ++k) {
              g_bytes = need - (k && need ? 1 : 0);
              const vc_status st = viscache_norm_rope_grad(&s, &rope, &nm, n, pos, nullptr, &r, &r, &r, w, &r, &r, &r, w, g_ws,
                                                           g_bytes, nullptr);
              CHECK(known(st) && (st != VC_ERR_HIP || (need > 0 && !k)));
            }
            g_bytes = need;
            CHECK(known(viscache_norm_rope_grad(&s, &rope, &nm, n, pos, nullptr, &r, &r, &r, w, nullptr, nullptr, nullptr,
                                                nullptr, g_ws, g_bytes, nullptr)));
            g_calls += 5;
          }
      }
    }
  }
  std::printf("mass host checks ok: %ld calls, %ld plans\n", g_calls, g_plans);
  return g_plans > 1000 ? 0 : 1;
}
