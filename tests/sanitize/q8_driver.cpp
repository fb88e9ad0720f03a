// q8_driver.cpp -- the host side of the 8-bit cache and the rotary positions
// (argument checks, attention cuts, workspace layout, rotation tables) under
// the sanitizers, without a GPU: the launchers are stand-ins that hold every
// plan against what its kernel takes for granted, then report a failed launch.
// Any call must end in a status, whatever its arguments.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>

#include "../../include/viscache.h"
#include "../../paper_2608_24063_amd/csrc/vc_q8.h"

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

namespace vc {

static void attention(const Q8Attn &p) {
  ++g_plans;
  const int64_t units = (int64_t)p.L * p.B * p.Hkv;
  CHECK(units == p.units && p.G >= 1 && p.G <= 16 && p.G * p.Hkv == p.Hq && p.cols == (int64_t)p.n * p.G);
  CHECK(p.wgs >= 1 && p.wgs < 1 << 23 && std::isfinite(p.sc));
  const uint8_t *o = reinterpret_cast<uint8_t *>(p.part_o), *ml = reinterpret_cast<uint8_t *>(p.part_ml),
                *np = reinterpret_cast<uint8_t *>(p.np);
  CHECK(o == g_ws && ml >= o && np >= ml && (size_t)(np - o) <= g_bytes);
  const int64_t blocks = ((int64_t)p.max_rows + kQ8Block - 1) / kQ8Block;
  int64_t slots = 0, words = 0;
  if (p.cols <= 16) {
    CHECK(p.qcols == 16 && p.piece >= 1 && p.npmax >= 1 && (int64_t)p.piece * p.npmax >= blocks);
    CHECK(p.wgs == units * p.npmax);
    if (p.npmax > 1) slots = (int64_t)p.wgs * 16;
    if (p.npmax > 1 && p.step) words = units;
  } else {
    const int64_t tiles = units * p.nqt;
    CHECK(!p.step && p.npmax == 1 && (p.qcols == 128 || p.qcols == 256));
    CHECK((int64_t)p.nqt * p.qcols >= p.cols && (int64_t)(p.nqt - 1) * p.qcols < p.cols);
    if (p.ns == 1) {
      CHECK(p.wgs == tiles);
    } else {
      // Shares: at most 256 tiles in a wave's registers, and a cut that exists.
      CHECK(tiles <= kQ8SplitTiles && p.wgs >= 2 * tiles);
      slots = (int64_t)p.wgs * p.qcols;
      words = 2 * tiles;
    }
  }
  if (slots) {
    CHECK((int64_t)(ml - o) >= slots * p.d * 4 && (int64_t)(np - ml) >= slots * 8);
    CHECK(units * p.cols < (int64_t)1 << 24);  // the join's launch
  }
  CHECK((int64_t)g_bytes - (np - o) >= words * 4);
}

static void rows(const Q8Rows &p) {
  ++g_plans;
  CHECK(p.units >= 1 && p.nj >= 1 && (int64_t)p.units * p.nj < 1 << 23 && p.n >= 1);
}

hipError_t launch_q8_append(const Q8Rows &p, int, hipStream_t) {
  rows(p);
  CHECK(p.nj == 1 || (int64_t)(p.nj - 1) * kQ8Block >= p.n);
  return hipErrorInvalidValue;
}
hipError_t launch_q8_read(const Q8Rows &p, int, hipStream_t) {
  rows(p);
  CHECK((int64_t)p.nj * kQ8Block >= p.n);
  return hipErrorInvalidValue;
}
hipError_t launch_q8_decode(const Q8Attn &p, int, hipStream_t) {
  CHECK(p.cols <= 16);
  attention(p);
  return hipErrorInvalidValue;
}
hipError_t launch_q8_prompt(const Q8Attn &p, int, hipStream_t) {
  CHECK(p.cols > 16);
  attention(p);
  return hipErrorInvalidValue;
}
hipError_t launch_rope(const RopePlan &p, hipStream_t) {
  ++g_plans;
  CHECK((int64_t)p.L * p.B * p.n < 1 << 24 && p.t.rot >= 16 && p.t.rot <= p.d && p.t.rot % 16 == 0);
  for (int i = 0; i < p.t.rot / 2; ++i) CHECK(std::isfinite(p.t.turns[i]));
  CHECK((p.t.axis1 & p.t.axis2) == 0);
  return hipErrorInvalidValue;
}

}  // namespace vc

static bool known(vc_status s) { return s >= VC_OK && s <= VC_ERR_HIP; }

int main() {
  const int32_t big = std::numeric_limits<int32_t>::max(), low = std::numeric_limits<int32_t>::min();
  const int64_t far = std::numeric_limits<int64_t>::max();
  void *dev = reinterpret_cast<void *>(uintptr_t(0x700000000000));  // an address that is never read
  const vc_q8cache cache{VC_Q8_INT8, dev, dev, (float *)dev, (float *)dev, dev, dev, (int64_t *)dev, (int32_t *)dev,
                         (int32_t *)dev, nullptr};
  const vc_decode_shape shapes[] = {
      {1, 1, 1, 1, 64},        {1, 28, 28, 4, 128},    {8, 28, 28, 4, 128},  {3, 1, 28, 4, 128},  {130, 1, 4, 1, 64},
      {70, 2, 14, 2, 64},      {1, 1, 16, 1, 128},     {2, 80, 64, 8, 128},  {256, 1, 2, 1, 64},  {257, 1, 2, 1, 64},
      {big, 1, 1, 1, 64},      {46341, 46341, 1, 1, 64}, {big, big, big, big, 128}, {1, 1, 17, 1, 64}, {1, 1, 3, 2, 64},
      {0, 1, 1, 1, 64},        {low, 1, 1, 1, 64},     {1, 1, 4, 4, 96},     {1 << 20, 7, 16, 1, 128},
  };
  const int32_t ns[] = {low, -1, 0, 1, 2, 4, 5, 16, 17, 64, 65, 256, 257, 1000, 1 << 20, 1 << 24, big};
  const int32_t mr[] = {low, -1, 0, 1, 63, 64, 65, 511, 512, 5000, 23040, 1 << 20, big - 127, big};
  char name[256];
  for (const auto &s : shapes) {
    const int64_t d = s.d, H = s.Hq > 0 && s.Hq < 1 << 20 ? s.Hq : 1;
    for (int32_t n : ns) {
      const int64_t N = n > 0 ? n : 1, B = s.B > 0 ? s.B : 1;
      // token, head, sequence, layer from the innermost; and strides that overflow.
      const vc_rows t{dev, H * d * N <= far / 64 / B ? B * N * H * d : 0, N * H * d, H * d, d};
      const vc_rows wild[] = {t, {dev, far, far, far, far}, {dev, -8, 0, d, d}, {nullptr, 0, 0, 0, 0}, {dev, 0, 0, 0, 0}};
      for (int32_t rows : mr) {
        const size_t need = viscache_q8_attend_workspace_bytes(&s, n, rows);
        for (const auto &r : wild) {
          std::snprintf(name, sizeof name, "B %d L %d Hq %d Hkv %d d %d n %d rows %d strides %lld %lld %lld %lld", s.B, s.L,
                        s.Hq, s.Hkv, s.d, n, rows, (long long)r.layer, (long long)r.seq, (long long)r.token,
                        (long long)r.head);
          g_case = name;
          for (int k = 0; k < 2; ++k) {
            g_bytes = need - (k && need ? 1 : 0);
            const vc_status st = viscache_q8_attend(&s, &cache, &r, &r, n, nullptr, k, 1, 0.1f, rows, g_ws, g_bytes, nullptr);
            CHECK(known(st) && (st != VC_ERR_HIP || need > 0));
            if (k) CHECK(st != VC_ERR_HIP);  // a byte too few
            ++g_calls;
          }
          g_bytes = viscache_q8_attend_workspace_bytes(&s, 1, rows);
          CHECK(known(viscache_q8_step(&s, &cache, nullptr, nullptr, &r, &r, &r, &r, 0, 0.1f, rows, g_ws, g_bytes, nullptr)));
          CHECK(known(viscache_q8_read(&s, &cache, rows, &r, &r, nullptr, 1, nullptr)));
          CHECK(known(viscache_q8_read(&s, &cache, rows, &r, &r, (int64_t *)dev, 0, nullptr)));
          g_calls += 3;
        }
      }
      for (const auto &r : wild) {
        CHECK(known(viscache_q8_append(&s, &cache, &r, &r, n, nullptr, nullptr, nullptr)));
        CHECK(known(viscache_q8_append(&s, &cache, &r, &r, n, nullptr, (int64_t *)dev, nullptr)));
        double own[64];
        for (double &x : own) x = 1e300;
        const double inf = std::numeric_limits<double>::infinity();
        const vc_rope ropes[] = {
            {s.d, {s.d / 2, 0, 0}, 0, 0, 0, 0, 1.f, 1e6, nullptr}, {s.d, {s.d / 2 - 16, 8, 8}, 1, 1, 1, 1, 1.f, 1e-300, nullptr},
            {16, {2, 3, 3}, 1, 0, 0, 0, 2.f, 1e300, own},          {64, {32, 0, 0}, 0, 0, 0, 0, 1.f, inf, nullptr},
            {big, {big, big, big}, 0, 0, 0, 0, 1.f, 1e6, nullptr}, {64, {big, big, 34}, 0, 0, 0, 0, 1.f, 1e6, nullptr},
            {low, {low, low, low}, 0, 0, 0, 0, 1.f, 1e6, nullptr}, {0, {0, 0, 0}, 0, 0, 0, 0, 1.f, 1e6, nullptr}};
        for (const auto &rope : ropes) {
          CHECK(known(viscache_rope(&s, &rope, n, (int32_t *)dev, nullptr, &r, &r, &r, &r, nullptr)));
          CHECK(known(viscache_rope(&s, &rope, n, (int32_t *)dev, nullptr, nullptr, nullptr, &r, &r, nullptr)));
          g_calls += 2;
        }
        g_calls += 2;
      }
    }
  }
  std::printf("q8 host checks ok: %ld calls, %ld plans\n", g_calls, g_plans);
  return g_plans > 1000 ? 0 : 1;
}
