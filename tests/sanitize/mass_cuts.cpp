// mass_cuts.cpp -- prints the cut of attention calls over the cache with masses: for each
// seven arguments (L B Hq Hkv d n max_rows) a line of name=value pairs, from launchers that
// launch nothing.
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "../../include/viscache.h"
#include "../../paper_2608_24063_amd/csrc/vc_mass.h"

namespace vc {

hipError_t launch_mass_token(const MassAttn &p, hipStream_t) {
  std::printf("kind=token waves=%d piece=%d npmax=%d here=%d ldr=%d finish=%d finish_wgs=%d\n", p.waves, p.piece, p.npmax,
              p.here, p.ldr, p.finish, p.finish_wgs);
  return hipSuccess;
}
hipError_t launch_mass_prompt(const MassAttn &p, hipStream_t) {
  std::printf("kind=prompt qcols=%d nqt=%d ns=%d ktiles=%d csplit=%d\n", p.qcols, p.nqt, p.ns, p.ktiles, p.csplit);
  return hipSuccess;
}
hipError_t launch_mass_evict(const EvictPlan &, hipStream_t) { return hipSuccess; }

}  // namespace vc

int main(int argc, char **argv) {
  alignas(256) static uint8_t ws[256];  // stands for any workspace: nothing is written
  void *dev = reinterpret_cast<void *>(uintptr_t(0x700000000000));
  const vc_mass_cache cache{dev, dev, (float *)dev, (int64_t *)dev, (int32_t *)dev, (int32_t *)dev, nullptr};
  for (int i = 1; i + 6 < argc; i += 7) {
    int32_t a[7];
    for (int j = 0; j < 7; ++j) a[j] = std::atoi(argv[i + j]);
    const vc_decode_shape s{a[1], a[0], a[2], a[3], a[4]};
    const int64_t H = s.Hq, d = s.d, n = a[5];
    const vc_rows r{dev, s.B * n * H * d, n * H * d, H * d, d};
    const vc_status st = viscache_mass_attend(&s, &cache, &r, &r, &r, &r, a[5], nullptr, 0, 0.1f, 1.f, a[6], ws,
                                              viscache_mass_attend_workspace_bytes(&s, a[5], a[6]), nullptr);
    if (st != VC_OK) return 1;
  }
  return 0;
}
