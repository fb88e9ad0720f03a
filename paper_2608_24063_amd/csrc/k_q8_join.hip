// k_q8_join.hip -- joins the partial results (max, sum, O) that an attention
// over the 8-bit cache leaves for a column whose rows went to several
// workgroups.
//
// Bound by latency: a workgroup takes one column and deals its parts to groups
// of D / 4 threads, four parts in flight each, so that a unit cut into many
// parts costs few round trips.  A launch of its own costs less than the last
// workgroup's joining them in the attention's launch did: there the partials
// need device-coherent stores, a wait for them and an atomic, and one workgroup
// joins a whole unit (4 units of 12544 rows: 18.5 us in one launch).
#include "vc_q8_device.h"

namespace vc {

namespace {

constexpr float kNegInf = -__builtin_inff();

template <int D>
__global__ __launch_bounds__(256) void k_join(Q8Attn p) {
  constexpr int TPG = D / 4, NG = 256 / TPG, U = 4;
  __shared__ float so[NG][D + 4];
  __shared__ float2 sml[NG];
  const int u = (int)(blockIdx.x / (uint32_t)p.cols), col = (int)(blockIdx.x % (uint32_t)p.cols);
  const int tid = threadIdx.x, grp = tid / TPG, ch = tid % TPG * 4;
  const int g = u % p.Hkv, lb = u / p.Hkv, b = lb % p.B;
  const int len_ = ldg(p.c.len + u), cap_ = ldg(p.c.cap + u), cnt_ = p.count ? ldg(p.count + b) : p.n;
  int2 tiles = make_int2(0, 0);
  if (p.npmax == 1 && p.count) tiles = count_tiles(p, b, tid & 63);
  if (col >= min(max(cnt_, 0), p.n) * p.G) return;
  int64_t at;  // part 0 of the column
  int ns;
  if (p.npmax > 1) {  // pieces: as many as the unit's rows make; a single one wrote its output
    const int rows = min(max(min(len_, cap_), 0), p.max_rows);
    ns = ((rows + kQ8Block - 1) / kQ8Block + p.piece - 1) / p.piece;
    if (ns <= 1) return;
    at = (int64_t)u * p.npmax * p.qcols + col;
  } else {
    int64_t tile = (int64_t)u * p.nqt;
    ns = p.ns;
    if (p.count) {  // as share_of has them
      ns = splits_of(p, tiles.x, (uint32_t)p.wgs);
      tile = ((int64_t)(lb / p.B) * tiles.x + tiles.y) * p.Hkv + (int64_t)g * tiles_of(p, b);
    }
    if (ns == 1) return;  // written already
    at = (tile + col / p.qcols) * ns * p.qcols + col % p.qcols;
  }
  float M = kNegInf, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = grp; s0 < ns; s0 += NG * U) {
    float2 ml[U];
    u32x4 x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t a = at + (int64_t)min(s0 + k * NG, ns - 1) * p.qcols;
      ml[k] = ldg(p.part_ml + a);
      x[k] = ld16(p.part_o + a * D + ch);
    }
    float Mc = M;
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (s0 + k * NG < ns) Mc = fmaxf(Mc, ml[k].x);
    if (Mc == kNegInf) continue;
    const float f0 = fast_exp2(M - Mc);
    l *= f0;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= f0;
    M = Mc;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (s0 + k * NG >= ns) continue;
      const float f = fast_exp2(ml[k].x - Mc);
      l += f * ml[k].y;
      o[0] += f * __uint_as_float(x[k].x);
      o[1] += f * __uint_as_float(x[k].y);
      o[2] += f * __uint_as_float(x[k].z);
      o[3] += f * __uint_as_float(x[k].w);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) so[grp][ch + i] = o[i];
  if (ch == 0) sml[grp] = make_float2(M, l);
  __syncthreads();
  if (tid >= D) return;
  float Mt = kNegInf;
#pragma unroll
  for (int k = 0; k < NG; ++k) Mt = fmaxf(Mt, sml[k].x);
  float ot = 0.f, lt = 0.f;
  if (Mt != kNegInf) {
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      const float f = fast_exp2(sml[k].x - Mt);
      ot += f * so[k][tid];
      lt += f * sml[k].y;
    }
  }
  const float v = lt > 0.f ? ot / lt : 0.f;
  const int64_t to = (int64_t)(lb / p.B) * p.out.layer + (int64_t)b * p.out.seq + (int64_t)(col / p.G) * p.out.token +
                     (int64_t)(g * p.G + col % p.G) * p.out.head + tid;
  if (p.fp32)
    stg(reinterpret_cast<float *>(p.out.base) + to, v);
  else
    stg(reinterpret_cast<uint16_t *>(p.out.base) + to, (uint16_t)pack_bf16(v, 0.f));
}

}  // namespace

hipError_t launch_q8_join(const Q8Attn &p, hipStream_t st) {
  const dim3 grid((uint32_t)((int64_t)p.units * p.cols)), block(256);
  if (p.d == 128)
    hipLaunchKernelGGL((k_join<128>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((k_join<64>), grid, block, 0, st, p);
  return hipGetLastError();
}

}  // namespace vc
