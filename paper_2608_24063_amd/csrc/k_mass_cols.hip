// k_mass_cols.hip -- what every row of a cache was given by a prompt's queries, once
// their maxima and sums are known: mass[t] <- decay mass[t] + sum over the columns that
// see row t of exp2(s - m) / l, the logits computed again.
//
// Bound by the vector unit (an exponential and two fused multiply-adds a logit) beside
// the matrix cores.  A wave keeps 64 rows' keys in registers and the workgroup's four
// walk the columns in blocks of 64 through LDS, double buffered, so that a row's sum
// stays in registers too, is formed in a fixed order and needs no atomics:
//   S = K Q^T in 32x32x16 products, a lane holding 2 x 16 rows of its column.
#include <algorithm>

#include "vc_mass_device.h"

namespace vc {

namespace {


constexpr int kCols = 64;  // columns of a block

template <int D>
struct Smem {
  uint16_t q[2][kCols][D + 8] __attribute__((aligned(16)));  // pitch: 16-byte reads of 32 columns without conflicts
  float2 stat[2][kCols];
};

template <int D>
__global__ __launch_bounds__(256, 2) void k_mass_cols(MassAttn p) {
  constexpr int KS = D / 16, CPR = D / 8, IT = kCols * CPR / 256;
  __shared__ Smem<D> sm;
  __shared__ float red[4][64][2];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ln = lane & 31, hf = lane >> 5;
  const uint32_t tiles = gridDim.x / (uint32_t)p.units;
  const int id = (int)xcd_block(blockIdx.x, gridDim.x), u = id / (int)tiles, kt = id % (int)tiles;
  MassUnit x;
  if (p.append) {
    const u32x4 s = ld16(p.state + u);
    x = MassUnit{ldg(p.c.row_off + u), (int)s.x, (int)s.y, (int)s.x, (int)s.z};
  } else {
    x = mass_unit(p, u);
  }
  if (x.cnt == 0) return;
  if (p.append && kt == 0 && tid == 0) stg(p.c.len + u, x.held);
  const int k0 = kt * kMassKeys, emax = min(x.held, p.max_rows);
  if (k0 >= emax) return;
  const int cols = x.cnt * p.G;
  auto rows_seen = [&](int col) { return max(min(x.base + (int)((uint32_t)col / (uint32_t)p.G) + 1, emax), 0); };
  // The first column that sees the first row.
  const int first = min((int64_t)max(k0 - x.base, 0) * p.G, (int64_t)cols) / kCols, nb = (cols + kCols - 1) / kCols;
  const int r0 = k0 + 64 * w;  // the wave's rows
  bf16x8 k[2][KS];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const uint16_t *src = p.c.kp + (x.off + min(r0 + 32 * kb + ln, emax - 1)) * D + 8 * hf;
#pragma unroll
    for (int s = 0; s < KS; ++s) k[kb][s] = as_bf16x8(ld16(src + 16 * s));
  }
  u32x4 rq[IT];
  float2 rs;
  auto fetch = [&](int b) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + 256 * it, col = min(b * kCols + e / CPR, cols - 1);
      rq[it] = ld16(reinterpret_cast<const uint16_t *>(p.q.base) + mass_col(p, p.q, u, col) + 8 * (e % CPR));
    }
    rs = ldg(p.stat + (int64_t)u * p.cols + min(b * kCols + (tid & 63), cols - 1));
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + 256 * it;
      *reinterpret_cast<u32x4 *>(&sm.q[buf][e / CPR][8 * (e % CPR)]) = rq[it];
    }
    if (tid < kCols) sm.stat[buf][tid] = rs;
  };
  float acc[2][16];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[kb][i] = 0.f;
  if (first < nb) {
    fetch(first);
    stage(0);
    fetch(min(first + 1, nb - 1));
    __syncthreads();
  }
  for (int b = first; b < nb; ++b) {
    const int buf = (b - first) & 1;
#pragma unroll
    for (int cb = 0; cb < 2; ++cb) {
      const int c0 = b * kCols + 32 * cb, col = c0 + ln;
      if (c0 >= cols) continue;  // uniform
      const float2 st = sm.stat[buf][32 * cb + ln];
      f32x16 S[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) S[kb][i] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const bf16x8 q = as_bf16x8(*reinterpret_cast<const u32x4 *>(&sm.q[buf][32 * cb + ln][16 * s + 8 * hf]));
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) S[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb][s], q, S[kb], 0, 0, 0);
      }
      if (rows_seen(c0) < r0 + 64 || c0 + 32 > cols) {  // wave-uniform: a row unseen, or a column past the last
        const int end = col < cols ? rows_seen(col) : 0;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float e = fast_exp2(fmaf(S[kb][i], p.sc, -st.x)) * st.y;
            acc[kb][i] += r0 + 32 * kb + 8 * (i / 4) + 4 * hf + i % 4 < end ? e : 0.f;
          }
      } else {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[kb][i] = fmaf(fast_exp2(fmaf(S[kb][i], p.sc, -st.x)), st.y, acc[kb][i]);
      }
    }
    stage(buf ^ 1);
    fetch(min(b + 2, nb - 1));
    __syncthreads();
  }
  // The rows' sums over the lanes of their column.
  float *part = &red[w][0][0];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = acc[kb][i];
#pragma unroll
      for (int y = 1; y < 16; y *= 2) v += shfl_xor(v, y);
      if ((lane & 15) == 0) part[2 * (32 * kb + 8 * (i / 4) + 4 * hf + i % 4) + ((lane >> 4) & 1)] = v;
    }
  __syncthreads();
  const int row = r0 + lane;
  if (row < emax) {
    float *to = p.c.mass + x.off + row;
    stg(to, fmaf(p.decay, row < x.len0 ? ldg(to) : 0.f, part[2 * lane] + part[2 * lane + 1]));
  }
}

}  // namespace

hipError_t launch_mass_cols(const MassAttn &p, hipStream_t st) {
  const int64_t tiles = std::max<int64_t>(1, ((int64_t)p.max_rows + kMassKeys - 1) / kMassKeys);
  const dim3 grid((uint32_t)(p.units * tiles));
  if (p.d == 128)
    hipLaunchKernelGGL((k_mass_cols<128>), grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((k_mass_cols<64>), grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace vc
