// k_mass_cols.hip -- what every row of a cache was given by a prompt's queries, once
// their maxima and sums are known: mass[t] <- decay mass[t] + sum over the columns that
// see row t of exp2(s - m) / l, the logits computed again.
//
// Bound by the vector unit (an exponential and two fused multiply-adds a logit) beside
// the matrix cores.  A wave keeps 64 rows' keys in registers and the workgroup's waves
// walk the columns in blocks of 64 through LDS, double buffered, so that a row's sum
// stays in registers too, is formed in a fixed order and needs no atomics:
//   S = K Q^T in 32x32x16 products, a lane holding 2 x 16 rows of its column.
// 16384 columns over 8 units of 25088 rows, 128 channels: 795 to 840 us (1.0 PFLOP/s of
// products, the matrix cores busy for half of the time; 1120 before products and weights were
// interleaved), and 5 to add up the parts.  455 columns over 12 units of 9000 to 12900 rows:
// 33 to 36 (0.44 PFLOP/s: each workgroup has a start that nothing hides, and where sequences
// have 65, 40 and 15 queries, units on one XCD leave the XCDs 122 to 513 blocks to do).
#include <type_traits>

#include "vc_mass_device.h"

namespace vc {

namespace {

constexpr int kCols = 64;  // columns of a block
constexpr int kSum = 64;   // blocks whose weights a lane adds up in fp32
constexpr int NW = kMassKeys / 64, NT = kMassKeys;  // waves and threads of a workgroup

template <int D>
struct Smem {
  uint16_t q[2][kCols][D + 8] __attribute__((aligned(16)));  // pitch: 16-byte reads of 32 columns without conflicts
  float2 stat[2][kCols];
};

template <int D>
__global__ __launch_bounds__(NT, 2) void k_mass_cols(MassAttn p) {
  constexpr int KS = D / 16, CPR = D / 8, IT = kCols * CPR / NT, CS = NT / CPR;
  __shared__ Smem<D> sm;
  __shared__ float red[NW][64][2];   // the rows' sums, by halves of the lanes
  __shared__ double sums[NW][64][2];  // those of all blocks but the last kSum
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ln = lane & 31, hf = lane >> 5;
  // Splits of a tile's columns innermost, a unit's tiles on one XCD (they share its L2).
  const int id = (int)xcd_block(blockIdx.x, gridDim.x), sp = id % p.csplit, ut = id / p.csplit;
  const int u = ut / p.ktiles, kt = ut % p.ktiles;
  MassUnit x;
  if (p.append) {
    const u32x4 s = ld16(p.state + u);
    x = MassUnit{ldg(p.c.row_off + u), (int)s.x, (int)s.y, (int)s.x, (int)s.z};
  } else {
    x = mass_unit(p, u);
  }
  if (x.cnt == 0) return;
  if (p.append && kt == 0 && sp == 0 && tid == 0) stg(p.c.len + u, x.held);
  const int k0 = kt * NT, emax = min(x.held, p.max_rows);
  if (k0 >= emax) return;
  const int cols = x.cnt * p.G;
  auto rows_seen = [&](int col) { return max(min(x.base + (int)((uint32_t)col / (uint32_t)p.G) + 1, emax), 0); };
  // The first column that sees row t.
  auto sees = [&](int t) { return (int)min((int64_t)max(t - x.base, 0) * p.G, (int64_t)cols); };
  // The split's blocks, of those whose columns see the tile's first row.
  const int all = (cols + kCols - 1) / kCols, lo = sees(k0) / kCols;
  const int first = lo + (int)((int64_t)(all - lo) * sp / p.csplit), nb = lo + (int)((int64_t)(all - lo) * (sp + 1) / p.csplit);
  const int r0 = k0 + 64 * w;  // the wave's rows
  // From this column on every column sees all of them.
  const int full = r0 + 64 <= emax ? sees(r0 + 63) : INT32_MAX;
  bf16x8 k[2][KS];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const uint16_t *src = p.c.kp + (x.off + min(r0 + 32 * kb + ln, emax - 1)) * D + 8 * hf;
#pragma unroll
    for (int s = 0; s < KS; ++s) k[kb][s] = as_bf16x8(ld16(src + 16 * s));
  }
  // A thread's columns, CS apart, go on by kCols a block: their addresses without a division
  // each (which took as many instructions as the logits), and where kCols is a multiple of
  // G, at one step for all.
  const uint16_t *const q0 = reinterpret_cast<const uint16_t *>(p.q.base) + mass_col(p, p.q, u, 0) + 8 * (tid % CPR);
  const int di = kCols / p.G, dh = kCols - di * p.G;
  int64_t at[IT];
  int head[IT];
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int col = first * kCols + tid / CPR + CS * it, i = col / p.G;
    head[it] = col - i * p.G;
    at[it] = i * p.q.token + head[it] * p.q.head;
  }
  int next = first;  // the block that fetch() requests
  const int64_t step = di * p.q.token + dh * p.q.head, turn = p.q.token - p.G * p.q.head;
  const float2 *const stat = p.stat + (int64_t)u * p.cols;
  u32x4 rq[IT];
  float2 rs;
  auto fetch = [&]() {
    if ((next + 1) * kCols <= cols) {  // uniform
#pragma unroll
      for (int it = 0; it < IT; ++it) rq[it] = ld16(q0 + at[it]);
    } else {
#pragma unroll
      for (int it = 0; it < IT; ++it) rq[it] = ld16(q0 + (next * kCols + tid / CPR + CS * it < cols ? at[it] : 0));
    }
    rs = ldg(stat + min(next * kCols + lane, cols - 1));
    ++next;
    if (dh == 0) {  // uniform
#pragma unroll
      for (int it = 0; it < IT; ++it) at[it] += step;
    } else {
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        head[it] += dh;
        at[it] += step;
        if (head[it] >= p.G) {
          head[it] -= p.G;
          at[it] += turn;
        }
      }
    }
  };
  constexpr int kBuf = kCols * (D + 8);
  uint16_t *const put = &sm.q[0][tid / CPR][8 * (tid % CPR)];
  auto stage = [&](int buf) {
    uint16_t *to = put + buf * kBuf;
#pragma unroll
    for (int it = 0; it < IT; ++it) *reinterpret_cast<u32x4 *>(to + it * CS * (D + 8)) = rq[it];
    if (tid < kCols) sm.stat[buf][tid] = rs;
  };
  const uint16_t *const get = &sm.q[0][ln][8 * hf];
  float acc[2][16];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[kb][i] = 0.f;
  // S = K Q^T of half a block in To, beside the weights of the half before it, whose
  // products are in From: two products, then what the vector unit can do in their time.
  // (Left to the compiler's order, products and weights follow one another.)
  auto half = [&](int buf, int cb, f32x16 (&To)[2], int c0, float2 st, const f32x16 (&From)[2], auto what) {
    constexpr int kWhat = decltype(what)::value;  // 0: no weights, 1: all rows seen, 2: masked
    constexpr int E = 32 / KS;                    // weights a step
    const int col = c0 + ln;
    const int end = kWhat == 2 ? (col < cols ? rows_seen(col) : 0) - r0 - 4 * hf : 0;
    u32x4 q[KS];
    const uint16_t *from = get + buf * kBuf;
    auto read = [&](int s) { q[s] = *reinterpret_cast<const u32x4 *>(from + 32 * cb * (D + 8) + 16 * s); };
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) To[kb][i] = 0.f;
    read(0);
    read(1);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if (s + 2 < KS) read(s + 2);
      if (kWhat) {
        float e[E];
#pragma unroll
        for (int j = 0; j < E; ++j) e[j] = fmaf(From[(E * s + j) / 16][(E * s + j) % 16], p.sc, -st.x);
#pragma unroll
        for (int j = 0; j < E; ++j) e[j] = fast_exp2(e[j]);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const int kb = (E * s + j) / 16, i = (E * s + j) % 16;
          if (kWhat == 2)
            acc[kb][i] += 32 * kb + 8 * (i / 4) + i % 4 < end ? e[j] * st.y : 0.f;
          else
            acc[kb][i] = fmaf(e[j], st.y, acc[kb][i]);
        }
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        To[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb][s], as_bf16x8(q[s]), To[kb], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  f32x16 Sa[2], Sb[2];
  if (first < nb) {
    fetch();
    stage(0);
    fetch();
    __syncthreads();
    half(0, 0, Sa, 0, make_float2(0.f, 0.f), Sb, std::integral_constant<int, 0>{});
  }
  // One block.  (Masked and other blocks are loops of their own, since one loop of both
  // would move every sum to another register in each turn.)
  auto block = [&](int b, auto what) {
    const int buf = (b - first) & 1;
    stage(buf ^ 1);
    fetch();
    const float2 sta = sm.stat[buf][ln], stb = sm.stat[buf][32 + ln];
    half(buf, 1, Sb, b * kCols, sta, Sa, what);
    __syncthreads();  // the next block is there, this one's columns are read
    half(buf ^ 1, 0, Sa, b * kCols + 32, stb, Sb, what);
  };
  // The rows' sums over the lanes: to(place in red, sum), in four lanes.
  auto over_lanes = [&](auto to) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[kb][i] = sum_lanes<16>(acc[kb][i]);
    if ((lane & 15) == 0) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          to(2 * (32 * kb + 8 * (i / 4) + 4 * hf + i % 4) + ((lane >> 4) & 1), acc[kb][i]);
    }
  };
  // (Small weights added one at a time to the sum of thousands would be rounded one at a time:
  // rows that got the same from each of 2^18 columns were 1.2e-4 off.)
  double *const far = &sums[w][0][0];
  const bool many = nb - first > kSum;  // uniform
  if (many) far[lane] = far[lane + 64] = 0.0;
  const int b0 = min(max(uniform((int)min((int64_t)full + kCols - 1, (int64_t)INT32_MAX) / kCols), first), nb);
  const int b1 = max(min(cols / kCols, nb), b0);  // blocks [b0, b1) are seen whole
  for (int b = first;;) {
    const int e = min(b + kSum, nb), e0 = min(b0, e), e1 = min(b1, e);
    for (; b < e0; ++b) block(b, std::integral_constant<int, 2>{});
    for (; b < e1; ++b) block(b, std::integral_constant<int, 1>{});
    for (; b < e; ++b) block(b, std::integral_constant<int, 2>{});
    if (e >= nb) break;
    over_lanes([&](int at, float x) { far[at] += (double)x; });
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[kb][i] = 0.f;
  }
  float *const part = &red[w][0][0];
  over_lanes([&](int at, float x) { part[at] = x; });
  __syncthreads();
  const int row = r0 + lane;
  if (row >= emax) return;
  float got = part[2 * lane] + part[2 * lane + 1];
  if (many) got = (float)((far[2 * lane] + far[2 * lane + 1]) + (double)got);
  float *to = p.c.mass + x.off + row;
  if (p.csplit > 1)
    stg(p.part_mass + ((int64_t)ut * p.csplit + sp) * NT + 64 * w + lane, got);
  else
    stg(to, fmaf(p.decay, row < fading_rows(p, x) ? ldg(to) : 0.f, got));
}

// The masses of a tile from its splits, in their order.
__global__ __launch_bounds__(kMassKeys) void k_mass_sum(MassAttn p) {
  const int u = (int)(blockIdx.x / (uint32_t)p.ktiles);
  const int row = (int)(blockIdx.x % (uint32_t)p.ktiles) * kMassKeys + threadIdx.x;
  MassUnit x;
  if (p.append) {  // (the launch before it has set the length)
    const u32x4 s = ld16(p.state + u);
    x = MassUnit{ldg(p.c.row_off + u), (int)s.x, (int)s.y, (int)s.x, (int)s.z};
  } else {
    x = mass_unit(p, u);
  }
  if (x.cnt == 0 || row >= min(x.held, p.max_rows)) return;
  float *to = p.c.mass + x.off + row;
  const float was = ldg(to);
  const float *from = p.part_mass + (int64_t)blockIdx.x * p.csplit * kMassKeys + threadIdx.x;
  double got = 0.0;
#pragma unroll 4
  for (int sp = 0; sp < p.csplit; ++sp) got += (double)ldg(from + (int64_t)sp * kMassKeys);
  stg(to, row < fading_rows(p, x) ? fmaf(p.decay, was, (float)got) : (float)got);
}

template <int D>
void launch(const MassAttn &p, hipStream_t st) {
  hipLaunchKernelGGL((k_mass_cols<D>), dim3((uint32_t)(p.units * p.ktiles * p.csplit)), dim3(NT), 0, st, p);
}

}  // namespace

hipError_t launch_mass_cols(const MassAttn &p, hipStream_t st) {
  if (p.d == 128)
    launch<128>(p, st);
  else
    launch<64>(p, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.csplit == 1) return e;
  hipLaunchKernelGGL(k_mass_sum, dim3((uint32_t)(p.units * p.ktiles)), dim3(kMassKeys), 0, st, p);
  return hipGetLastError();
}

}  // namespace vc
