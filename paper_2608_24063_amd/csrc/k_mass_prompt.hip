// k_mass_prompt.hip -- attention over a bf16 cache for several tokens at a time (more
// than 16 columns, a column being one query of one query head, per kv head), which
// leaves each column's maximum and sum for the pass that adds up the rows' weights
// (k_mass_cols.hip), and the append before it.
//
// Bound by the matrix cores and the exponentials beside them.  A workgroup takes NW x 32
// columns and walks the rows it can see in blocks of 64, through registers into LDS,
// double buffered, from where every wave reads them.  Per wave: S^T = K Q^T and O^T =
// V^T P^T in 32x32x16 products, with the block's rows dealt to the matrix rows so that
// a lane's logits are the k-elements of its own P^T operand; P never leaves the
// registers, and V's operands are transposing reads of its row-major block.
//
// 16384 columns over 8 units of 25088 rows, 128 channels: 1480 to 1590 us (1.02 to 1.1
// PFLOP/s, the matrix cores busy for 0.54 of the time, at the clock that they leave).
// Without the operands' reads and the weights it takes 1049, products and supply without
// weights 1250, weights and supply without products 892.  455 columns over 12 units of
// 9000 to 12900 rows: append 5, attention 40, join 8.
//
// With bf16 outputs a weight is rounded to bf16 before it meets its value (2^-8 of
// itself): a choice of speed, since the errors of a column's weights average out and
// stay under the half step of the output unless its values cancel, and a second part
// makes half as many products again (a call of those 16384 columns 2360 -> 2864 us).  The
// sum of the weights is of the unrounded ones.  With fp32 outputs P is cut in three bf16
// parts (24 bits; 3510 us, 2750 to 2830 of them here).  Sums, maxima, O and the partial
// results are fp32 in both.
#include "vc_mass_device.h"

namespace vc {

namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr int kBlock = kQ8Block;  // rows of a block
// A running maximum may lag behind by this many powers of two before O is rescaled.
constexpr float kLag = 8.f;

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// A unit as the append left it (its length is still the old one where it appends).
__device__ __forceinline__ MassUnit unit_now(const MassAttn &p, int u) {
  if (!p.append) return mass_unit(p, u);
  const u32x4 s = ld16(p.state + u);
  return MassUnit{ldg(p.c.row_off + u), (int)s.x, (int)s.y, (int)s.x, (int)s.z};
}

// Workgroup (unit, 256 chunks of 16 bytes of its new rows): keys and values into the pools,
// masses of zero.  The length itself follows in the last launch, since every workgroup
// here reads it.
__global__ __launch_bounds__(256) void k_append_mass(MassAttn p) {
  const int u = (int)(blockIdx.x % (uint32_t)p.units), j = (int)(blockIdx.x / (uint32_t)p.units);
  const int tid = threadIdx.x, cpr = p.d / 8;
  const MassUnit x = mass_unit(p, u);
  const int i = j * (256 / cpr) + tid / cpr, c = tid % cpr;
  const uint16_t *kn = new_rows(p, p.k, u), *vn = new_rows(p, p.v, u);
  if (j == 0 && tid == 0)
    st16(p.state + u, u32x4{(uint32_t)x.len0, (uint32_t)x.held, (uint32_t)x.cnt, 0u});
  if (i >= x.held - x.len0) return;
  const int64_t row = x.off + x.len0 + i, to = row * p.d + 8 * c;
  const u32x4 a = ld16(kn + i * p.k.token + 8 * c), b = ld16(vn + i * p.v.token + 8 * c);
  st16(p.c.kp + to, a);
  st16(p.c.vp + to, b);
  if (c == 0) stg(p.c.mass + row, 0.f);
}

// Pitches: 16-byte reads of 32 rows, and transposing reads of 4 rows x 64 bytes, without conflicts.
template <int D>
struct Keys {
  uint16_t k[kBlock][D + 8];
};
template <int D>
struct Values {
  uint16_t v[kBlock][D + 32];
};

// Where row r of a 32-row half sits in LDS: matrix row 8 j + 4 h + i holds row
// 16 (j / 2) + 8 h + 4 (j % 2) + i.
__device__ __forceinline__ int place(int r) {
  return (r & 32) | (16 * ((r >> 4) & 1) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3));
}

template <int D, int NW, bool F32>
__global__ __launch_bounds__(64 * NW, 2) void k_prompt(MassAttn p) {
  constexpr int NT = 64 * NW;
  constexpr int KS = D / 16, CB = D / 32, CPR = D / 8;
  constexpr int IT = kBlock * CPR / NT;  // 16-byte chunks of a block's keys (or values) per thread
  // Phases (see the loop) where there are two waves a SIMD and the matrix part is long.
  constexpr bool kPair = NW == 8 && D == 128 && !F32;
  __shared__ Keys<D> tk[2] __attribute__((aligned(16)));
  __shared__ Values<D> tv[2] __attribute__((aligned(16)));
  __shared__ int32_t bad[D];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ln = lane & 31, hf = lane >> 5;
  Share sh;
  if (p.append)  // (two copies, so that it is not asked tile by tile)
    sh = share_of(p, blockIdx.x, lane, [&](int u) {
      const u32x4 s = ld16(p.state + u);
      return Held{(int)s.y, (int)s.z, ldg(p.c.row_off + u)};
    });
  else
    sh = share_of(p, blockIdx.x, lane, [&](int u) {
      const MassUnit x = mass_unit(p, u);
      return Held{x.held, x.cnt, x.off};
    });
  const int u = sh.u, qt = sh.qt, sp = sh.sp, ns = sh.ns;
  if (u < 0) return;
  const int cols = sh.cnt * p.G, c0 = qt * p.qcols;
  if (c0 >= cols) return;
  const int base = uniform(unit_now(p, u).base), emax = min(sh.len, p.max_rows);
  const int cl = min(c0 + p.qcols, cols) - 1;  // last column of the workgroup
  auto rows_seen = [&](int col) { return max(min(base + (int)((uint32_t)col / (uint32_t)p.G) + 1, emax), 0); };
  const int most = rows_seen(cl), fewest = rows_seen(c0);
  const int nt = (most + kBlock - 1) / kBlock;
  const int t0 = (int)((int64_t)sp * nt / ns), T = (int)((int64_t)(sp + 1) * nt / ns) - t0;
  const int col = c0 + 32 * w + ln;
  const int end = rows_seen(min(col, cl));
  const int wmin = rows_seen(min(c0 + 32 * w, cl));  // fewest rows a column of the wave sees
  const bool live = c0 + 32 * w <= cl;  // the wave has columns (the others only stage)
  for (int c = tid; c < D; c += NT) bad[c] = INT32_MAX;

  const uint16_t *kp = uniform(p.c.kp + sh.off * D), *vp = uniform(p.c.vp + sh.off * D);
  u32x4 rk[IT], rv[IT];
  const int whole = uniform(most / kBlock);
  auto fetch = [&](const uint16_t *from, int t, u32x4 (&r)[IT]) {
    if (t < whole) {  // uniform
      const uint16_t *src = from + (int64_t)t * (kBlock * D);
#pragma unroll
      for (int it = 0; it < IT; ++it) r[it] = ld16(src + 8 * (tid + NT * it));
      return;
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + NT * it, row = min(t * kBlock + e / CPR, most - 1);
      r[it] = ld16(from + (int64_t)row * D + 8 * (e % CPR));
    }
  };
  // The queries' requests and the first block's, before anything waits.
  bf16x8 q[KS];
  {
    const uint16_t *qp = reinterpret_cast<const uint16_t *>(p.q.base) + mass_col(p, p.q, u, min(col, cl));
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = as_bf16x8(ld16(qp + 16 * s + 8 * hf));
  }
  if (T > 0) {
    fetch(kp, t0, rk);
    fetch(vp, t0, rv);
  }
  auto stage_k = [&](int buf) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + NT * it;
      *reinterpret_cast<u32x4 *>(&tk[buf].k[place(e / CPR)][8 * (e % CPR)]) = rk[it];
    }
  };
  auto stage_v = [&](int buf, int t) {
    if ((t + 1) * kBlock > fewest) {  // uniform: some column does not see all of it
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int e = tid + NT * it;
        if (any_nonfinite(rv[it])) rv[it] = without_nonfinite(rv[it], min(t * kBlock + e / CPR, most - 1), bad + 8 * (e % CPR));
      }
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + NT * it;
      *reinterpret_cast<u32x4 *>(&tv[buf].v[e / CPR][8 * (e % CPR)]) = rv[it];
    }
  };

  f32x16 O[CB], S[2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[cb][i] = 0.f;
  // The sum of the weights, block by block: small weights added one at a time to the sum of
  // thousands would be lost one at a time (7e-6 of the masses over 25000 rows), and what a
  // block's addition rounds off is kept.
  float m = kNegInf, l = 0.f, lost = 0.f;
  constexpr int NP = F32 ? 3 : 1;  // parts of P
  u32x4 P[NP][4];

  auto logits = [&](const Keys<D> &K) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int k = 0; k < 16; ++k) S[kb][k] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        S[kb] = mfma32(as_bf16x8(*reinterpret_cast<const u32x4 *>(&K.k[32 * kb + ln][16 * s + 8 * hf])), q[s], S[kb]);
  };
  // Lanes 16 g .. 16 g + 15 read rows 16 s + 8 hf + 0 .. 3 (and 4 .. 7) of 16 channels, and get
  // a channel each.
  const int vrow = 8 * hf + ((lane & 15) >> 2), vch = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto outputs = [&](const Values<D> &V) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const u32x2 a0 = lds_transposed(&V.v[16 * s + vrow][32 * cb + vch]);
        const u32x2 a1 = lds_transposed(&V.v[16 * s + vrow + 4][32 * cb + vch]);
        const bf16x8 a = as_bf16x8(u32x4{a0.x, a0.y, a1.x, a1.y});
#pragma unroll
        for (int y = 0; y < NP; ++y) O[cb] = mfma32(a, as_bf16x8(P[y][s]), O[cb]);
      }
  };
  // The matrix part of block i: the block before it into O, and its logits; the operands'
  // reads (two a product of V, one of K) run kAhead products ahead.
  auto products = [&](int i) {
    outputs(tv[(i & 1) ^ 1]);
    logits(tk[i & 1]);
    if (!F32) {
      constexpr int kPV = 4 * CB, kAll = 2 * KS + kPV, kAhead = 4;
      __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 0);
#pragma unroll
      for (int k = 0; k < kAll - kAhead; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        if (k + kAhead < kPV)
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        else
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, kAhead, 0);
    }
  };
  // The weights of block t0 + i from its logits.
  float inf = __builtin_inff();
  asm("" : "+s"(inf));  // (else the compiler makes med3 a maximum of quieted inputs)
  auto weights = [&](int i) {
    const int t = t0 + i;
    if ((t + 1) * kBlock > wmin) {  // wave-uniform
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int row = t * kBlock + 32 * kb + 16 * (k >> 3) + 8 * hf + 4 * ((k >> 2) & 1) + (k & 3);
          if (row >= end) S[kb][k] = kNegInf;
        }
    }
    // (med3 with infinity is a maximum that needs no quieted inputs.)
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = __builtin_amdgcn_fmed3f(S[0][k], S[1][k], inf);
    float mx = fmaxf(x[0], x[1]);
#pragma unroll
    for (int k = 2; k < 16; ++k) mx = fmaxf(mx, x[k]);
    mx = max_halves(mx) * p.sc;
    if (__builtin_amdgcn_ballot_w64(mx > m + kLag)) {
      const float mn = fmaxf(m, mx);
      const float alpha = mn == kNegInf ? 0.f : fast_exp2(m - mn);
      m = mn;
      l *= alpha;
      lost *= alpha;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) O[cb] *= alpha;
    }
    const float off = m == kNegInf ? 0.f : -m;
    float sum[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      float pr[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        pr[k] = fast_exp2(fmaf(S[s / 2][8 * (s % 2) + k], p.sc, off));
        sum[s] = k == 0 ? pr[0] : sum[s] + pr[k];
      }
      if (F32) {
#pragma unroll
        for (int y = 0; y < NP; ++y) {
          P[y][s] = u32x4{tops(pr[0], pr[1]), tops(pr[2], pr[3]), tops(pr[4], pr[5]), tops(pr[6], pr[7])};
#pragma unroll
          for (int k = 0; k < 8; ++k) pr[k] -= top_of(pr[k]);  // exact
        }
      } else {
        P[0][s] = u32x4{pack_bf16(pr[0], pr[1]), pack_bf16(pr[2], pr[3]), pack_bf16(pr[4], pr[5]), pack_bf16(pr[6], pr[7])};
      }
    }
    const float b = (sum[0] + sum[1]) + (sum[2] + sum[3]), to = l + b, was = to - b;
    lost += (l - was) + (b - (to - was));
    l = to;
  };
  // Keys of block i + 1 and values of block i into LDS, and the requests of the ones
  // after them.  Past the last block the last one again: under a condition the
  // requests would wait for each other.
  auto supply = [&](int i) {
    stage_k((i + 1) & 1);
    stage_v(i & 1, t0 + i);
    fetch(kp, t0 + min(i + 2, T - 1), rk);
    fetch(vp, t0 + min(i + 1, T - 1), rv);
  };

  __syncthreads();  // (bad is set)
  if (T > 0) {
    stage_k(0);
    fetch(kp, t0 + min(1, T - 1), rk);
    __syncthreads();
    if (kPair) {
      // Two waves share a SIMD: while one multiplies and stages, the other
      // weighs.  The second half of the waves runs one phase behind.
      const bool first = w < NW / 2;
      if (!first) __syncthreads();
      if (live) logits(tk[0]);
      supply(0);
      __syncthreads();
      for (int i = 1; i < T; ++i) {
        if (live) weights(i - 1);
        __syncthreads();
        if (live) products(i);
        supply(i);
        __syncthreads();
      }
      if (live) weights(T - 1);
      if (first) __syncthreads();
      if (live) outputs(tv[(T - 1) & 1]);
    } else {
      if (live) {
        logits(tk[0]);
        weights(0);
      }
      supply(0);
      __syncthreads();
      for (int i = 1; i < T; ++i) {
        if (live) {
          products(i);
          weights(i);
        }
        supply(i);
        __syncthreads();
      }
      if (live) outputs(tv[(T - 1) & 1]);
    }
  }
  l = sum_halves(l + lost);
  __syncthreads();  // (the last of bad)
  if ((t0 + T) * kBlock > fewest) {  // uniform
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (bad[32 * cb + 8 * (i / 4) + 4 * hf + i % 4] < end) O[cb][i] = __builtin_nanf("");
  }
  // (Here, since a store before the loop would keep loads in it out of scalar registers.)
  if (p.ns > 1 && sp == 0 && tid == 0)
    st8(reinterpret_cast<uint32_t *>(p.np) + 2 * (u * p.nqt + qt), u32x2{(uint32_t)sh.id, (uint32_t)ns});
  if (col > cl) return;
  const float mm = m == kNegInf ? 0.f : m;
  if (ns == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (hf == 0) stg(p.stat + (int64_t)u * p.cols + col, make_float2(mm, inv));
    const int64_t at = mass_col(p, p.out, u, col);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 32 * cb + 8 * i + 4 * hf;
        const float a = O[cb][4 * i] * inv, bb = O[cb][4 * i + 1] * inv, cc = O[cb][4 * i + 2] * inv,
                    d = O[cb][4 * i + 3] * inv;
        if (F32)
          st16(reinterpret_cast<float *>(p.out.base) + at + ch,
               u32x4{__float_as_uint(a), __float_as_uint(bb), __float_as_uint(cc), __float_as_uint(d)});
        else
          st8(reinterpret_cast<uint16_t *>(p.out.base) + at + ch, u32x2{pack_bf16(a, bb), pack_bf16(cc, d)});
      }
    return;
  }
  const int64_t at = (int64_t)sh.id * p.qcols + 32 * w + ln;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      st16(p.part_o + at * D + 32 * cb + 8 * i + 4 * hf,
           u32x4{__float_as_uint(O[cb][4 * i]), __float_as_uint(O[cb][4 * i + 1]), __float_as_uint(O[cb][4 * i + 2]),
                 __float_as_uint(O[cb][4 * i + 3])});
  if (hf == 0) stg(p.part_ml + at, make_float2(m, l));
}

// A column's parts, four channels a thread: the output and the column's maximum and sum.
template <int D>
__global__ __launch_bounds__(256) void k_join_mass(MassAttn p) {
  constexpr int TPC = D / 4, CPW = 256 / TPC, U = 8;  // threads a column, columns a workgroup, parts in flight
  const int tid = threadIdx.x, ch = tid % TPC * 4;
  const int64_t cg = (int64_t)blockIdx.x * CPW + tid / TPC;
  if (cg >= (int64_t)p.units * p.cols) return;
  const int u = (int)(cg / p.cols), col = (int)(cg % p.cols);
  const int cnt_ = p.count ? ldg(p.count + u / p.Hkv % p.B) : p.n;
  if (col >= min(max(cnt_, 0), p.n) * p.G) return;
  const u32x2 v = ld8(reinterpret_cast<const uint32_t *>(p.np) + 2 * (u * p.nqt + col / p.qcols));
  const int ns = (int)v.y;
  if (ns <= 1) return;  // written already
  const int64_t at = (int64_t)v.x * p.qcols + col % p.qcols;
  float M = kNegInf, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < ns; s0 += U) {
    float2 ml[U];
    u32x4 x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t a = at + (int64_t)min(s0 + k, ns - 1) * p.qcols;
      ml[k] = ldg(p.part_ml + a);
      x[k] = ld16(p.part_o + a * D + ch);
    }
    const float before = M;
#pragma unroll
    for (int k = 0; k < U; ++k) M = fmaxf(M, ml[k].x);
    // (Without a maximum there are no rows, all zeros, or only NaN, which stay.)
    const float r = M == kNegInf ? 0.f : M, f0 = fast_exp2(before - r);
    l *= f0;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= f0;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (s0 + k >= ns) continue;
      const float f = fast_exp2(ml[k].x - r);
      const uint32_t xs[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
      l += f * ml[k].y;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += f * __uint_as_float(xs[i]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (ch == 0) stg(p.stat + cg, make_float2(M == kNegInf ? 0.f : M, inv));
  const int64_t to = mass_col(p, p.out, u, col) + ch;
  if (p.fp32)
    st16(reinterpret_cast<float *>(p.out.base) + to,
         u32x4{__float_as_uint(o[0] * inv), __float_as_uint(o[1] * inv), __float_as_uint(o[2] * inv),
               __float_as_uint(o[3] * inv)});
  else
    st8(reinterpret_cast<uint16_t *>(p.out.base) + to,
        u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)});
}

template <int D, int NW>
void launch_nw(const MassAttn &p, hipStream_t st) {
  const dim3 grid((uint32_t)p.wgs), block(64 * NW);
  if (p.fp32)
    hipLaunchKernelGGL((k_prompt<D, NW, true>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((k_prompt<D, NW, false>), grid, block, 0, st, p);
}

template <int D>
hipError_t launch(const MassAttn &p, hipStream_t st) {
  hipError_t e;
  if (p.append) {
    const int64_t rows = 2048 / D, nj = (p.n + rows - 1) / rows;
    hipLaunchKernelGGL(k_append_mass, dim3((uint32_t)(p.units * nj)), dim3(256), 0, st, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (p.qcols == 256)
    launch_nw<D, 8>(p, st);
  else
    launch_nw<D, 4>(p, st);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (p.ns > 1) {
    constexpr int CPW = 256 / (D / 4);
    const int64_t cols = (int64_t)p.units * p.cols;
    hipLaunchKernelGGL((k_join_mass<D>), dim3((uint32_t)((cols + CPW - 1) / CPW)), dim3(256), 0, st, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return launch_mass_cols(p, st);
}

}  // namespace

hipError_t launch_mass_prompt(const MassAttn &p, hipStream_t st) {
  return p.d == 128 ? launch<128>(p, st) : launch<64>(p, st);
}

}  // namespace vc
