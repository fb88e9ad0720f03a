// k_q8_prompt.hip -- attention over the 8-bit cache for several tokens at a
// time (more than 16 columns, a column being one query of one query head, per
// kv head).
//
// Bound by the matrix cores and the exponentials beside them.  A workgroup
// takes NW x 32 columns and walks the rows it can see in blocks of 64; each
// block's codes are turned into fp16 (in which they are exact) once per
// workgroup on their way from registers into LDS, double buffered, and read
// from there by every wave.  Per wave: S^T = K Q^T and O^T = V^T P^T in
// 32x32x16 products, with the block's rows dealt to the matrix rows so that a
// lane's logits are the k-elements of its own P^T operand; P never leaves the
// registers.
//
// Scales: the key scale multiplies the logits.  With bf16 outputs the value
// scale goes into the exponent, p' = exp2(c s + log2 vs_b - m), m the running
// maximum of the same quantity, and the sum takes it out again,
// l += sum(p') / vs_b: O needs no pass of its own per block, and no block's p'
// exceeds the range of fp16.  p' is one fp16 value: 2^-12 of itself, and half of
// fp16's smallest step, 2^-33 of the column's largest weight times value scale.
// That is a choice of speed: the errors of a column's weights average out and
// stay under the half step of a bf16 output (2^-9 of it and more), unless its
// values cancel; a second part would make half as many products again.  With fp32
// outputs P is split in two fp16 parts (22 bits) and each block's product is scaled
// into O in fp32.  Sums, maxima, O and the partial results are fp32 in both.
//
// Measured: 2048 queries of 64 heads over 23040 rows, 128 channels, int8: 1315 to
// 1395 us on several machines, 1.06 to 1.13 PFLOP/s, 0.86 to 0.91 of a large library
// product's rate (1418 to 1435 us under the profiler).  Of a SIMD's cycles 54% are
// matrix instructions'; the vector unit's come on top of them, and the clock falls to
// 1.9 GHz.  Three ragged questions of up to 65 tokens over 9001 to 12801 rows: 46 us
// a call; under the profiler 42, 8.5 of them before the first block is in LDS, and 8
// to join.
#include "vc_q8_device.h"

namespace vc {

namespace {

constexpr float kNegInf = -__builtin_inff();
// A running maximum may lag behind by this many powers of two before O is
// rescaled, and p' is kept 2^kLift above 1: fp16 holds 2^(kLag + kLift).
constexpr float kLag = 6.f, kLift = 8.f;

__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Pitches in halves: 16-byte reads of 32 rows without conflicts.
template <int D>
struct Keys {
  _Float16 k[kQ8Block][D + 8];
};
template <int D>
struct Values {
  _Float16 v[D][kQ8Block + 8];
};

// Where row r of a 32-row half sits in LDS: matrix row 8 j + 4 h + i holds row
// 16 (j / 2) + 8 h + 4 (j % 2) + i.
__device__ __forceinline__ int place(int r) {
  return (r & 32) | (16 * ((r >> 4) & 1) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3));
}

template <int D, int FMT, int NW, bool F32>
__global__ __launch_bounds__(64 * NW, 2) void k_prompt8(Q8Attn p) {
  constexpr int NT = 64 * NW;
  constexpr int KS = D / 16, CB = D / 32;
  constexpr int kItems = kQ8Block * D / 16;           // 16-code chunks of a block's keys (or values)
  constexpr int IT = (kItems + NT - 1) / NT;
  constexpr bool kPart = kItems < NT;                 // only the first kItems threads have one
  // Phases (see the loop) pay where there are two waves a SIMD and the matrix
  // part is long: d = 128 with bf16 outputs.  (us, with and without: 2048 queries
  // over 23040 rows in 64 heads 1362, 1427; 64 over 1300 in 28 layers 52, 58; d =
  // 64, 1024 over 8192 in four sequences 132, 126; fp32 outputs, which then spill
  // registers, 2222, 2186.)
  constexpr bool kPair = NW == 8 && D == 128 && !F32;
  __shared__ Keys<D> tk[2] __attribute__((aligned(16)));
  __shared__ Values<D> tv[2] __attribute__((aligned(16)));
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ln = lane & 31, hf = lane >> 5;
  const Share sh = share_of(p, blockIdx.x, lane, [&](int u) {
    return Held{rows_held(ldg(p.c.len + u), ldg(p.c.cap + u)),
                p.count ? min(max(ldg(p.count + u / p.Hkv % p.B), 0), p.n) : p.n, ldg(p.c.row_off + u)};
  });
  const int u = sh.u, qt = sh.qt, sp = sh.sp, ns = sh.ns;
  if (u < 0) return;
  const int len = sh.len, cnt = sh.cnt, cols = cnt * p.G;
  const int c0 = qt * p.qcols;
  if (c0 >= cols) return;
  const int cl = min(c0 + p.qcols, cols) - 1;  // last column of the workgroup
  const int lim = p.causal ? len - cnt + 1 : len;
  auto rows_seen = [&](int col) { return max(min(p.causal ? lim + col / p.G : len, p.max_rows), 0); };
  const int emax = rows_seen(cl);
  const int nt = (emax + kQ8Block - 1) / kQ8Block;
  const int t0 = (int)((int64_t)sp * nt / ns), T = (int)((int64_t)(sp + 1) * nt / ns) - t0;
  const int col = c0 + 32 * w + ln;
  const int end = rows_seen(min(col, cl));
  const int wmin = rows_seen(min(c0 + 32 * w, cl));  // fewest rows a column of the wave sees
  const bool live = c0 + 32 * w <= cl;  // the wave has columns (the others only stage)
  const int64_t blk0 = sh.off / kQ8Block;
  const int nsealed = len / kQ8Block;
  const int g = u % p.Hkv, lb = u / p.Hkv;
  auto row_of = [&](const RowsDesc &r, int cc) {
    return (int64_t)(lb / p.B) * r.layer + (int64_t)(lb % p.B) * r.seq + (int64_t)(cc / p.G) * r.token +
           (int64_t)(g * p.G + cc % p.G) * r.head;
  };

  u32x4 rk[IT], rv[IT];
  auto fetch_k = [&](int t) {
    const uint8_t *k = p.c.kc + (blk0 + t) * (kQ8Block * D);
#pragma unroll
    for (int it = 0; it < IT; ++it) rk[it] = ld16(k + 16 * (kPart ? min(tid, kItems - 1) : tid + NT * it));
  };
  auto fetch_v = [&](int t) {
    const uint8_t *v = p.c.vc + (blk0 + t) * (kQ8Block * D);
#pragma unroll
    for (int it = 0; it < IT; ++it) rv[it] = ld16(v + 16 * (kPart ? min(tid, kItems - 1) : tid + NT * it));
  };
  // The queries' requests and the first block's, before anything waits.
  const int Tc = max(min(t0 + T, nsealed) - t0, 0);  // sealed blocks
  f16x8 q[KS];
  float cq;
  {
    const uint16_t *qp = reinterpret_cast<const uint16_t *>(p.q.base) + row_of(p.q, min(col, cl));
    u32x4 x[KS];
    uint32_t mag = 0u;
#pragma unroll
    for (int s = 0; s < KS; ++s) x[s] = ld16(qp + 16 * s + 8 * hf);
    if (Tc > 0) {
      fetch_k(t0);
      fetch_v(t0);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s)
      mag = max_mag(max_mag(max_mag(max_mag(mag, x[s].x), x[s].y), x[s].z), x[s].w);
    uint32_t mm = max(mag & 0xFFFFu, mag >> 16);
    mm = max(mm, (uint32_t)__shfl_xor((int)mm, 32, 64));
    const float qs = open_scale(mm);
    cq = p.sc * qs;
    const float inv = 1.f / qs;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = half8_of_bf16(x[s], inv);
  }

  auto stage_k = [&](int buf) {
    if (kPart && tid >= kItems) return;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + NT * it;
      _Float16 *to = &tk[buf].k[place(e / (D / 16))][16 * (e % (D / 16))];
      *reinterpret_cast<f16x8 *>(to) = Q8<FMT>::half8(rk[it].x, rk[it].y);
      *reinterpret_cast<f16x8 *>(to + 8) = Q8<FMT>::half8(rk[it].z, rk[it].w);
    }
  };
  auto stage_v = [&](int buf) {
    if (kPart && tid >= kItems) return;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + NT * it;
      _Float16 *to = &tv[buf].v[e / 4][16 * (e % 4)];
      *reinterpret_cast<f16x8 *>(to) = Q8<FMT>::half8(rv[it].x, rv[it].y);
      *reinterpret_cast<f16x8 *>(to + 8) = Q8<FMT>::half8(rv[it].z, rv[it].w);
    }
  };
  // The open block: bf16 rows scaled by their powers of two, zeros past its end.
  const int orows = len - nsealed * kQ8Block;
  auto open_rows = [&](const uint16_t *tail, const float *scale, auto put) {
    const float inv = 1.f / ldg(scale + blk0 + nsealed);
    for (int e = tid; e < kQ8Block * D / 8; e += NT) {
      const int row = e / (D / 8), c = e % (D / 8);
      const u32x4 x = row < orows ? ld16(tail + (int64_t)u * kQ8Block * D + row * D + 8 * c) : u32x4{0u, 0u, 0u, 0u};
      put(row, 8 * c, half8_of_bf16(x, inv));
    }
  };
  auto open_k = [&](int buf) {
    open_rows(p.c.kt, p.c.ks, [&](int row, int c, f16x8 x) { *reinterpret_cast<f16x8 *>(&tk[buf].k[place(row)][c]) = x; });
  };
  auto open_v = [&](int buf) {
    open_rows(p.c.vt, p.c.vs, [&](int row, int c, f16x8 x) {
#pragma unroll
      for (int k = 0; k < 8; ++k) tv[buf].v[c + k][row] = x[k];
    });
  };

  f32x16 O[CB], S[2];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[cb][i] = 0.f;
  float m = kNegInf, l = 0.f;
  f16x8 hi[4], lo[4];
  float vprev = 1.f;  // the value scale that belongs to hi and lo

  auto logits = [&](const Keys<D> &K) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int k = 0; k < 16; ++k) S[kb][k] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        S[kb] = mfma32(*reinterpret_cast<const f16x8 *>(&K.k[32 * kb + ln][16 * s + 8 * hf]), q[s], S[kb]);
  };
  auto outputs = [&](const Values<D> &V) {
    if (F32) {
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        f32x16 acc;
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[k] = 0.f;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const f16x8 a = *reinterpret_cast<const f16x8 *>(&V.v[32 * cb + ln][16 * s + 8 * hf]);
          acc = mfma32(a, lo[s], mfma32(a, hi[s], acc));
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) O[cb][k] = fmaf(acc[k], vprev, O[cb][k]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
          O[cb] = mfma32(*reinterpret_cast<const f16x8 *>(&V.v[32 * cb + ln][16 * s + 8 * hf]), hi[s], O[cb]);
    }
  };
  // The open block's into O, for the columns that see a row of it: the weights of the
  // others are zero, but an infinity or a NaN among its values is not.
  auto open_outputs = [&](const Values<D> &V) {
    const bool sees = end > nsealed * kQ8Block;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      f32x16 acc;
#pragma unroll
      for (int k = 0; k < 16; ++k) acc[k] = 0.f;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const f16x8 a = *reinterpret_cast<const f16x8 *>(&V.v[32 * cb + ln][16 * s + 8 * hf]);
        acc = mfma32(a, hi[s], acc);
        if (F32) acc = mfma32(a, lo[s], acc);
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) O[cb][k] = fmaf(sees ? acc[k] : 0.f, F32 ? vprev : 1.f, O[cb][k]);
    }
  };
  // The matrix part of block i: its logits, and the block before it into O; the
  // operands' reads run kAhead products ahead.
  auto products = [&](int i) {
    outputs(tv[(i & 1) ^ 1]);
    logits(tk[i & 1]);
    if (!F32) {
      constexpr int kAll = 2 * KS + 4 * CB, kAhead = 4;
      __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
      for (int k = 0; k < kAll - kAhead; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, kAhead, 0);
    }
  };
  // The weights of block t0 + i from its logits.
  auto weights = [&](int i, float ks, float vs) {
    const int t = t0 + i;
    const float c = fmaxf(cq * ks, 1e-37f);
    if ((t + 1) * kQ8Block > wmin) {  // wave-uniform
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int row = t * kQ8Block + 32 * kb + 16 * (k >> 3) + 8 * hf + 4 * ((k >> 2) & 1) + (k & 3);
          if (row >= end) S[kb][k] = kNegInf;
        }
    }
    // (med3 with infinity is a maximum that needs no quieted inputs.)
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = __builtin_amdgcn_fmed3f(S[0][k], S[1][k], __builtin_inff());
    float mx = fmaxf(x[0], x[1]);
#pragma unroll
    for (int k = 2; k < 16; ++k) mx = fmaxf(mx, x[k]);
    const float lvs = F32 ? 0.f : __builtin_amdgcn_logf(vs);
    mx = fmaf(max_halves(mx), c, lvs);
    if (__builtin_amdgcn_ballot_w64(mx > (F32 ? m : m + kLag))) {
      const float mn = fmaxf(m, mx);
      const float alpha = mn == kNegInf ? 0.f : fast_exp2(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) O[cb] *= alpha;
    }
    // lvs less the maximum, plus the lift; anything finite while the column
    // has seen no row.
    const float off = (m == kNegInf ? 0.f : lvs - m) + (F32 ? 0.f : kLift);
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float pr = fast_exp2(fmaf(S[kb][k], c, off));
        sum += pr;
        if (F32) {
          const float ps = pr * 16384.f;
          const _Float16 h = (_Float16)ps;
          hi[2 * kb + k / 8][k % 8] = h;
          lo[2 * kb + k / 8][k % 8] = (_Float16)(ps - (float)h);
        } else {
          hi[2 * kb + k / 8][k % 8] = (_Float16)pr;
        }
      }
    l = F32 ? l + sum : fmaf(sum, __builtin_amdgcn_rcpf(vs), l);
    vprev = vs;
  };
  // Keys of sealed block i + 1 and values of block i into LDS, and the requests
  // of the ones after them.  Past the last block the last one again: under a
  // condition the requests would wait for each other.
  auto supply = [&](int i) {
    stage_k((i + 1) & 1);
    stage_v(i & 1);
    fetch_k(t0 + min(i + 2, Tc - 1));
    fetch_v(t0 + min(i + 1, Tc - 1));
  };
  auto scale_at = [&](const float *scale, int i) { return ldg(scale + blk0 + t0 + min(i, Tc - 1)); };

  if (Tc > 0) {
    stage_k(0);
    fetch_k(t0 + min(1, Tc - 1));
    __syncthreads();
    if (kPair) {
      // Two waves share a SIMD: while one multiplies and stages, the other
      // weighs.  The second half of the waves runs one phase behind.
      const bool first = w < NW / 2;
      float ks = scale_at(p.c.ks, 0), vs = scale_at(p.c.vs, 0);
      if (!first) __syncthreads();
      if (live) logits(tk[0]);
      supply(0);
      __syncthreads();
      for (int i = 1; i < Tc; ++i) {
        if (live) weights(i - 1, ks, vs);
        ks = scale_at(p.c.ks, i), vs = scale_at(p.c.vs, i);
        __syncthreads();
        if (live) products(i);
        supply(i);
        __syncthreads();
      }
      if (live) weights(Tc - 1, ks, vs);
      if (first) __syncthreads();
      if (live) outputs(tv[(Tc - 1) & 1]);
    } else {
      float ks = scale_at(p.c.ks, 0), vs = scale_at(p.c.vs, 0);
      if (live) {
        logits(tk[0]);
        weights(0, ks, vs);
      }
      supply(0);
      __syncthreads();
      for (int i = 1; i < Tc; ++i) {
        ks = scale_at(p.c.ks, i), vs = scale_at(p.c.vs, i);
        if (live) {
          products(i);
          weights(i, ks, vs);
        }
        supply(i);
        __syncthreads();
      }
      if (live) outputs(tv[(Tc - 1) & 1]);
    }
  }
  if (T > Tc) {  // the open block, by itself
    __syncthreads();  // the last values are read
    open_k(Tc & 1);
    open_v(Tc & 1);
    __syncthreads();
    if (live) {
      const float ks = ldg(p.c.ks + blk0 + nsealed), vs = ldg(p.c.vs + blk0 + nsealed);
      logits(tk[Tc & 1]);
      weights(Tc, ks, vs);
      open_outputs(tv[Tc & 1]);
    }
  }
  l = sum_halves(l);
  if (F32) l *= 16384.f;  // the factor that P's two parts carry
  // (Here, since a store before the loop would keep its scales out of scalar loads.)
  if (p.ns > 1 && sp == 0 && tid == 0)
    st8(reinterpret_cast<uint32_t *>(p.np) + 2 * (u * p.nqt + qt), u32x2{(uint32_t)sh.id, (uint32_t)ns});
  if (col > cl) return;
  if (ns == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = row_of(p.out, col);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 32 * cb + 8 * i + 4 * hf;
        const float a = O[cb][4 * i] * inv, bb = O[cb][4 * i + 1] * inv, cc = O[cb][4 * i + 2] * inv,
                    d = O[cb][4 * i + 3] * inv;
        if (p.fp32)
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

template <int D, int FMT, int NW>
void launch_nw(const Q8Attn &p, hipStream_t st) {
  const dim3 grid((uint32_t)p.wgs), block(64 * NW);
  if (p.fp32)
    hipLaunchKernelGGL((k_prompt8<D, FMT, NW, true>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((k_prompt8<D, FMT, NW, false>), grid, block, 0, st, p);
}

template <int D, int FMT>
hipError_t launch(const Q8Attn &p, hipStream_t st) {
  if (p.qcols == 256)
    launch_nw<D, FMT, 8>(p, st);
  else
    launch_nw<D, FMT, 4>(p, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.ns == 1) return e;
  return launch_q8_join(p, st);
}

}  // namespace

hipError_t launch_q8_prompt(const Q8Attn &p, int format, hipStream_t st) {
  if (p.d == 128) return format == kInt8 ? launch<128, kInt8>(p, st) : launch<128, kE4m3>(p, st);
  return format == kInt8 ? launch<64, kInt8>(p, st) : launch<64, kE4m3>(p, st);
}

}  // namespace vc
