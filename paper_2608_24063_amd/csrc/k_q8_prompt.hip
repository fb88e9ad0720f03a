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
// exceeds the range of fp16.  p' is one fp16 value (2^-12 relative, against the
// output's 2^-9).  With fp32 outputs P is split in two fp16 parts and each
// block's product is scaled into O in fp32.
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

__device__ __forceinline__ f16x8 half8_of_bf16(u32x4 w, float f) {
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
  f16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = (_Float16)(bf16_lo(ws[i]) * f);
    r[2 * i + 1] = (_Float16)(bf16_hi(ws[i]) * f);
  }
  return r;
}

template <int D>
struct Tile {
  static constexpr int KP = D + 8;           // pitches in halves: 16-byte reads of 32 rows without conflicts
  static constexpr int VP = kQ8Block + 8;
  _Float16 k[kQ8Block][KP];
  _Float16 v[D][VP];
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
  __shared__ Tile<D> tile[2] __attribute__((aligned(16)));
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ln = lane & 31, hf = lane >> 5;
  // Workgroups of a unit follow each other on one XCD and share its L2.
  const uint32_t id = xcd_block(blockIdx.x, gridDim.x);
  const int per = p.nqt * p.ns;
  const int u = (int)(id / (uint32_t)per), rest = (int)(id % (uint32_t)per);
  const int qt = rest / p.ns, sp = rest % p.ns;
  const int b = u / p.Hkv % p.B;
  const int len = max(min(ldg(p.c.len + u), ldg(p.c.cap + u)), 0);
  const int cnt = p.count ? min(max(ldg(p.count + b), 0), p.n) : p.n;
  const int cols = cnt * p.G;
  const int c0 = qt * p.qcols;
  if (c0 >= cols) return;
  const int cl = min(c0 + p.qcols, cols) - 1;  // last column of the workgroup
  const int lim = p.causal ? len - cnt + 1 : len;
  auto rows_seen = [&](int col) { return max(min(p.causal ? lim + col / p.G : len, p.max_rows), 0); };
  const int emax = rows_seen(cl);
  const int nt = (emax + kQ8Block - 1) / kQ8Block;
  const int t0 = (int)((int64_t)sp * nt / p.ns), t1 = (int)((int64_t)(sp + 1) * nt / p.ns);
  const int col = c0 + 32 * w + ln;
  const int end = rows_seen(min(col, cl));
  const int wmin = rows_seen(min(c0 + 32 * w, cl));  // fewest rows a column of the wave sees
  const bool live = c0 + 32 * w <= cl;  // the wave has columns (the others only stage)
  const int64_t blk0 = ldg(p.c.row_off + u) / kQ8Block;
  const int nsealed = len / kQ8Block;
  const int g = u % p.Hkv, lb = u / p.Hkv;
  auto row_of = [&](const RowsDesc &r, int cc) {
    return (int64_t)(lb / p.B) * r.layer + (int64_t)(lb % p.B) * r.seq + (int64_t)(cc / p.G) * r.token +
           (int64_t)(g * p.G + cc % p.G) * r.head;
  };

  f16x8 q[KS];
  float cq;
  {
    const uint16_t *qp = reinterpret_cast<const uint16_t *>(p.q.base) + row_of(p.q, min(col, cl));
    u32x4 x[KS];
    uint32_t mag = 0u;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      x[s] = ld16(qp + 16 * s + 8 * hf);
      mag = max_mag(max_mag(max_mag(max_mag(mag, x[s].x), x[s].y), x[s].z), x[s].w);
    }
    uint32_t mm = max(mag & 0xFFFFu, mag >> 16);
    mm = max(mm, (uint32_t)__shfl_xor((int)mm, 32, 64));
    const float qs = open_scale(mm);
    cq = p.sc * qs;
    const float inv = 1.f / qs;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = half8_of_bf16(x[s], inv);
  }

  u32x4 rk[IT], rv[IT];
  auto fetch = [&](int t) {
    const uint8_t *k = p.c.kc + (blk0 + t) * (kQ8Block * D), *v = p.c.vc + (blk0 + t) * (kQ8Block * D);
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = kPart ? min(tid, kItems - 1) : tid + NT * it;
      rk[it] = ld16(k + 16 * e);
      rv[it] = ld16(v + 16 * e);
    }
  };
  auto stage = [&](int buf) {
    if (kPart && tid >= kItems) return;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int e = tid + NT * it;
      const int row = place(e / (D / 16)), c = e % (D / 16);
      _Float16 *kd = &tile[buf].k[row][16 * c];
      *reinterpret_cast<f16x8 *>(kd) = Q8<FMT>::half8(rk[it].x, rk[it].y);
      *reinterpret_cast<f16x8 *>(kd + 8) = Q8<FMT>::half8(rk[it].z, rk[it].w);
      _Float16 *vd = &tile[buf].v[e / 4][16 * (e % 4)];
      *reinterpret_cast<f16x8 *>(vd) = Q8<FMT>::half8(rv[it].x, rv[it].y);
      *reinterpret_cast<f16x8 *>(vd + 8) = Q8<FMT>::half8(rv[it].z, rv[it].w);
    }
  };
  // The open block: bf16 rows scaled by their powers of two, zeros past its end.
  auto stage_open = [&](int buf) {
    const int rows = len - nsealed * kQ8Block;
    const uint16_t *kt = p.c.kt + (int64_t)u * kQ8Block * D, *vt = p.c.vt + (int64_t)u * kQ8Block * D;
    const float kinv = 1.f / ldg(p.c.ks + blk0 + nsealed), vinv = 1.f / ldg(p.c.vs + blk0 + nsealed);
    for (int e = tid; e < kQ8Block * D / 8; e += NT) {
      const int row = e / (D / 8), c = e % (D / 8);
      const bool in = row < rows;
      const u32x4 zero = {0u, 0u, 0u, 0u};
      *reinterpret_cast<f16x8 *>(&tile[buf].k[place(row)][8 * c]) =
          half8_of_bf16(in ? ld16(kt + row * D + 8 * c) : zero, kinv);
      const f16x8 v = half8_of_bf16(in ? ld16(vt + row * D + 8 * c) : zero, vinv);
#pragma unroll
      for (int k = 0; k < 8; ++k) tile[buf].v[8 * c + k][row] = v[k];
    }
  };

  f32x16 O[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[cb][i] = 0.f;
  float m = kNegInf, l = 0.f;

  // Block t, staged in T, into the wave's state.
  auto absorb = [&](int t, const Tile<D> &T) {
    const float ks = ldg(p.c.ks + blk0 + t), vs = ldg(p.c.vs + blk0 + t);
    f32x16 S[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) S[kb][i] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s)
        S[kb] = mfma32(*reinterpret_cast<const f16x8 *>(&T.k[32 * kb + ln][16 * s + 8 * hf]), q[s], S[kb]);
    }
    const float c = fmaxf(cq * ks, 1e-37f);
    if ((t + 1) * kQ8Block > wmin) {  // wave-uniform
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = t * kQ8Block + 32 * kb + 16 * (i >> 3) + 8 * hf + 4 * ((i >> 2) & 1) + (i & 3);
          if (row >= end) S[kb][i] = kNegInf;
        }
    }
    float mx = fmaxf(S[0][0], S[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, fmaxf(S[0][i], S[1][i]));
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
    f16x8 hi[4], lo[4];
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float pr = fast_exp2(fmaf(S[kb][i], c, off));
        sum += pr;
        if (F32) {
          const float ps = pr * 16384.f;
          const _Float16 h = (_Float16)ps;
          hi[2 * kb + i / 8][i % 8] = h;
          lo[2 * kb + i / 8][i % 8] = (_Float16)(ps - (float)h);
        } else {
          hi[2 * kb + i / 8][i % 8] = (_Float16)pr;
        }
      }
    l = F32 ? l + sum : fmaf(sum, __builtin_amdgcn_rcpf(vs), l);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      f32x16 acc;
      if (F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
      } else {
        acc = O[cb];
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const f16x8 v = *reinterpret_cast<const f16x8 *>(&T.v[32 * cb + ln][16 * s + 8 * hf]);
        acc = mfma32(v, hi[s], acc);
        if (F32) acc = mfma32(v, lo[s], acc);
      }
      if (F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) O[cb][i] = fmaf(acc[i], vs, O[cb][i]);
      } else {
        O[cb] = acc;
      }
    }
  };

  if (t0 < t1) {
    if (t0 < nsealed) {
      fetch(t0);
      stage(0);
    } else {
      stage_open(0);
    }
  }
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    const bool more = t + 1 < t1, code = t + 1 < nsealed;
    if (more && code) fetch(t + 1);
    if (live) absorb(t, tile[buf]);
    if (more) {
      if (code)
        stage(buf ^ 1);
      else
        stage_open(buf ^ 1);
    }
    __syncthreads();
  }
  l = sum_halves(l);
  if (F32) l *= 16384.f;  // the factor that P's two parts carry
  if (col > cl) return;
  if (p.ns == 1) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
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
  const int64_t slot = ((int64_t)u * p.nqt + qt) * p.ns + sp;
  const int64_t at = slot * p.qcols + 32 * w + ln;
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
  const dim3 grid((uint32_t)((int64_t)p.units * p.nqt * p.ns)), block(64 * NW);
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
