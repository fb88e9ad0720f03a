// k_norm_rope.hip -- norm of each query and key head, its weight and the rotation
// by positions in one pass, and the gradient of all three:
//   r = (mean x^2 + eps)^-1/2,  y = w x r,  out = R y,
//   g = R^T dout,  n = x r,  dx = r (w g - n mean(w g n)),  dw = sum g n
// over a layer's tokens and heads.  R is the rotation of k_rope.hip (its angles in 64
// bits); all else is fp32, rounded once to the rows' type.  d is a power of two, so
// the means are exact products.
//
// Bound by memory: every value is read and written once, streamed.  A row lies over d /
// (2N) lanes (N values in 16 bytes), which exchange its sums by DPP.  A wave's first rows
// are requested before the weights and the positions that it turns them by.  12608
// tokens of 28 + 4 bf16 heads, 128 channels: 39 us (5.2 TB/s); the gradient over 16382
// tokens of 64 + 8: 176 to 187 us (4.8 to 5.1 TB/s), 5 of them the sum of the weights'.
#include "vc_norm.h"
#include "vc_q8_device.h"

namespace vc {

namespace {

// A lane's place in the rows: chunks at elements o1 and o2, frequencies N c ...
template <bool F32, bool ADJ, int D>
struct Place {
  using C = Chunk<F32>;
  static constexpr int N = C::N, PER = D / (2 * N), HS = 64 / PER;  // lanes of a row, rows of a wave
  int c, o1, o2;
  bool rotated;
  __device__ __forceinline__ Place(int lane, int rot) {
    c = lane % PER;
    rotated = c < rot / (2 * N);
    o1 = rotated && !ADJ ? N * c : 2 * N * c;
    o2 = rotated && !ADJ ? rot / 2 + N * c : 2 * N * c + N;
  }
  // The weights of the lane's channels.
  __device__ __forceinline__ void weights(const void *w, int l, int w_fp32, float (&f)[2 * N]) const {
    if (!w) {
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) f[i] = 0.f;
      return;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = l * D + (h ? o2 : o1);
      if (w_fp32) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const u32x4 v = ld16(static_cast<const float *>(w) + at + i);
          f[h * N + i] = __uint_as_float(v.x);
          f[h * N + i + 1] = __uint_as_float(v.y);
          f[h * N + i + 2] = __uint_as_float(v.z);
          f[h * N + i + 3] = __uint_as_float(v.w);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const u32x2 v = ld8(static_cast<const uint16_t *>(w) + at + i);
          f[h * N + i] = bf16_lo(v.x);
          f[h * N + i + 1] = bf16_hi(v.x);
          f[h * N + i + 2] = bf16_lo(v.y);
          f[h * N + i + 3] = bf16_hi(v.y);
        }
      }
    }
  }
  static __device__ __forceinline__ void unpack(u32x4 a, u32x4 b, float (&f)[2 * N]) {
    float x[N], y[N];
    C::unpack(a, x);
    C::unpack(b, y);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = x[i], f[N + i] = y[i];
  }
  __device__ __forceinline__ void rotate(float (&f)[2 * N], const float2 (&w)[N]) const {
    if (!rotated) return;
    if (ADJ) {
#pragma unroll
      for (int m = 0; m < N; ++m) turn(f[2 * m], f[2 * m + 1], w[m]);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) turn(f[k], f[N + k], w[k]);
    }
  }
  // Rounded to the rows' type, the only rounding to fewer bits.
  __device__ __forceinline__ void store(char *row, const float (&f)[2 * N]) const {
    float x[N], y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = f[i], y[i] = f[N + i];
    st16_stream(row + sizeof(uint32_t) / (F32 ? 1 : 2) * o1, C::pack(x));
    st16_stream(row + sizeof(uint32_t) / (F32 ? 1 : 2) * o2, C::pack(y));
  }
  static __device__ __forceinline__ float squares(const float (&f)[2 * N]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) s = fmaf(f[i], f[i], s);
    return sum_lanes<PER>(s);
  }
};

// (mean + eps)^-1/2 of a sum of squares, within 1.5 steps of fp32.  (A step of Newton's brings
// fp32 outputs no nearer to 64 bits: a norm of 6.2e-8 without it, 6.4e-8 with it.)
template <int D>
__device__ __forceinline__ float inv_rms(float sum, float eps) {
  return __builtin_amdgcn_rsqf(fmaf(sum, 1.f / D, eps));
}

// A workgroup takes TPW tokens of one layer, each with 4 / TPW waves.
template <bool F32, bool ADJ, int D, int TPW>
__global__ __launch_bounds__(256) void k_norm_rope(NormPlan p) {
  using Pl = Place<F32, ADJ, D>;
  constexpr int N = Pl::N, HS = Pl::HS, kWaves = 4 / TPW;
  __shared__ float2 cs[TPW][kRopeMaxHalf];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t toks = (int64_t)p.B * p.n;
  const int64_t groups = (toks + TPW - 1) / TPW;
  const int64_t bid = blockIdx.x;
  const int l = (int)(bid / groups);
  const int64_t g0 = bid % groups * TPW;
  const int half = p.t.rot / 2;
  const Pl pl(lane, p.t.rot);
  const int t = w / kWaves, sub = w % kWaves;
  const int64_t g = g0 + t, gc = g < toks ? g : toks - 1;
  const int b = (int)(gc / p.n), i = (int)(gc % p.n);
  const int H = p.Hq + p.Hkv;
  constexpr int64_t E = F32 ? 4 : 2;
  auto row0 = [&](const RowsDesc &r) { return r.base + E * (l * r.layer + b * r.seq + i * r.token); };
  const uint64_t qi = row0(p.qi), qo = row0(p.qo), ki = row0(p.ki), ko = row0(p.ko);
  const int64_t qih = E * p.qi.head, qoh = E * p.qo.head, kih = E * p.ki.head, koh = E * p.ko.head;
  u32x4 x0, x1;
  auto request = [&](int h) {
    const bool isq = h < p.Hq;
    const int hh = isq ? h : h - p.Hq;
    const char *src = reinterpret_cast<const char *>((isq ? qi : ki) + hh * (isq ? qih : kih));
    x0 = ld16_stream(src + E * pl.o1);
    x1 = ld16_stream(src + E * pl.o2);
  };
  // The first rows' requests, the weights' and the positions', before anything waits.
  const int h0 = sub * HS + lane / Pl::PER;
  request(min(h0, H - 1));
  float wq[2 * N], wk[2 * N];
  pl.weights(p.qw, l, p.w_fp32, wq);
  pl.weights(p.kw, l, p.w_fp32, wk);
  for (int e = tid; e < TPW * kRopeMaxHalf; e += 256) {
    const int tt = e / kRopeMaxHalf, f = e % kRopeMaxHalf;
    const int64_t gg = g0 + tt;
    if (f < half && gg < toks) cs[tt][f] = turn_of(p.t, f, ldg(p.pos + axis_of(p.t, f) * toks + gg));
  }
  __syncthreads();
  if (g >= toks) return;
  if (p.count && i >= ldg(p.count + b)) return;
  float2 w2[N];
#pragma unroll
  for (int k = 0; k < N; ++k) w2[k] = pl.rotated ? cs[t][N * pl.c + k] : make_float2(1.f, 0.f);
  for (int h = h0; h < H; h += kWaves * HS) {
    const bool isq = h < p.Hq;
    const int hh = isq ? h : h - p.Hq;
    char *dst = reinterpret_cast<char *>((isq ? qo : ko) + hh * (isq ? qoh : koh));
    float x[2 * N];
    Pl::unpack(x0, x1, x);
    request(min(h + kWaves * HS, H - 1));  // the next rows', which no output overlaps
    const float r = inv_rms<D>(Pl::squares(x), p.eps);
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) x[k] = x[k] * r * (isq ? wq[k] : wk[k]);
    pl.rotate(x, w2);
    pl.store(dst, x);
  }
}

// The gradient.  A wave takes every (4 groups)-th token of its layer, one at a time, the
// queries and then the keys, and keeps its lanes' sums for dw, which go to the wave's in LDS,
// in 64 bits, when they have kSum terms (thousands added one after another in fp32 would be
// off by 1e-4 where they are alike); the workgroup's sums go to `part`, and k_dweight adds
// those up in a fixed order.
constexpr int kSum = 256;
template <bool F32, bool ADJ, int D>
__global__ __launch_bounds__(256) void k_norm_rope_grad(NormPlan p) {
  using Pl = Place<F32, ADJ, D>;
  constexpr int N = Pl::N, HS = Pl::HS, PER = Pl::PER;
  constexpr int64_t E = F32 ? 4 : 2;
  __shared__ float2 cs[4][kRopeMaxHalf];
  __shared__ double sums[4][2][D];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t toks = (int64_t)p.B * p.n;
  const int l = (int)(blockIdx.x / (uint32_t)p.groups), grp = (int)(blockIdx.x % (uint32_t)p.groups);
  const int half = p.t.rot / 2;
  const Pl pl(lane, p.t.rot);
  float ws[2][2 * N], dw[2][2 * N];
  pl.weights(p.qw, l, p.w_fp32, ws[0]);
  pl.weights(p.kw, l, p.w_fp32, ws[1]);
#pragma unroll
  for (int k = 0; k < 2 * N; ++k) dw[0][k] = dw[1][k] = 0.f;
  for (int e = lane; e < 2 * D; e += 64) (&sums[w][0][0])[e] = 0.0;
  // A side's terms since its lanes' sums, over the lanes of the same channels, went to LDS.
  int terms[2] = {0, 0};
  auto close = [&](int s) {
    terms[s] = 0;
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) {
      float v = dw[s][k];
#pragma unroll
      for (int m = PER; m < 64; m *= 2) v += shfl_xor(v, m);
      if (lane < PER) sums[w][s][(k < N ? pl.o1 : pl.o2 - N) + k] += (double)v;
      dw[s][k] = 0.f;
    }
  };
  for (int64_t g = (int64_t)grp * 4 + w; g < toks; g += 4 * (int64_t)p.groups) {
    const int b = (int)(g / p.n), i = (int)(g % p.n);
    if (p.count && i >= ldg(p.count + b)) continue;  // wave-uniform
    if (lane < half) cs[w][lane] = turn_of(p.t, lane, ldg(p.pos + axis_of(p.t, lane) * toks + g));
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the wave's own table is written
    __builtin_amdgcn_wave_barrier();
    float2 w2[N];
#pragma unroll
    for (int k = 0; k < N; ++k) w2[k] = pl.rotated ? cs[w][N * pl.c + k] : make_float2(1.f, 0.f);
    auto side = [&](int H, const RowsDesc &xi, const RowsDesc &gi, const RowsDesc &xo, const float (&wt)[2 * N],
                    float (&acc)[2 * N]) {
      auto row0 = [&](const RowsDesc &r) { return r.base + E * (l * r.layer + b * r.seq + i * r.token); };
      const uint64_t xb = row0(xi), gb = row0(gi), ob = row0(xo);
      for (int h = lane / PER; h < H; h += HS) {
        const char *xs = reinterpret_cast<const char *>(xb + E * h * xi.head);
        const char *gs = reinterpret_cast<const char *>(gb + E * h * gi.head);
        float x[2 * N], q[2 * N];
        const u32x4 a0 = ld16_stream(xs + E * pl.o1), a1 = ld16_stream(xs + E * pl.o2);
        const u32x4 b0 = ld16_stream(gs + E * pl.o1), b1 = ld16_stream(gs + E * pl.o2);
        Pl::unpack(a0, a1, x);
        Pl::unpack(b0, b1, q);
        pl.rotate(q, w2);
        const float r = inv_rms<D>(Pl::squares(x), p.eps);
        float dot = 0.f;
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) {
          x[k] *= r;                           // n
          acc[k] = fmaf(q[k], x[k], acc[k]);   // g n
          q[k] *= wt[k];                       // w g
          dot = fmaf(q[k], x[k], dot);
        }
        const float m = sum_lanes<PER>(dot) * (1.f / D);
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) q[k] = r * fmaf(-x[k], m, q[k]);
        pl.store(reinterpret_cast<char *>(ob + E * h * xo.head), q);
      }
    };
    side(p.Hq, p.qi, p.qg, p.qo, ws[0], dw[0]);
    side(p.Hkv, p.ki, p.kg, p.ko, ws[1], dw[1]);
    __builtin_amdgcn_wave_barrier();
    if ((terms[0] += (p.Hq + HS - 1) / HS) >= kSum) close(0);
    if ((terms[1] += (p.Hkv + HS - 1) / HS) >= kSum) close(1);
  }
  close(0);
  close(1);
  __syncthreads();
  float *to = p.part + (int64_t)blockIdx.x * 2 * D;
  for (int e = tid; e < 2 * D; e += 256) {
    const double *f = &sums[0][0][0] + e;
    stg(to + e, (float)((f[0] + f[2 * D]) + (f[4 * D] + f[6 * D])));
  }
}

// dw of 16 channels of one layer and side: 64 threads a channel add up the groups' sums, in
// 64 bits.
template <int D>
__global__ __launch_bounds__(1024) void k_dweight(NormPlan p) {
  __shared__ double red[64][17];
  const int tid = threadIdx.x, ch = tid % 16, j0 = tid / 16;
  constexpr int CG = D / 16;
  const int cg = (int)(blockIdx.x % CG), s = (int)(blockIdx.x / CG % 2), l = (int)(blockIdx.x / (2 * CG));
  float *out = s ? p.dkw : p.dqw;
  if (!out) return;  // (uniform)
  const float *from = p.part + (int64_t)l * p.groups * 2 * D + s * D + cg * 16 + ch;
  double v = 0.0;
#pragma unroll 8
  for (int j = j0; j < p.groups; j += 64) v += (double)ldg(from + (int64_t)j * 2 * D);
  red[j0][ch] = v;
  __syncthreads();
  for (int m = 32; m >= 1; m /= 2) {
    if (j0 < m) red[j0][ch] += red[j0 + m][ch];
    __syncthreads();
  }
  if (j0 == 0) stg(out + l * D + cg * 16 + ch, (float)red[0][ch]);
}

template <bool F32, bool ADJ, int D>
hipError_t launch(const NormPlan &p, bool grad, hipStream_t st) {
  const int64_t toks = (int64_t)p.B * p.n;
  if (grad) {
    hipLaunchKernelGGL((k_norm_rope_grad<F32, ADJ, D>), dim3((uint32_t)(p.groups * p.L)), dim3(256), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_dweight<D>), dim3((uint32_t)(p.L * 2 * (D / 16))), dim3(1024), 0, st, p);
    return hipGetLastError();
  }
  // Four tokens a workgroup, a wave each, where a wave then has few passes over a token's
  // heads and the tokens fill the chip; else a token a workgroup.  (us, one token and four:
  // bf16, 128 channels, 10 heads, 1024, 2048, 32000 tokens 4.8 4.5, 7.6 5.4, 87 41; 32 heads
  // (4 passes) 5.9 6.9, 9.8 9.3, 114 90; 72 heads (9) 9.3 11.4, 15.9 16.1, 193 199.  bf16, 64
  // channels, 72 heads (5) 6.9 7.7, 12.2 11.0, 140 116.  fp32, 128 channels, 10 heads (3) 4.8
  // 4.6, 6.9 5.6, 69 55, 32 heads (8) 172 189; 64 channels, 32 heads (4) 8.6 8.4, 85 91.)
  constexpr int HS = Place<F32, ADJ, D>::HS;
  if ((p.Hq + p.Hkv + HS - 1) / HS <= (F32 ? 3 : 5) && toks * p.L >= 2048)
    hipLaunchKernelGGL((k_norm_rope<F32, ADJ, D, 4>), dim3((uint32_t)((toks + 3) / 4 * p.L)), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((k_norm_rope<F32, ADJ, D, 1>), dim3((uint32_t)(toks * p.L)), dim3(256), 0, st, p);
  return hipGetLastError();
}

template <bool F32, bool ADJ>
hipError_t launch(const NormPlan &p, bool grad, hipStream_t st) {
  return p.d == 128 ? launch<F32, ADJ, 128>(p, grad, st) : launch<F32, ADJ, 64>(p, grad, st);
}

hipError_t launch(const NormPlan &p, bool grad, hipStream_t st) {
  if (p.fp32) return p.t.adjacent ? launch<true, true>(p, grad, st) : launch<true, false>(p, grad, st);
  return p.t.adjacent ? launch<false, true>(p, grad, st) : launch<false, false>(p, grad, st);
}

}  // namespace

hipError_t launch_norm_rope(const NormPlan &p, hipStream_t st) { return launch(p, false, st); }
hipError_t launch_norm_rope_grad(const NormPlan &p, hipStream_t st) { return launch(p, true, st); }

}  // namespace vc
