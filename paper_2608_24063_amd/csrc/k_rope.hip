// k_rope.hip -- rotary positions with several axes: the pair (x1, x2) of
// frequency i turns by a = pos[axis(i)] f_i, so that a visual token's time,
// height and width each turn their own channels.  The angle is reduced in 64
// bits, as a number of turns (pos f_i / 2 pi less its nearest whole number):
// in 32 bits a position of 2^20 would leave 2^-4 of a turn unknown.  Sine and
// cosine of the reduced angle and the rotation itself are in 32 bits, rounded
// once to the output's type (fp32 rows at positions below 2^20 are 4.1e-8 of
// themselves off; 5.5e-8 without the angle's last bits).  The gradient of the
// rotation is the rotation by -a (the sign of the sine).
//
// Bound by memory: every value is read and written once, streamed.  12608 tokens
// of 28 + 4 bf16 heads take 35.8 us (5.8 TB/s), 8198 of 64 + 8 fp32 ones 103 (5.9).
// (Streaming: 43.4 -> 39.7 and 120 -> 112, with four tokens a workgroup.)  A token's d/2
// (sine, cosine) pairs serve all of its heads, so they are computed once per
// token and layer, one per thread, and shared through LDS; a lane then keeps
// the pairs of its own channels in registers while it walks the heads.
#include "vc_q8_device.h"

namespace vc {

namespace {

// 16 bytes of a row as floats, and back.
template <bool F32>
struct Chunk {
  static constexpr int N = F32 ? 4 : 8;
  static __device__ __forceinline__ void unpack(u32x4 w, float (&f)[N]) {
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (F32) {
        f[i] = __uint_as_float(ws[i]);
      } else {
        f[(2 * i) % N] = bf16_lo(ws[i]);
        f[(2 * i + 1) % N] = bf16_hi(ws[i]);
      }
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&f)[N]) {
    if (F32)
      return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    return u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2 % N], f[3 % N]), pack_bf16(f[4 % N], f[5 % N]),
                 pack_bf16(f[6 % N], f[7 % N])};
  }
};

// A workgroup takes TPW tokens of one layer, each with 4 / TPW waves.
template <bool F32, bool ADJ, int TPW>
__global__ __launch_bounds__(256) void k_rope(RopePlan p) {
  using C = Chunk<F32>;
  constexpr int N = C::N;
  constexpr int kWaves = 4 / TPW;  // waves per token
  __shared__ float2 cs[TPW][kRopeMaxHalf];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t toks = (int64_t)p.B * p.n;
  const int64_t groups = (toks + TPW - 1) / TPW;
  const int64_t bid = blockIdx.x;
  const int l = (int)(bid / groups);
  const int64_t g0 = bid % groups * TPW;
  const int half = p.t.rot / 2;
  // (sine, cosine) of token g0 + t, frequency i.
  for (int e = tid; e < TPW * kRopeMaxHalf; e += 256) {
    const int t = e / kRopeMaxHalf, i = e % kRopeMaxHalf;
    const int64_t g = g0 + t;
    if (i < half && g < toks) {
      cs[t][i] = turn_of(p.t, i, ldg(p.pos + axis_of(p.t, i) * toks + g));
    }
  }
  __syncthreads();
  const int t = w / kWaves, sub = w % kWaves;
  const int64_t g = g0 + t;
  if (g >= toks) return;
  const int b = (int)(g / p.n), i = (int)(g % p.n);
  if (p.count && i >= ldg(p.count + b)) return;
  // Lane: chunk pair c of head h.  Halves: channels [Nc, Nc+N) and the same
  // past rot/2; adjacent: 2N channels in a row.  Lanes past the rotated
  // channels copy the rest.
  const int per = p.d / (2 * N);    // chunk pairs per row (a power of two)
  const int rper = p.t.rot / (2 * N);  // rotated ones
  const int c = lane % per, hl = lane / per, hs = 64 / per;
  const bool rotated = c < rper;
  const int o1 = rotated ? (ADJ ? 2 * N * c : N * c) : 2 * N * c;
  const int o2 = rotated ? (ADJ ? 2 * N * c + N : half + N * c) : 2 * N * c + N;
  float2 w2[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    // Frequencies of this lane: N of them, for the halves Nc + k, for
    // adjacent pairs Nc + k as well (2N channels hold N pairs).
    w2[k] = rotated ? cs[t][N * c + k] : make_float2(1.f, 0.f);
  }
  // Rows of this token by head; the descriptors' products once, not in the loop.
  const int H = p.Hq + p.Hkv;
  constexpr int64_t E = F32 ? 4 : 2;
  auto row0 = [&](const RowsDesc &r) { return r.base + E * (l * r.layer + b * r.seq + i * r.token); };
  const uint64_t qi = row0(p.qi), qo = row0(p.qo), ki = row0(p.ki), ko = row0(p.ko);
  const int64_t qih = E * p.qi.head, qoh = E * p.qo.head, kih = E * p.ki.head, koh = E * p.ko.head;
  for (int h = sub * hs + hl; h < H; h += kWaves * hs) {
    const bool isq = h < p.Hq;
    const int hh = isq ? h : h - p.Hq;
    const char *src = reinterpret_cast<const char *>((isq ? qi : ki) + hh * (isq ? qih : kih));
    char *dst = reinterpret_cast<char *>((isq ? qo : ko) + hh * (isq ? qoh : koh));
    float x[N], y[N];
    C::unpack(ld16_stream(src + E * o1), x);
    C::unpack(ld16_stream(src + E * o2), y);
    if (rotated) {
      if (ADJ) {
        // Pairs (2m, 2m+1): N/2 of them in x, N/2 in y.
#pragma unroll
        for (int m = 0; m < N / 2; ++m) {
          turn(x[2 * m], x[2 * m + 1], w2[m]);
          turn(y[2 * m], y[2 * m + 1], w2[N / 2 + m]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) turn(x[k], y[k], w2[k]);
      }
    }
    st16_stream(dst + E * o1, C::pack(x));
    st16_stream(dst + E * o2, C::pack(y));
  }
}

template <bool F32, bool ADJ>
hipError_t launch(const RopePlan &p, hipStream_t st) {
  const int64_t toks = (int64_t)p.B * p.n;
  // A wave's pass takes as many heads as chunk pairs of a row leave lanes for.  Four
  // tokens a workgroup, a wave each, where that is two passes of a wave or fewer and
  // the tokens fill the chip; else a token a workgroup.  (us, one token and four:
  // bf16, 128 channels, 32000 tokens of 2, 10, 16, 32 heads 41.3 20.2, 54.0 29.9, 57.0
  // 45.0, 83.8 92.7; 2000 of 16 and 32 6.8 6.1, 8.8 9.2; 500 of 2 and 16 4.8 4.9, 4.3 4.9.
  // fp32, 128 channels, 32000 of 8, 16, 32 heads 56.0 43.9, 83.7 87.3, 169 191; bf16, 64
  // channels, 16 and 32 heads 45.0 28.7, 58.5 57.4.)
  const int lanes = p.d / (2 * Chunk<F32>::N), heads = 64 / lanes;  // lanes of a row, heads of a pass
  if (p.Hq + p.Hkv <= 2 * heads && toks * p.L >= 2048) {
    const int64_t grid = (toks + 3) / 4 * p.L;
    hipLaunchKernelGGL((k_rope<F32, ADJ, 4>), dim3((uint32_t)grid), dim3(256), 0, st, p);
  } else {
    hipLaunchKernelGGL((k_rope<F32, ADJ, 1>), dim3((uint32_t)(toks * p.L)), dim3(256), 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopePlan &p, hipStream_t st) {
  if (p.fp32) return p.t.adjacent ? launch<true, true>(p, st) : launch<true, false>(p, st);
  return p.t.adjacent ? launch<false, true>(p, st) : launch<false, false>(p, st);
}

}  // namespace vc
