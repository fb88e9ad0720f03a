// vc_q8_device.h -- the 8-bit types of the cache on gfx950: rounding to them,
// and their values as fp32 and fp16 (int8 and e4m3 codes are exact in both).
// Internal to libviscache.
#pragma once
#include "vc_device.h"
#include "vc_q8.h"

namespace vc {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

enum { kInt8 = 0, kE4m3 = 1 };

template <int FMT>
struct Q8 {
  static constexpr float kTop = FMT == kInt8 ? 127.f : 448.f;
  static constexpr float kEffMin = kTop * 0x1p-60f, kEffMax = kTop * 0x1p60f;

  // Q x / eff to 20 significant bits, clamped.  x and eff are bf16 values (or
  // eff a bound that makes inv a power of two), so the exact quotient is
  // either a midpoint of two codes (at most 8 significant bits) or at least
  // 2^-17 of itself away from every midpoint: for int8 |254 X 2^i - M A 2^j| >=
  // 1 with X, A < 2^8 and M odd <= 253, for e4m3 |7 X 2^i - M A 2^j| >= 1 with
  // M <= 31.  The product with the rounded inverse is off by less than 2^-22
  // of itself; cutting it to 20 bits puts midpoints back where they are and
  // moves nothing across one, so ties go to even without a division per value.
  static __device__ __forceinline__ float code_value(float x, float inv) {
    const float y = __uint_as_float((__float_as_uint(x * inv) + 8u) & ~15u);
    return __builtin_amdgcn_fmed3f(y, -kTop, kTop);
  }
  // Codes of four values, the first in the low byte.
  static __device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    if (FMT == kInt8) {
      // The sum with 1.5 * 2^23 rounds to a whole number, ties to even, and
      // holds it in its low byte.
      const uint32_t ia = __float_as_uint(a + 12582912.f), ib = __float_as_uint(b + 12582912.f);
      const uint32_t ic = __float_as_uint(c + 12582912.f), id = __float_as_uint(d + 12582912.f);
      const uint32_t lo = __builtin_amdgcn_perm(ib, ia, 0x0c0c0400u), hi = __builtin_amdgcn_perm(id, ic, 0x04000c0cu);
      return lo | hi;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  }
  // The four codes of a word as fp32.
  static __device__ __forceinline__ void unpack4(uint32_t w, float (&f)[4]) {
    if (FMT == kInt8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = (float)(int)(int8_t)(w >> (8 * i));
      return;
    }
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = a[0];
    f[1] = a[1];
    f[2] = b[0];
    f[3] = b[1];
  }
  // The four codes of a word as fp16: e4m3 by the converting instruction;
  // int8, moved to 0..255, as the low bits of 1024 + u, less 1152.
  static __device__ __forceinline__ u32x2 half4(uint32_t w) {
    f16x2 a, b;
    if (FMT == kInt8) {
      const uint32_t u = w ^ 0x80808080u;
      const f16x2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
      a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
      b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
    } else {
      a = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, false));
      b = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, true));
    }
    return u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
  }
  static __device__ __forceinline__ f16x8 half8(uint32_t w0, uint32_t w1) {
    const u32x2 a = half4(w0), b = half4(w1);
    return __builtin_bit_cast(f16x8, u32x4{a.x, a.y, b.x, b.y});
  }
};

// Accesses that ask the caches not to keep what passes through once and in bulk.
template <typename T>
__device__ __forceinline__ void st16_stream(T *p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<VC_GLOBAL u32x4 *>(gp(p)));
}
template <typename T>
__device__ __forceinline__ u32x4 ld16_stream(const T *p) {
  return __builtin_nontemporal_load(reinterpret_cast<const VC_GLOBAL u32x4 *>(gp(p)));
}

// Largest magnitude of packed bf16 pairs, as bf16 bits (unsigned compare of
// the bits without the sign).
__device__ __forceinline__ uint32_t max_mag(uint32_t m, uint32_t w) {
  const u16x2 a = __builtin_bit_cast(u16x2, m), b = __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a, b));
}

// The power of two that puts a largest magnitude (bf16 bits) into [2^14,
// 2^15), at least 2^-60: with it a row's bf16 values are exact in fp16 down to
// 2^-31 of the largest.
__device__ __forceinline__ float open_scale(uint32_t mag) {
  const int e = max((int)(mag >> 7) - 14, 127 - 60);
  return __uint_as_float((uint32_t)e << 23);
}

// Eight bf16 values times a power of two, as fp16.
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

// 4 x 4 bytes transposed: byte j of word i becomes byte i of word j.
__device__ __forceinline__ u32x4 transpose4(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
  const uint32_t t0 = __builtin_amdgcn_perm(w1, w0, 0x05010400u), t1 = __builtin_amdgcn_perm(w3, w2, 0x05010400u);
  const uint32_t t2 = __builtin_amdgcn_perm(w1, w0, 0x07030602u), t3 = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
  return u32x4{__builtin_amdgcn_perm(t1, t0, 0x05040100u), __builtin_amdgcn_perm(t1, t0, 0x07060302u),
               __builtin_amdgcn_perm(t3, t2, 0x05040100u), __builtin_amdgcn_perm(t3, t2, 0x07060302u)};
}

// The pair (x1, x2) turned: cs = scale (cos a, sin a).
__device__ __forceinline__ void turn(float &x1, float &x2, float2 cs) {
  const float a = x1, b = x2;
  x1 = fmaf(a, cs.x, -(b * cs.y));
  x2 = fmaf(b, cs.x, a * cs.y);
}
// scale (cos, sin) of the angle of a position: reduced in 64 bits as a number
// of turns, then 32; what that rounding leaves of the angle (e, below 2^-23)
// turns the result.
__device__ __forceinline__ float2 turn_of(const RopeTable &t, int i, int pos) {
  double a = (double)pos * t.turns[i];
  a -= rint(a);
  const float h = (float)a, e = 6.2831853f * (float)(a - h);
  float s, c;
  sincospif(2.f * h, &s, &c);
  return make_float2(fmaf(-s, e, c) * t.scale, fmaf(c, e, s) * t.scale * t.sgn);
}
// The axis of frequency i.
__device__ __forceinline__ int axis_of(const RopeTable &t, int i) {
  return (int)(t.axis1 >> i & 1) + 2 * (int)(t.axis2 >> i & 1);
}

// Largest over 256 threads (waves of one half of `red`) of per-thread packed
// magnitudes; one barrier of the whole workgroup (the next use of `red` must
// come after another one).
__device__ __forceinline__ uint32_t max_of_256(uint32_t (&red)[4], uint32_t m, int tid) {
  uint32_t x = max(m & 0xFFFFu, m >> 16);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, k, 64));
  if ((tid & 63) == 0) red[tid >> 6] = x;
  __syncthreads();
  return max(max(red[0], red[1]), max(red[2], red[3]));
}

// Quantises a block of 64 rows with 256 threads: get(row, c) is 16-byte chunk c
// of a row, codes go to dst (row-major, or channel-major for values, through
// `lds`, 64 rows of D + 8 bytes) and the scale to *scale.  The rows are in
// registers between the search for the largest and the rounding, so they are
// read once.  Two barriers of the whole workgroup.
template <int D, int FMT, typename Get>
__device__ __forceinline__ void seal_block(uint32_t (&red)[4], uint8_t *lds, int tid, bool values, Get get, uint8_t *dst,
                                           float *scale) {
  constexpr int CPR = D / 16;                // 16-channel chunks per row
  constexpr int IT = kQ8Block * CPR / 256;   // chunks per thread (2 or 1)
  constexpr int VP = D + 8;                  // pitch of the value codes' rows, bytes
  u32x4 x[IT][2];
  uint32_t mag = 0u;
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int e = tid + 256 * it, row = e / CPR, c = e % CPR;
    x[it][0] = get(row, 2 * c);
    x[it][1] = get(row, 2 * c + 1);
  }
#pragma unroll
  for (int it = 0; it < IT; ++it)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mag = max_mag(max_mag(mag, x[it][h].x), x[it][h].y);
      mag = max_mag(max_mag(mag, x[it][h].z), x[it][h].w);
    }
  const float top = __uint_as_float(max_of_256(red, mag, tid) << 16);
  const float eff = fminf(fmaxf(top, Q8<FMT>::kEffMin), Q8<FMT>::kEffMax);
  const float inv = __fdiv_rn(Q8<FMT>::kTop, eff);
  if (tid == 0) stg(scale, __fdiv_rn(eff, Q8<FMT>::kTop));
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int e = tid + 256 * it, row = e / CPR, c = e % CPR;
    uint32_t o[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t ws[4] = {x[it][h].x, x[it][h].y, x[it][h].z, x[it][h].w};
#pragma unroll
      for (int k = 0; k < 2; ++k)
        o[2 * h + k] = Q8<FMT>::pack4(
            Q8<FMT>::code_value(bf16_lo(ws[2 * k]), inv), Q8<FMT>::code_value(bf16_hi(ws[2 * k]), inv),
            Q8<FMT>::code_value(bf16_lo(ws[2 * k + 1]), inv), Q8<FMT>::code_value(bf16_hi(ws[2 * k + 1]), inv));
    }
    if (!values) {
      st16(dst + row * D + 16 * c, u32x4{o[0], o[1], o[2], o[3]});
    } else {
      u32x2 *t = reinterpret_cast<u32x2 *>(lds + row * VP + 16 * c);
      t[0] = u32x2{o[0], o[1]};
      t[1] = u32x2{o[2], o[3]};
    }
  }
  __syncthreads();
  if (values) {
    // Thread: channels 4 cq .. 4 cq + 3, rows 8 rg .. 8 rg + 7.
    const int rg = tid % 8;
#pragma unroll
    for (int cq = tid / 8; cq < D / 4; cq += 32) {
      uint32_t w[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) w[r] = *reinterpret_cast<const uint32_t *>(lds + (8 * rg + r) * VP + 4 * cq);
      const u32x4 a = transpose4(w[0], w[1], w[2], w[3]), b = transpose4(w[4], w[5], w[6], w[7]);
      const uint32_t as[4] = {a.x, a.y, a.z, a.w}, bs[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) st8(dst + (4 * cq + k) * kQ8Block + 8 * rg, u32x2{as[k], bs[k]});
    }
  }
}

// Rows a unit holds: its length within its capacity, and so that the end of
// its last block still is a row index.
constexpr int kQ8MaxRows = INT32_MAX - 2 * kQ8Block;
__device__ __forceinline__ int rows_held(int len, int cap) { return max(min(min(len, cap), kQ8MaxRows), 0); }

// First element of row i of unit u = (l*B + b)*Hkv + g in a strided tensor.
__device__ __forceinline__ int64_t unit_base(const RowsDesc &r, const int64_t *unit_off, int u, int B, int Hkv) {
  if (unit_off) return ldg(unit_off + u);
  const int g = u % Hkv, lb = u / Hkv;
  return (int64_t)(lb / B) * r.layer + (int64_t)(lb % B) * r.seq + (int64_t)g * r.head;
}

// Sum over a wave.
__device__ __forceinline__ float wave_sum(float x) {
  const auto bits = [&] { return (int)__float_as_uint(x); };
  // (shifts and broadcasts as in wave_incl_scan)
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, bits(), 0x111, 0xF, 0xF, false));
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, bits(), 0x112, 0xF, 0xF, false));
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, bits(), 0x114, 0xF, 0xF, false));
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, bits(), 0x118, 0xF, 0xF, false));
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, bits(), 0x142, 0xA, 0xF, false));
  x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, bits(), 0x143, 0xC, 0xF, false));
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
}

// Which column tile and key split a prompt's workgroup takes, of how many, and
// what the tile's unit is.
struct Share {
  int u, qt, sp, ns;  // unit (-1: nothing to do), tile, split of ns
  int id;             // where its partial results go
  int len, cnt;       // rows held, queries
  int64_t blk0;       // the unit's first block
};

// Workgroup `bid` of a prompt: tiles in the order of their units, splits
// innermost, those of a unit on one XCD (they share its L2); every lane of the
// wave takes part.  Where few tiles are cut along
// their rows, as many blocks go to each workgroup as make no more splits than
// workgroups: sequences without queries take none, longer units take more.  (us,
// with partial results in fp16, with as many splits for every tile and so: four sequences of 3000 to 12801
// rows with 40 queries each 56.5, 47.8, with up to 40 44.6, 36.5; three of 9001 to
// 12801 with up to 65 51.6, 48.9; one of 12544 with 30 23.7, 24.0, with 1024 202,
// 205.)
__device__ __forceinline__ Share share_of(const Q8Attn &p, uint32_t bid, int lane) {
  auto queries = [&](int u) { return p.count ? min(max(ldg(p.count + u / p.Hkv % p.B), 0), p.n) : p.n; };
  if (p.ns == 1) {
    const int id = (int)xcd_block(bid, (uint32_t)p.wgs), u = id / p.nqt;
    return Share{u, id % p.nqt, 0, 1, id, rows_held(ldg(p.c.len + u), ldg(p.c.cap + u)), queries(u),
                 ldg(p.c.row_off + u) / kQ8Block};
  }
  // Lane: tiles K lane .. K lane + K - 1, by their blocks.  Of 256 columns no more
  // than 128, a wave a SIMD, take three quarters of the time (1.4 to 1.6 us a
  // block against 2.0), and count as that.
  constexpr int KM = kQ8SplitTiles / 64;
  const int tiles = p.units * p.nqt, K = (tiles + 63) / 64;
  int nb[KM], held[KM], cnt[KM];
  int64_t off[KM];
  float all = 0.f;
#pragma unroll
  for (int k = 0; k < KM; ++k) {
    if (k >= K) break;  // uniform
    const int t = K * lane + k, u = (int)((uint32_t)min(t, tiles - 1) / (uint32_t)p.nqt);
    held[k] = rows_held(ldg(p.c.len + u), ldg(p.c.cap + u));
    cnt[k] = queries(u);
    off[k] = ldg(p.c.row_off + u);
    const int c0 = (t - u * p.nqt) * p.qcols, cl = min(c0 + p.qcols, cnt[k] * p.G) - 1;
    const int seen = min(p.causal ? held[k] - cnt[k] + 1 + (int)((uint32_t)max(cl, 0) / (uint32_t)p.G) : held[k], p.max_rows);
    nb[k] = t < tiles && cl >= c0 ? max((seen + kQ8Block - 1) / kQ8Block, 1) : 0;
    if (p.qcols == 256 && cl - c0 < 128) nb[k] -= nb[k] / 4;
    all += (float)nb[k];
  }
  all = wave_sum(all);
  // The fewest blocks a split: sum ceil(nb / q) <= wgs, which q >= sum nb /
  // (wgs - tiles) always meets.
  int lo = max(kQ8SplitBlocks, (int)(all / (float)p.wgs));
  int hi = max(lo, (int)(all * 1.0001f / (float)(p.wgs - tiles)) + 1);
  auto splits = [&](int q) {
    int s = 0;
#pragma unroll
    for (int k = 0; k < KM; ++k)
      if (k < K) s += (int)((uint32_t)(nb[k] + q - 1) / (uint32_t)q);
    return s;
  };
  while (lo < hi) {
    const int q = lo + (hi - lo) / 2;
    if (__builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)splits(q)), 63) <= p.wgs)
      hi = q;
    else
      lo = q + 1;
  }
  const int own = splits(lo);
  int first = (int)wave_incl_scan((uint32_t)own);
  const uint32_t used = (uint32_t)__builtin_amdgcn_readlane(first, 63);
  Share s{-1, 0, 0, 0, 0, 0, 0, 0};
  if (bid >= used) return s;
  const int id = (int)xcd_block(bid, used);
  first -= own;
  const uint64_t hit = __builtin_amdgcn_ballot_w64(first <= id && id < first + own);
  int t = 0;
#pragma unroll
  for (int k = 0; k < KM; ++k) {
    if (k >= K) break;
    const int ns = (int)((uint32_t)(nb[k] + lo - 1) / (uint32_t)lo);
    if (first <= id && id < first + ns) t = K * lane + k, s = Share{0, 0, id - first, ns, id, held[k], cnt[k], off[k]};
    first += ns;
  }
  const int src = __builtin_ctzll(hit);
  auto of = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
  t = of(t);
  const uint64_t at = (uint32_t)of((int)s.blk0) | (uint64_t)(uint32_t)of((int)(s.blk0 >> 32)) << 32;
  return Share{t / p.nqt, t % p.nqt, of(s.sp), of(s.ns), id, of(s.len), of(s.cnt), (int64_t)at / kQ8Block};
}

}  // namespace vc
