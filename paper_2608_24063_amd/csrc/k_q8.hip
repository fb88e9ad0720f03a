// k_q8.hip -- the 8-bit cache as it is written and read back.  64 rows of a
// (layer, sequence, kv head) share a scale, keys and values apart:
//   eff = clamp(max |x|, Q 2^-60, Q 2^60), scale = eff / Q, code = Q x / eff
// rounded to nearest even, Q = 127 (int8) or 448 (e4m3).  A block is sealed
// (quantised) when its 64th row arrives; until then its rows stay in the
// unit's bf16 tail, so the cache is a function of its rows, not of how many
// came at a time.  Keys are stored row-major [64][d]; values channel-major
// [d][64], which is the order the attention's products take them in, so the
// transposition is paid once, here.
//
// Bound by memory: 2 bytes a value in, 1 out.  A workgroup takes a block's
// keys with one half of its waves and its values with the other.  Measured over
// 3.63 million rows of 128 channels, keys and values: written in 521 us (5.3
// TB/s), read back in fp32 in 859 (5.4); 118000 rows in 23 us (4.0), and back in
// bf16 in 17 (5.3).
#include "vc_q8_device.h"

namespace vc {

namespace {

constexpr int kThreads = 512;  // 256 for keys, 256 for values
constexpr int kHalf = 256;

// Workgroup j of a unit's nj seals blocks j, j + nj, ... of those its new rows
// fill; workgroup 0 also takes an open last block, since that goes over the
// tail rows the first block is made of.
template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void k_append_rows(Q8Rows p) {
  __shared__ uint8_t lds[kQ8Block * (D + 8)] __attribute__((aligned(16)));
  __shared__ uint32_t red[2][4];
  constexpr int CPR = D / 16;                     // 16-channel chunks per row
  const int u = (int)(blockIdx.x / (uint32_t)p.nj), j = (int)(blockIdx.x % (uint32_t)p.nj);
  const int side = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8), tid = threadIdx.x & 255;
  const int len0 = max(ldg(p.c.len + u), 0), cap = min(ldg(p.c.cap + u), kQ8MaxRows);
  const int want = p.count ? min(max(ldg(p.count + u / p.Hkv), 0), p.n) : p.n;
  const int m = min(want, max(cap - len0, 0));
  if (m <= 0) return;
  const int end = len0 + m, b0 = len0 / kQ8Block;
  const int nblk = (end + kQ8Block - 1) / kQ8Block - b0;
  const bool open = end % kQ8Block != 0;
  const int nfull = open ? nblk - 1 : nblk;
  if (j >= max(nfull, 1)) return;
  const int64_t blk0 = ldg(p.c.row_off + u) / kQ8Block + b0;
  const RowsDesc &rd = side ? p.v : p.k;
  const uint16_t *src = reinterpret_cast<const uint16_t *>(rd.base) + unit_base(rd, p.unit_off, u, p.B, p.Hkv);
  uint16_t *tail = (side ? p.c.vt : p.c.kt) + (int64_t)u * kQ8Block * D;
  float *scales = side ? p.c.vs : p.c.ks;

  auto seal = [&](int jb) {
    const int lo = jb == 0 ? len0 % kQ8Block : 0;
    const int64_t r0 = (int64_t)(b0 + jb) * kQ8Block - len0;  // new row of the block's row 0
    seal_block<D, FMT>(
        red[side], lds, tid, side == 1,
        [&](int row, int c) { return ld16((row < lo ? tail + row * D : src + (r0 + row) * rd.token) + 8 * c); },
        (side ? p.c.vc : p.c.kc) + (blk0 + jb) * (kQ8Block * D), scales + blk0 + jb);
  };
  // Rows lo .. hi - 1 of open block jb into the tail.
  auto leave_open = [&](int jb) {
    const int lo = jb == 0 ? len0 % kQ8Block : 0, hi = end % kQ8Block;
    const int64_t r0 = (int64_t)(b0 + jb) * kQ8Block - len0;
    uint32_t mag = 0u;
    for (int e = tid; e < (hi - lo) * CPR; e += kHalf) {
      const int row = lo + e / CPR, c = e % CPR;
      const uint16_t *s = src + (r0 + row) * rd.token + 16 * c;
      const u32x4 a = ld16(s), b = ld16(s + 8);
      st16(tail + row * D + 16 * c, a);
      st16(tail + row * D + 16 * c + 8, b);
      mag = max_mag(max_mag(max_mag(max_mag(mag, a.x), a.y), a.z), a.w);
      mag = max_mag(max_mag(max_mag(max_mag(mag, b.x), b.y), b.z), b.w);
    }
    const float s = open_scale(max_of_256(red[side], mag, tid));
    if (tid == 0) stg(scales + blk0 + jb, lo > 0 ? fmaxf(s, ldg(scales + blk0 + jb)) : s);
  };
  for (int jb = j; jb < nfull; jb += p.nj) seal(jb);
  if (j == 0 && open) leave_open(nblk - 1);  // (every tail row of a sealed block 0 was read before a barrier)
  // One workgroup a unit: every thread has read the length (a barrier ago).
  if (p.nj == 1 && threadIdx.x == 0) stg(p.c.len + u, end);
}

// The lengths, where several workgroups of a unit read them.
__global__ __launch_bounds__(256) void k_append_len(Q8Rows p) {
  const int u = (int)(blockIdx.x * 256 + threadIdx.x);
  if (u >= p.units) return;
  const int len0 = max(ldg(p.c.len + u), 0);
  const int want = p.count ? min(max(ldg(p.count + u / p.Hkv), 0), p.n) : p.n;
  const int m = min(want, max(min(ldg(p.c.cap + u), kQ8MaxRows) - len0, 0));
  if (m > 0) stg(p.c.len + u, len0 + m);
}

// 16 bytes of a row: 4 fp32 or 8 bf16 values.  (Streamed: reading back 3.6 M
// rows in fp32 and writing them before 1432 -> 1390 us, 118000 in bf16 50 -> 43; the
// codes that an append writes are read soon, and streaming them cost the
// smaller case 5 us.)
template <bool F32>
__device__ __forceinline__ void put16(char *dst, const float (&f)[8]) {
  st16_stream(dst, F32 ? u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])}
                : u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])});
}

// Workgroup (unit, block): the block's rows below the unit's length (and the
// row bound) as code * scale, or the tail's rows.  A lane writes 16 bytes and
// its neighbours the bytes beside them.
template <int D, int FMT, bool F32>
__global__ __launch_bounds__(kThreads) void k_read_rows(Q8Rows p) {
  constexpr int VP = kQ8Block + 4;  // pitch of a channel's codes, bytes
  constexpr int E = F32 ? 4 : 2;
  constexpr int N = 16 / E;   // values a lane writes at once
  constexpr int PR = D / N;   // lanes per row
  __shared__ uint32_t vt[D * VP / 4];
  const int u = (int)(blockIdx.x / (uint32_t)p.nj), j = (int)(blockIdx.x % (uint32_t)p.nj);
  const int side = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8), tid = threadIdx.x & 255;
  const int len = rows_held(ldg(p.c.len + u), ldg(p.c.cap + u));
  const int rows = min(min(len, p.n) - j * kQ8Block, kQ8Block);
  if (rows <= 0) return;
  const int64_t blk = ldg(p.c.row_off + u) / kQ8Block + j;
  const RowsDesc &rd = side ? p.v : p.k;
  char *out = reinterpret_cast<char *>(rd.base) +
              E * (unit_base(rd, p.unit_off, u, p.B, p.Hkv) + (int64_t)j * kQ8Block * rd.token);
  const int64_t pitch = E * rd.token;
  if (j >= len / kQ8Block) {  // uniform: the open block
    const uint16_t *tail = (side ? p.c.vt : p.c.kt) + (int64_t)u * kQ8Block * D;
    for (int e = tid; e < rows * PR; e += kHalf) {
      const int row = e / PR, c = e % PR;
      const u32x2 x = ld8(tail + row * D + N * c);
      const u32x2 y = F32 ? x : ld8(tail + row * D + N * c + 4);
      const float f[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y),
                          bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y)};
      put16<F32>(out + row * pitch + 16 * c, f);
    }
    return;
  }
  const uint8_t *codes = (side ? p.c.vc : p.c.kc) + blk * (kQ8Block * D);
  const float s = ldg((side ? p.c.vs : p.c.ks) + blk);
  auto values = [&](uint32_t w0, uint32_t w1, float(&f)[8]) {
    float a[4], b[4];
    Q8<FMT>::unpack4(w0, a);
    if (!F32) Q8<FMT>::unpack4(w1, b);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[k] = a[k] * s;
      f[4 + k] = F32 ? 0.f : b[k] * s;
    }
  };
  if (side == 1) {
#pragma unroll
    for (int e = tid; e < D * kQ8Block / 16; e += kHalf) {
      const int ch = e / 4, rg = e % 4;
      const u32x4 x = ld16(codes + ch * kQ8Block + 16 * rg);
      uint32_t *t = vt + ch * (VP / 4) + 4 * rg;
      t[0] = x.x;
      t[1] = x.y;
      t[2] = x.z;
      t[3] = x.w;
    }
  }
  __syncthreads();
  if (side == 0) {
#pragma unroll
    for (int e = tid; e < kQ8Block * PR; e += kHalf) {
      const int row = e / PR, c = e % PR;
      const uint8_t *src = codes + row * D + N * c;
      u32x2 w;
      if (F32)
        w = u32x2{ldg(reinterpret_cast<const uint32_t *>(src)), 0u};
      else
        w = ld8(src);
      float f[8];
      values(w.x, w.y, f);
      if (row < rows) put16<F32>(out + row * pitch + 16 * c, f);
    }
  } else {
    // Thread: N channels of rows 4 rq .. 4 rq + 3.
#pragma unroll
    for (int e = tid; e < PR * 16; e += kHalf) {
      const int c = e % PR, rq = e / PR;
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < N; ++k) w[k] = vt[(N * c + k) * (VP / 4) + rq];
      const u32x4 a = transpose4(w[0], w[1], w[2], w[3]);
      const u32x4 b = F32 ? a : transpose4(w[4], w[5], w[6], w[7]);
      const uint32_t as[4] = {a.x, a.y, a.z, a.w}, bs[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float f[8];
        values(as[r], bs[r], f);
        if (4 * rq + r < rows) put16<F32>(out + (4 * rq + r) * pitch + 16 * c, f);
      }
    }
  }
}

template <int FMT>
hipError_t append(const Q8Rows &p, hipStream_t st) {
  const dim3 grid((uint32_t)((int64_t)p.units * p.nj)), block(kThreads);
  if (p.d == 128)
    hipLaunchKernelGGL((k_append_rows<128, FMT>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((k_append_rows<64, FMT>), grid, block, 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nj == 1) return e;
  hipLaunchKernelGGL(k_append_len, dim3((uint32_t)((p.units + 255) / 256)), dim3(256), 0, st, p);
  return hipGetLastError();
}

template <int FMT, bool F32>
hipError_t read(const Q8Rows &p, hipStream_t st) {
  const dim3 grid((uint32_t)((int64_t)p.units * p.nj)), block(kThreads);
  if (p.d == 128)
    hipLaunchKernelGGL((k_read_rows<128, FMT, F32>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((k_read_rows<64, FMT, F32>), grid, block, 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_append(const Q8Rows &p, int format, hipStream_t st) {
  return format == kInt8 ? append<kInt8>(p, st) : append<kE4m3>(p, st);
}

hipError_t launch_q8_read(const Q8Rows &p, int format, hipStream_t st) {
  if (format == kInt8) return p.fp32 ? read<kInt8, true>(p, st) : read<kInt8, false>(p, st);
  return p.fp32 ? read<kE4m3, true>(p, st) : read<kE4m3, false>(p, st);
}

}  // namespace vc
