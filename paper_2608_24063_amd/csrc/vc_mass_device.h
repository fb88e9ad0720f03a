// vc_mass_device.h -- what the kernels over a cache with its rows' attention weight
// share.  Internal to libviscache.
#pragma once
#include "vc_mass.h"
#include "vc_q8_device.h"

namespace vc {

// A unit in a call: rows before it and with what it appends, and its queries, of which
// query i sees rows t < min(base + i + 1, held, max_rows).
struct MassUnit {
  int64_t off;  // first pool row
  int len0, held, base, cnt;
};
__device__ __forceinline__ MassUnit mass_unit(const MassAttn &p, int u) {
  const int len_ = ldg(p.c.len + u), cap_ = ldg(p.c.cap + u);
  const int cnt_ = p.count ? ldg(p.count + u / p.Hkv % p.B) : p.n;
  MassUnit x;
  x.off = ldg(p.c.row_off + u);
  x.cnt = min(max(cnt_, 0), p.n);
  const int cap = max(min(cap_, kMassMaxRows), 0);
  x.len0 = min(max(len_, 0), cap);
  x.held = p.append ? x.len0 + min(x.cnt, cap - x.len0) : x.len0;
  x.base = p.append ? x.len0 : x.held - x.cnt;
  return x;
}

// Of a unit's rows, those whose mass from before the call fades; of the others nothing is
// left: they are new, or decay is 0 (which takes nothing over of a mass that is infinite or no
// number either).
__device__ __forceinline__ int fading_rows(const MassAttn &p, const MassUnit &x) {
  return p.decay == 0.f ? 0 : x.len0;
}

// Column col of unit u (query col / G, head col % G of its kv head) in q or out.
__device__ __forceinline__ int64_t mass_col(const MassAttn &p, const RowsDesc &r, int u, int col) {
  const int g = u % p.Hkv, lb = u / p.Hkv;
  const int i = (int)((uint32_t)col / (uint32_t)p.G), h = col - i * p.G;
  return (int64_t)(lb / p.B) * r.layer + (int64_t)(lb % p.B) * r.seq + (int64_t)i * r.token +
         (int64_t)(g * p.G + h) * r.head;
}

// First element of the new rows of unit u.
__device__ __forceinline__ const uint16_t *new_rows(const MassAttn &p, const RowsDesc &r, int u) {
  const int g = u % p.Hkv, lb = u / p.Hkv;
  return reinterpret_cast<const uint16_t *>(r.base) + (int64_t)(lb / p.B) * r.layer + (int64_t)(lb % p.B) * r.seq +
         (int64_t)g * r.head;
}

// Two fp32 values' upper halves: bf16, rounded toward zero.
__device__ __forceinline__ uint32_t tops(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float top_of(float a) { return __uint_as_float(__float_as_uint(a) & 0xFFFF0000u); }

// Values of a row that not every column of a product sees: an infinity or a NaN, whose
// weight is zero there, would still reach them.  Such values become zeros, and the
// first row of each channel that had one (bad[channel], INT32_MAX: none) makes NaN of
// the columns that do see it.  (Rows that every column sees go through the product as they
// are: an infinity stays one, or becomes NaN where a part of its weight is zero.)
__device__ __forceinline__ bool any_nonfinite(u32x4 w) {
  const uint32_t m = max_mag(max_mag(max_mag(max_mag(0u, w.x), w.y), w.z), w.w);
  return (m & 0xFFFFu) >= 0x7F80u || (m >> 16) >= 0x7F80u;
}
__device__ __forceinline__ u32x4 without_nonfinite(u32x4 w, int row, int32_t *bad) {
  uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((x[i] & 0x7F80u) == 0x7F80u) {
      atomicMin(bad + 2 * i, row);
      x[i] &= 0xFFFF0000u;
    }
    if ((x[i] & 0x7F800000u) == 0x7F800000u) {
      atomicMin(bad + 2 * i + 1, row);
      x[i] &= 0x0000FFFFu;
    }
  }
  return u32x4{x[0], x[1], x[2], x[3]};
}

__device__ __forceinline__ u32x2 lds_transposed(const uint16_t *p) {
  typedef short v4i16 __attribute__((ext_vector_type(4)));
  const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)(p));
  return __builtin_bit_cast(u32x2, v);
}

}  // namespace vc
