// k_q8_decode.hip -- attention over the 8-bit cache for single tokens (up to
// 16 (token, query head) columns per kv head).
//
// Bound by memory: every code is read once, by one wave, and used for all the
// columns of its kv head.  The codes enter the matrix cores as fp16, in which
// int8 and e4m3 are exact; the query's bf16 values are scaled by a power of two
// per head and are exact there too.  A block's key scale multiplies its
// logits, its value scale the block's product:
//   O <- alpha O + vs_b (P_b Vc_b),
// P split in two fp16 parts whatever the output's type: 22 bits of a weight down
// to 2^-14 of the largest one of its column, a step of 2^-38 below that (the
// parts are of 2^14 p, and fp16's smallest step is 2^-24).  Sums, maxima and O are
// fp32.  (The second part's products do not show beside the memory: a step of 896
// units of 800 to 2200 rows with bf16 outputs 80.9 us with one part, 81.1 with two,
// timed in turn.)
//
// Layout: S^T = K Q^T with the rows of a 64-row block dealt to the matrix
// rows so that a lane ends with the logits of rows 16 lg .. 16 lg + 15 of its
// column; those are the k-elements of P^T, and the value codes' channel-major
// order gives the same 16 rows in one 16-byte load, so neither P nor V passes
// through LDS.  The open block's bf16 rows, 16 a wave, are scaled into fp16 by
// their power of two and their values transposed through LDS; they are
// requested with the first block, since the whole kernel waits for them (read
// by one wave after its own blocks they took 8 of 25 us).
//
// Measured: 896 units of 2300 to 5800 rows, 128 channels, 169 to 174 us (5.5 TB/s, the
// rate of reads alone); 112 units of about 1050 rows, 15 to 16 us, of which the bytes
// at that rate are 5.5 and the launch and the chain of round trips (length,
// codes, partials in LDS) the rest.
//
// A step is one launch: every workgroup turns its unit's queries itself while
// its first blocks are on their way, and the one with the unit's last rows
// appends the new one, sealing the block that it completes first.
#include "vc_q8_device.h"

namespace vc {

namespace {

constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// 16 rows of k instead of 32: four elements a lane, rows 4 lg .. 4 lg + 3.
__device__ __forceinline__ f32x4 mfma16x4(f16x4 a, f16x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f16x8 pack8(const _Float16 *h) {
  return f16x8{h[0], h[1], h[2], h[3], h[4], h[5], h[6], h[7]};
}

constexpr int kWaves = 4;

template <int D>
struct Smem {
  static constexpr int VP = D + 16;  // pitch of the open block's values: conflict-free transposing reads
  static constexpr size_t kO = sizeof(float) * kWaves * 16 * (D + 4);
  static constexpr size_t kT = sizeof(uint16_t) * kQ8Block * VP;
  // The open block's values (16 rows a wave), then the waves' O.
  uint8_t buf[kO > kT ? kO : kT] __attribute__((aligned(16)));
  float2 ml[kWaves][16];
  // A step's rows: the query heads, the new key (16) and value (17).
  uint16_t rows[18][D + 8] __attribute__((aligned(16)));
  float2 cs[kRopeMaxHalf];
  uint32_t red[4];
};

// What a wave carries over its blocks, per lane: the column's running maximum
// and its own rows' sum, and O^T (channels 16 mb + 4 lg + i of column lr).
template <int D>
struct State {
  float m, l;
  f32x4 O[D / 16];
};

// Logits into the state: S (raw products; row rowof(k) in S[k / 4][k % 4], k <
// 4 NB) times c, rows at or past `end` masked.  Returns the weights, as the fp16
// parts hi + lo of 2^14 p.
template <int D, int NB, typename RowOf>
__device__ __forceinline__ void weigh(State<D> &st, f32x4 (&S)[NB], float c, int end, bool mask, RowOf rowof,
                                      _Float16 (&hi)[4 * NB], _Float16 (&lo)[4 * NB]) {
  c = fmaxf(c, 1e-37f);  // not zero, so that a masked row stays at -inf
  if (mask) {  // uniform
#pragma unroll
    for (int k = 0; k < 4 * NB; ++k)
      if (rowof(k) >= end) S[k / 4][k % 4] = kNegInf;
  }
  float mx = S[0][0];
#pragma unroll
  for (int k = 1; k < 4 * NB; ++k) mx = fmaxf(mx, S[k / 4][k % 4]);
  mx = fmaxf(mx, swap16(mx));
  mx = max_halves(mx) * c;
  const float mn = fmaxf(st.m, mx);
  const float ref = mn == kNegInf ? 0.f : mn;
  if (__builtin_amdgcn_ballot_w64(mn != st.m)) {  // some column's maximum moved
    const float alpha = fast_exp2(st.m - ref);
    st.l *= alpha;
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) st.O[mb] *= alpha;
  }
  st.m = mn;
#pragma unroll
  for (int k = 0; k < 4 * NB; ++k) {
    const float pr = fast_exp2(fmaf(S[k / 4][k % 4], c, -ref));
    st.l += pr;
    // 2^14 keeps the small ones clear of fp16's subnormals.
    const float ps = pr * 16384.f;
    hi[k] = (_Float16)ps;
    lo[k] = (_Float16)(ps - (float)hi[k]);
  }
}

__device__ __forceinline__ u32x2 lds_read_tr16(const uint16_t *p) {
  typedef short v4i16 __attribute__((ext_vector_type(4)));
  const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)(p));
  return __builtin_bit_cast(u32x2, v);
}

// Columns of the products: column c is query c / G, head c % G of its kv head.
__device__ __forceinline__ int64_t out_row(const Q8Attn &p, const RowsDesc &r, int u, int col) {
  const int g = u % p.Hkv, lb = u / p.Hkv;
  const int i = col / p.G, h = col % p.G;
  return (int64_t)(lb / p.B) * r.layer + (int64_t)(lb % p.B) * r.seq + (int64_t)i * r.token +
         (int64_t)(g * p.G + h) * r.head;
}

__device__ __forceinline__ void put(const Q8Attn &p, int64_t at, float v) {
  if (p.fp32)
    stg(reinterpret_cast<float *>(p.out.base) + at, v);
  else
    stg(reinterpret_cast<uint16_t *>(p.out.base) + at, (uint16_t)pack_bf16(v, 0.f));
}

// The query heads of the unit (rows 0 .. G - 1), the new key (16) and the new
// value (17) into LDS, queries and key turned to their position; two barriers.
template <int D>
__device__ __forceinline__ void step_rows(const Q8Attn &p, Smem<D> &sm, int u, int tid) {
  const int g = u % p.Hkv, lb = u / p.Hkv, b = lb % p.B, l = lb / p.B;
  for (int e = tid; e < (p.G + 2) * (D / 8); e += 256) {
    const int r = e / (D / 8), c = e % (D / 8);
    const RowsDesc &d = r < p.G ? p.q : r == p.G ? p.k : p.v;
    const int64_t at = (int64_t)l * d.layer + (int64_t)b * d.seq + (int64_t)(r < p.G ? g * p.G + r : g) * d.head;
    *reinterpret_cast<u32x4 *>(&sm.rows[r < p.G ? r : 16 + r - p.G][8 * c]) =
        ld16(reinterpret_cast<const uint16_t *>(d.base) + at + 8 * c);
  }
  const int half = p.rope.rot / 2;
  if (tid < half) sm.cs[tid] = turn_of(p.rope, tid, ldg(p.pos + (int64_t)axis_of(p.rope, tid) * p.B + b));
  __syncthreads();
  for (int e = tid; e < (p.G + 1) * half; e += 256) {
    const int r = e / half, i = e % half;
    uint16_t *row = sm.rows[r < p.G ? r : 16];
    uint16_t *x1 = row + (p.rope.adjacent ? 2 * i : i), *x2 = row + (p.rope.adjacent ? 2 * i + 1 : i + half);
    float a = __uint_as_float((uint32_t)*x1 << 16), c = __uint_as_float((uint32_t)*x2 << 16);
    turn(a, c, sm.cs[i]);
    *x1 = (uint16_t)pack_bf16(a, 0.f);
    *x2 = (uint16_t)pack_bf16(c, 0.f);
  }
  if (half > 0) __syncthreads();
}

// The open block's scale once `row` is its row `slot`.
template <int D>
__device__ __forceinline__ float grown_scale(const uint16_t *row, int slot, float before, int lane) {
  uint32_t m = 0u;
  if (lane < D / 2) m = max_mag(0u, reinterpret_cast<const uint32_t *>(row)[lane]);
  uint32_t x = max(m & 0xFFFFu, m >> 16);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, k, 64));
  const float s = open_scale(x);
  return slot > 0 ? fmaxf(s, before) : s;
}

// Workgroup (unit, piece): blocks [j piece, (j + 1) piece) of the unit, dealt
// to the four waves in turn.
template <int D, int FMT, bool STEP>
__global__ __launch_bounds__(64 * kWaves, 2) void k_decode8(Q8Attn p) {
  constexpr int MB = D / 16, CH = D / 64;
  __shared__ Smem<D> sm;
  const int i = (int)(blockIdx.x % (uint32_t)p.units), j = (int)(blockIdx.x / (uint32_t)p.units);
  const int u = p.c.order ? ldg(p.c.order + i) : i;
  if (u < 0 || u >= p.units) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int b = u / p.Hkv % p.B;
  // What the unit is, in one round trip.
  const int len_ = ldg(p.c.len + u), cap_ = ldg(p.c.cap + u), cnt_ = p.count ? ldg(p.count + b) : p.n;
  const int64_t row_off = ldg(p.c.row_off + u);
  const int len0 = rows_held(len_, cap_), cnt = min(max(cnt_, 0), p.n);
  const bool room = STEP && len_ >= 0 && len_ < min(cap_, kQ8MaxRows);  // a step appends a row
  const int len = len0 + room;
  const int cols = cnt * p.G;
  const int emax = cols > 0 ? min(len, p.max_rows) : 0;  // rows any column sees
  const int nt = (emax + kQ8Block - 1) / kQ8Block;
  const int np = max((nt + p.piece - 1) / p.piece, 1);
  if (j >= np || cols == 0) return;
  // Rows this lane's column sees, and the fewest any column does.
  const int qi = min(lr, cols - 1) / p.G;
  const int lim = p.causal ? len - cnt + 1 : len;
  const int end = max(min(p.causal ? lim + qi : len, p.max_rows), 0);
  const int emin = min(lim, p.max_rows);
  const int64_t blk0 = row_off / kQ8Block;
  const int nsealed = len / kQ8Block;
  // The unit's last piece appends, at `slot` of the open block.
  const bool mine = room && j == np - 1;
  const int slot = len0 % kQ8Block;
  const int64_t tail = (int64_t)u * kQ8Block * D;
  const bool seals = STEP && mine && slot == kQ8Block - 1;
  if (seals) {  // the new row completes its block, which is read as codes below
    step_rows<D>(p, sm, u, tid);
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
      const uint16_t *from = (side ? p.c.vt : p.c.kt) + tail;
      const int64_t blk = blk0 + len0 / kQ8Block;
      seal_block<D, FMT>(
          sm.red, sm.buf, tid, side == 1,
          [&](int row, int c) {
            return row < slot ? ld16(from + row * D + 8 * c)
                              : *reinterpret_cast<const u32x4 *>(&sm.rows[16 + side][8 * c]);
          },
          (side ? p.c.vc : p.c.kc) + blk * (kQ8Block * D), (side ? p.c.vs : p.c.ks) + blk);
      __threadfence_block();
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();  // the codes are written, sm.buf and sm.red are free
    }
  }

  // The query's requests, then the first block's, before anything waits.
  u32x4 qx[CH][2];
  if (!STEP) {
    const uint16_t *qp = reinterpret_cast<const uint16_t *>(p.q.base) + out_row(p, p.q, u, min(lr, cols - 1));
#pragma unroll
    for (int h = 0; h < CH; ++h)
#pragma unroll
      for (int k = 0; k < 2; ++k) qx[h][k] = ld16(qp + 64 * h + 16 * lg + 8 * k);
  }
  State<D> st;
  st.m = kNegInf;
  st.l = 0.f;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) st.O[mb] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int t0 = j * p.piece, t1 = min(nt, t0 + p.piece);
  const int ts = min(t1, nsealed);  // sealed blocks end
  const int krow = 16 * (lr >> 2) + (lr & 3);
  u32x4 kc[4][CH], vcode[MB];
  float ks = 0.f, vs = 0.f;
  auto load_k = [&](int t) {
    const uint8_t *k = p.c.kc + (blk0 + t) * (kQ8Block * D);
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
#pragma unroll
      for (int h = 0; h < CH; ++h) kc[rb][h] = ld16(k + (krow + 4 * rb) * D + 64 * h + 16 * lg);
    ks = ldg(p.c.ks + blk0 + t);
  };
  auto load_v = [&](int t) {
    const uint8_t *v = p.c.vc + (blk0 + t) * (kQ8Block * D);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) vcode[mb] = ld16(v + (16 * mb + lr) * kQ8Block + 16 * lg);
    vs = ldg(p.c.vs + blk0 + t);
  };
  int t = t0 + w;
  if (t < ts) {
    load_k(t);
    load_v(t);
  }
  // The open block, if it is in this piece: a wave takes 16 of its rows.
  constexpr int VT = D / 32;
  const bool open = nsealed >= t0 && nsealed < t1;
  const int orows = len - nsealed * kQ8Block;  // 1 .. 63 where open
  u32x4 ok[CH][2], ov[VT];
  float kse = 1.f, vse = 1.f;
  if (open) {
    const uint16_t *kt = p.c.kt + tail + min(16 * w + lr, orows - 1) * D + 16 * lg;
#pragma unroll
    for (int h = 0; h < CH; ++h)
#pragma unroll
      for (int x = 0; x < 2; ++x) ok[h][x] = ld16(kt + 64 * h + 8 * x);
#pragma unroll
    for (int it = 0; it < VT; ++it) ov[it] = ld16(p.c.vt + tail + 16 * w * D + 8 * (lane + 64 * it));
    kse = ldg(p.c.ks + blk0 + nsealed);
    vse = ldg(p.c.vs + blk0 + nsealed);
  }
  if (STEP) {
    if (!seals) step_rows<D>(p, sm, u, tid);
    if (mine && !seals) {
      if (tid < 2 * (D / 8)) {
        const int side = tid / (D / 8), c = tid % (D / 8);
        st16((side ? p.c.vt : p.c.kt) + tail + slot * D + 8 * c,
             *reinterpret_cast<const u32x4 *>(&sm.rows[16 + side][8 * c]));
      }
      // The block's scales grow with the row (the same in every wave, whether it
      // has read them before or after wave 0 wrote them) ...
      const int64_t blk = blk0 + len0 / kQ8Block;
      kse = grown_scale<D>(sm.rows[16], slot, ldg(p.c.ks + blk), lane);
      vse = grown_scale<D>(sm.rows[17], slot, ldg(p.c.vs + blk), lane);
      if (tid == 0) {
        stg(p.c.ks + blk, kse);
        stg(p.c.vs + blk, vse);
      }
      // ... and the row itself comes from LDS.
      if (min(16 * w + lr, orows - 1) == slot) {
#pragma unroll
        for (int h = 0; h < CH; ++h)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            ok[h][x] = *reinterpret_cast<const u32x4 *>(&sm.rows[16][64 * h + 16 * lg + 8 * x]);
      }
#pragma unroll
      for (int it = 0; it < VT; ++it) {
        const int e = lane + 64 * it;
        if (16 * w + e / (D / 8) == slot) ov[it] = *reinterpret_cast<const u32x4 *>(&sm.rows[17][8 * (e % (D / 8))]);
      }
    }
#pragma unroll
    for (int h = 0; h < CH; ++h)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        qx[h][k] = *reinterpret_cast<const u32x4 *>(&sm.rows[min(lr, cols - 1)][64 * h + 16 * lg + 8 * k]);
  }
  // The column's query as fp16 operands, scaled by a power of two.
  f16x8 q[CH][2];
  float cq;
  {
    uint32_t mag = 0u;
#pragma unroll
    for (int h = 0; h < CH; ++h)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        mag = max_mag(max_mag(max_mag(max_mag(mag, qx[h][k].x), qx[h][k].y), qx[h][k].z), qx[h][k].w);
    uint32_t mm = max(mag & 0xFFFFu, mag >> 16);
    mm = max(mm, (uint32_t)__shfl_xor((int)mm, 16, 64));
    mm = max(mm, (uint32_t)__shfl_xor((int)mm, 32, 64));
    const float qs = open_scale(mm);
    cq = p.sc * qs;
    const float inv = 1.f / qs;  // exact: a power of two
#pragma unroll
    for (int h = 0; h < CH; ++h)
#pragma unroll
      for (int k = 0; k < 2; ++k) q[h][k] = half8_of_bf16(qx[h][k], inv);
  }
  for (; t < ts; t += kWaves) {
    f32x4 S[4];
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      S[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < CH; ++h) {
        S[rb] = mfma16(Q8<FMT>::half8(kc[rb][h].x, kc[rb][h].y), q[h][0], S[rb]);
        S[rb] = mfma16(Q8<FMT>::half8(kc[rb][h].z, kc[rb][h].w), q[h][1], S[rb]);
      }
    }
    const float c = cq * ks, v = vs;
    const int tn = min(t + kWaves, ts - 1);  // the last block again where there is no next (never used)
    load_k(tn);
    _Float16 hi[16], lo[16];
    weigh<D, 4>(
        st, S, c, end, (t + 1) * kQ8Block > emin,
        [&](int k) { return t * kQ8Block + 16 * lg + k; }, hi, lo);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const f16x8 a = x == 0 ? Q8<FMT>::half8(vcode[mb].x, vcode[mb].y) : Q8<FMT>::half8(vcode[mb].z, vcode[mb].w);
        o = mfma16(a, pack8(hi + 8 * x), o);
        o = mfma16(a, pack8(lo + 8 * x), o);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) st.O[mb][i] = fmaf(o[i], v, st.O[mb][i]);
    }
    load_v(tn);
  }
  // The open block.
  if (open) {
    const float kinv = 1.f / kse, vinv = 1.f / vse;  // powers of two
    uint16_t *lv = reinterpret_cast<uint16_t *>(sm.buf) + w * 16 * Smem<D>::VP;
#pragma unroll
    for (int it = 0; it < VT; ++it) {
      const int e = lane + 64 * it, row = e / (D / 8), cc = e % (D / 8);
      // Rows past the end hold anything: zeros meet their zero weights.
      const u32x4 x = 16 * w + row < orows ? ov[it] : u32x4{0u, 0u, 0u, 0u};
      *reinterpret_cast<f16x8 *>(lv + row * Smem<D>::VP + 8 * cc) = half8_of_bf16(x, vinv);
    }
    f32x4 S[1] = {{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int h = 0; h < CH; ++h)
#pragma unroll
      for (int x = 0; x < 2; ++x) S[0] = mfma16(half8_of_bf16(ok[h][x], kinv), q[h][x], S[0]);
    _Float16 hi[4], lo[4];
    weigh<D, 1>(
        st, S, cq * kse, end, true, [&](int k) { return nsealed * kQ8Block + 16 * w + 4 * lg + k; }, hi, lo);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's LDS writes landed
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const f16x4 a = __builtin_bit_cast(
          f16x4, lds_read_tr16(lv + (4 * lg + (lr >> 2)) * Smem<D>::VP + 16 * mb + 4 * (lr & 3)));
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      o = mfma16x4(a, f16x4{hi[0], hi[1], hi[2], hi[3]}, o);
      o = mfma16x4(a, f16x4{lo[0], lo[1], lo[2], lo[3]}, o);
      // (A column that sees no row of the block takes nothing of it: its weights
      // are zero, but an infinity or a NaN among the values is not.)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.O[mb][i] = fmaf(end > nsealed * kQ8Block ? o[i] : 0.f, vse, st.O[mb][i]);
    }
  }

  // The waves' states.
  st.l = sum_halves(st.l + swap16(st.l));
  __syncthreads();  // the open block's values are read
  if (STEP && tid == 0) {
    // The length: by the join where there is one, since the other pieces read it.
    if (p.npmax > 1) {
      if (j == np - 1) stg(p.np + u, np | (int)room << 30);
    } else if (room) {
      stg(p.c.len + u, len_ + 1);
    }
  }
  float(*wo)[16][D + 4] = reinterpret_cast<float(*)[16][D + 4]>(sm.buf);
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
    *reinterpret_cast<f32x4 *>(&wo[w][lr][16 * mb + 4 * lg]) = st.O[mb];
  if (lg == 0) sm.ml[w][lr] = make_float2(st.m, st.l);
  __syncthreads();
  const int x = tid % D;
  const int64_t part = (int64_t)u * p.npmax + j;
  for (int col = tid / D; col < cols; col += 64 * kWaves / D) {
    float M = kNegInf;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) M = fmaxf(M, sm.ml[k][col].x);
    // (Without a maximum there are no rows, all zeros, or only NaN, which stay.)
    const float ref = M == kNegInf ? 0.f : M;
    float o = 0.f, s = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float f = fast_exp2(sm.ml[k][col].x - ref);
      o += f * wo[k][col][x];
      s += f * sm.ml[k][col].y;
    }
    o *= 0x1p-14f;
    if (np == 1) {
      put(p, out_row(p, p.out, u, col) + x, s == 0.f ? 0.f : o / s);
    } else {
      stg(p.part_o + (part * 16 + col) * D + x, o);
      if (x == 0) stg(p.part_ml + part * 16 + col, make_float2(M, s));
    }
  }
}

template <int D, int FMT>
hipError_t launch(const Q8Attn &p, hipStream_t st) {
  const dim3 grid((uint32_t)p.wgs), block(64 * kWaves);
  if (p.step)
    hipLaunchKernelGGL((k_decode8<D, FMT, true>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((k_decode8<D, FMT, false>), grid, block, 0, st, p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || p.npmax == 1 ? e : launch_q8_join(p, st);
}

}  // namespace

hipError_t launch_q8_decode(const Q8Attn &p, int format, hipStream_t st) {
  if (p.d == 128) return format == kInt8 ? launch<128, kInt8>(p, st) : launch<128, kE4m3>(p, st);
  return format == kInt8 ? launch<64, kInt8>(p, st) : launch<64, kE4m3>(p, st);
}

}  // namespace vc
