// k_mass_token.hip -- attention over a bf16 cache for single tokens (up to 16 (token,
// query head) columns per kv head) that also adds what every row was given to the
// row's mass, and appends the tokens' own rows on its way.
//
// A row's weight, exp(s - m) / l, is known only after the last row, and to compute the
// logits again would read the keys again.  So the logits wait until the maximum and the
// sum are known: where a unit is one workgroup's, in LDS as far as there is room, and
// the rest, as those of units that are cut, in the workspace.  (In the workspace they
// are 4 bytes a column and row beside the row's 4 d, but cost more than their share: of
// 896 units of 2300 to 5800 rows and 7 columns, 320 us without them, 404 where they are
// written, 443 where they are read back too.)  A second launch joins the outputs of
// units that are cut and adds their weights up.
//
// Bound by memory: those 896 units take 352 us (5.3 TB/s of rows).  Fewer units than CUs
// are bound by the longest one, since a CU reads no more than 51 GB/s: 112 of 620 to 1490
// rows 24 us, 7 of them the chain of length, first rows, join and masses that 8 units of
// 90 to 170 rows take too.  A wave takes tiles of 32 rows, keys straight into the A operands of
//   S^T = K Q^T,  O^T = V^T P^T,
// values through LDS, read back transposed; the next tile is requested as soon as a
// tile's registers are free.  P enters in three bf16 parts, cut and not rounded, which
// hold all 24 bits of a weight; logits, sums, O and masses are fp32.
#include "vc_mass_device.h"

namespace vc {

namespace {

constexpr float kNegInf = -__builtin_inff();

// NW waves.  Four: 78 KB, two workgroups a CU.  Eight, one a CU: values pass 16 rows at a
// time, which leaves room for three times the logits.
template <int D, int NW>
struct Smem {
  static constexpr int VR = NW == 8 ? 16 : 32;  // rows of values at a time
  static constexpr int VP = D + 16;  // pitch of the values: conflict-free transposing reads
  static constexpr size_t kO = sizeof(float) * 4 * 16 * (D + 4);
  static constexpr size_t kT = sizeof(uint16_t) * NW * VR * VP;
  uint8_t buf[kO > kT ? kO : kT] __attribute__((aligned(16)));  // the waves' values, then O of four waves
  float2 ml[NW][16];
  float2 stat[16];  // maximum and 1 / sum of each column
  int32_t bad[D];   // (without_nonfinite)
  float logits[NW == 8 ? kMassHeld8 : kMassHeld4];
};

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ void put(const MassAttn &p, int64_t at, float v) {
  if (p.fp32)
    stg(reinterpret_cast<float *>(p.out.base) + at, v);
  else
    stg(reinterpret_cast<uint16_t *>(p.out.base) + at, (uint16_t)pack_bf16(v, 0.f));
}

// A logit's weight by its column's maximum and 1 / sum.  (-inf is a row that the column does
// not see, also where the sum is NaN.)
__device__ __forceinline__ float weight_of(const MassAttn &p, float s, float2 st) {
  const float e = fast_exp2(fmaf(s, p.sc, -st.x)) * st.y;
  return s == kNegInf ? 0.f : e;
}

// The masses of rows t .. t + R - 1 (R 1, or 4 and t a multiple of 4) below `last`, from the
// logits of all columns in the workspace, of which eight columns' are in flight at a time.
template <int R>
struct MassRows {
  static constexpr int U = 8;
  float was[R], s[U][R];
  __device__ __forceinline__ void request(const MassAttn &p, const MassUnit &x, const float *logits, int cols, int t,
                                          int last) {
#pragma unroll
    for (int i = 0; i < R; ++i) was[i] = ldg(p.c.mass + x.off + min(t + i, last - 1));
    columns(p, logits, cols, t, 0);
  }
  __device__ __forceinline__ void columns(const MassAttn &p, const float *logits, int cols, int t, int c0) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float *from = logits + (int64_t)min(c0 + k, cols - 1) * p.ldr + t;
      if (R == 4) {
        const u32x4 v = ld16(from);
        s[k][0] = __uint_as_float(v.x);
        s[k][1 % R] = __uint_as_float(v.y);
        s[k][2 % R] = __uint_as_float(v.z);
        s[k][3 % R] = __uint_as_float(v.w);
      } else {
        s[k][0] = ldg(from);
      }
    }
  }
  __device__ __forceinline__ void finish(const MassAttn &p, const MassUnit &x, const float *logits, const float2 *stat,
                                         int cols, int t, int last) {
    float got[R] = {};
    for (int c0 = 0; c0 < cols; c0 += U) {
      if (c0 > 0) columns(p, logits, cols, t, c0);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const float2 st = stat[(c0 + k) & 15];
#pragma unroll
        for (int i = 0; i < R; ++i) got[i] += weight_of(p, c0 + k < cols ? s[k][i] : kNegInf, st);
      }
    }
    const int fades = fading_rows(p, x);
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (t + i < last) stg(p.c.mass + x.off + t + i, t + i < fades ? fmaf(p.decay, was[i], got[i]) : got[i]);
  }
};

// New rows from `first` on into the pools: those past the row bound, whose mass starts at 0.
template <int D, int NT>
__device__ __forceinline__ void append_rest(const MassAttn &p, const MassUnit &x, int u, int first, int tid) {
  const uint16_t *kn = new_rows(p, p.k, u), *vn = new_rows(p, p.v, u);
  const int n = x.held - max(first, x.len0);
  for (int e = tid; e < n * (D / 8); e += NT) {
    const int row = max(first, x.len0) + e / (D / 8), c = e % (D / 8);
    const int64_t to = (x.off + row) * D + 8 * c;
    st16(p.c.kp + to, ld16(kn + (int64_t)(row - x.len0) * p.k.token + 8 * c));
    st16(p.c.vp + to, ld16(vn + (int64_t)(row - x.len0) * p.v.token + 8 * c));
    if (c == 0) stg(p.c.mass + x.off + row, 0.f);
  }
}

// The unit of workgroup i, or -1.
__device__ __forceinline__ int unit_of(const MassAttn &p, int i) {
  const int u = p.order ? ldg(p.order + i) : i;
  return u < p.units ? u : -1;
}

// Workgroup (unit, piece): tiles [j piece, (j + 1) piece) of the unit, dealt to the waves in
// turn.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_token(MassAttn p) {
  using Sm = Smem<D, NW>;
  constexpr int NT = 64 * NW, KS = D / 32, MB = D / 16, CPR = D / 8, VIT = kMassTile * CPR / 64, VP = Sm::VP;
  constexpr int VH = kMassTile / Sm::VR, VN = VIT / VH;  // parts of a tile's values, chunks of each
  __shared__ Sm sm;
  const int u = unit_of(p, (int)(blockIdx.x % (uint32_t)p.units)), j = (int)(blockIdx.x / (uint32_t)p.units);
  if (u < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const MassUnit x = mass_unit(p, u);
  const int cols = x.cnt * p.G;
  const int emax = min(x.held, p.max_rows);
  const int nt = (emax + kMassTile - 1) / kMassTile;
  const int np = max((nt + p.piece - 1) / p.piece, 1);
  if (j >= np || cols == 0) return;
  if (emax == 0) {  // nothing to see: zeros
    for (int e = tid; e < cols * D; e += NT) put(p, mass_col(p, p.out, u, e / D) + e % D, 0.f);
    if (p.append) append_rest<D, NT>(p, x, u, 0, tid);
    if (p.npmax == 1) __syncthreads();  // (every thread has read the length)
    if (tid == 0) {
      if (p.npmax > 1)
        st16(p.state + u, u32x4{(uint32_t)x.len0, (uint32_t)x.held, (uint32_t)x.cnt, 1u});
      else if (p.append)
        stg(p.c.len + u, x.held);
    }
    return;
  }
  // Rows this lane's column sees, and the fewest any column does.
  auto sees = [&](int i) { return max(min(x.base + i + 1, emax), 0); };
  const int end = sees(min(lr, cols - 1) / p.G), emin = sees(0);
  const int t0 = j * p.piece, t1 = min(nt, t0 + p.piece);
  // Rows whose logits stay here, `pitch` a row (odd: no bank conflicts when read by rows).
  const int pitch = p.cols | 1;
  const int here = np > 1 ? 0 : p.here;
  // The query's requests, then the first tile's, before anything waits.
  u32x4 q[KS];
  {
    const uint16_t *qp = reinterpret_cast<const uint16_t *>(p.q.base) + mass_col(p, p.q, u, min(lr, cols - 1));
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = ld16(qp + 32 * s + 8 * lg);
  }
  const uint16_t *kp = p.c.kp + x.off * D, *vp = p.c.vp + x.off * D;
  const uint16_t *kn = kp, *vn = vp;  // new rows, by their row index
  int64_t kst = D, vst = D;
  if (p.append) {
    kst = p.k.token;
    vst = p.v.token;
    kn = new_rows(p, p.k, u) - x.len0 * kst;
    vn = new_rows(p, p.v, u) - x.len0 * vst;
  }
  // Tiles of old rows alone come from one address and a lane's constant offsets (the
  // general form's 64-bit products per row took half of a tile's instructions).
  u32x4 k[2][KS], v[VIT];
  const int whole = uniform(min(x.len0, emax) / kMassTile);
  const uint32_t ko = (uint32_t)(lr * D + 8 * lg), vo = (uint32_t)(8 * lane);
  const uint16_t *ku = uniform(kp), *vu = uniform(vp);
  auto load_k = [&](int t) {
    if (t < whole) {  // uniform
      const uint16_t *src = ku + (int64_t)t * (kMassTile * D);
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int s = 0; s < KS; ++s) k[rb][s] = ld16(src + ko + (16 * rb * D + 32 * s));
      return;
    }
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      const int row = min(t * kMassTile + 16 * rb + lr, emax - 1);
      const bool old = row < x.len0;
      const uint16_t *src = (old ? kp : kn) + row * (old ? (int64_t)D : kst) + 8 * lg;
#pragma unroll
      for (int s = 0; s < KS; ++s) k[rb][s] = ld16(src + 32 * s);
    }
  };
  auto load_v = [&](int t, int half) {
    if (t < whole) {
      const uint16_t *src = vu + (int64_t)t * (kMassTile * D);
#pragma unroll
      for (int it = half * VN; it < (half + 1) * VN; ++it) v[it] = ld16(src + vo + 512 * it);
      return;
    }
#pragma unroll
    for (int it = half * VN; it < (half + 1) * VN; ++it) {
      const int e = lane + 64 * it, row = min(t * kMassTile + e / CPR, emax - 1);
      const bool old = row < x.len0;
      v[it] = ld16((old ? vp : vn) + row * (old ? (int64_t)D : vst) + 8 * (e % CPR));
    }
  };
  // (Loads under a condition, or a query still on its way at the loop's head, would make
  // every turn wait for all that is in flight; a wave without a tile reads the last one.)
  int t = t0 + w;
  load_k(min(t, t1 - 1));
#pragma unroll
  for (int h = 0; h < VH; ++h) load_v(min(t, t1 - 1), h);
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[s]));
  const bool drafts = emin < emax;  // some column does not see every row
  if (drafts) {
    for (int c = tid; c < D; c += NT) sm.bad[c] = INT32_MAX;
    __syncthreads();
  }
  float m = kNegInf, l = 0.f;
  f32x4 O[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) O[mb] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint16_t *lv = reinterpret_cast<uint16_t *>(sm.buf) + w * Sm::VR * VP;
  float *far = p.logits + ((int64_t)u * p.cols + min(lr, cols - 1)) * p.ldr + 4 * lg - here;
  for (; t < t1; t += NW) {
    f32x4 S[2];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      S[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) S[rb] = mfma_bf16(as_bf16x8(k[rb][s]), as_bf16x8(q[s]), S[rb]);
    }
    const int r0 = t * kMassTile;
    if (r0 + kMassTile > x.len0) {  // new rows (uniform): into the pools as they pass
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        const int row = r0 + 16 * rb + lr;
        if (row >= x.len0 && row < emax)
#pragma unroll
          for (int s = 0; s < KS; ++s) st16(p.c.kp + (x.off + row) * D + 32 * s + 8 * lg, k[rb][s]);
      }
#pragma unroll
      for (int it = 0; it < VIT; ++it) {
        const int e = lane + 64 * it, row = r0 + e / CPR;
        if (row >= x.len0 && row < emax) st16(p.c.vp + (x.off + row) * D + 8 * (e % CPR), v[it]);
      }
    }
    const int tn = min(t + NW, t1 - 1);  // the last tile again where there is no next (never used)
    load_k(tn);
    if (r0 + kMassTile > emin) {  // uniform
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + 16 * (i / 4) + 4 * lg + i % 4 >= end) S[i / 4][i % 4] = kNegInf;
      if (drafts) {
#pragma unroll
        for (int it = 0; it < VIT; ++it) {
          const int e = lane + 64 * it;
          if (any_nonfinite(v[it]))
            v[it] = without_nonfinite(v[it], min(r0 + e / CPR, emax - 1), sm.bad + 8 * (e % CPR));
        }
      }
    }
    auto stage = [&](int half) {
#pragma unroll
      for (int it = half * VN; it < (half + 1) * VN; ++it) {
        const int e = lane + 64 * (it - half * VN);
        *reinterpret_cast<u32x4 *>(lv + (e / CPR) * VP + 8 * (e % CPR)) = v[it];
      }
      load_v(tn, half);
    };
    stage(0);
    if (lr < cols) {
      if (r0 < here) {  // uniform; `here` is a multiple of the tile
#pragma unroll
        for (int i = 0; i < 8; ++i) sm.logits[(r0 + 16 * (i / 4) + 4 * lg + i % 4) * pitch + lr] = S[i / 4][i % 4];
      } else {
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
          st16(far + r0 + 16 * rb, u32x4{__float_as_uint(S[rb][0]), __float_as_uint(S[rb][1]), __float_as_uint(S[rb][2]),
                                         __float_as_uint(S[rb][3])});
      }
    }
    float mx = S[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, S[i / 4][i % 4]);
    mx = max_halves(fmaxf(mx, swap16(mx))) * p.sc;
    const float mn = fmaxf(m, mx), ref = mn == kNegInf ? 0.f : mn;
    if (__builtin_amdgcn_ballot_w64(mn != m)) {  // some column's maximum moved
      const float alpha = fast_exp2(m - ref);
      l *= alpha;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) O[mb] *= alpha;
    }
    m = mn;
    float pr[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pr[i] = fast_exp2(fmaf(S[i / 4][i % 4], p.sc, -ref));
    // (Together first: small weights added one at a time to a long sum would be lost.)
    l += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
    u32x4 part[3];
#pragma unroll
    for (int y = 0; y < 3; ++y) {
      part[y] = u32x4{tops(pr[0], pr[1]), tops(pr[2], pr[3]), tops(pr[4], pr[5]), tops(pr[6], pr[7])};
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] -= top_of(pr[i]);  // exact
    }
    // O^T += V^T P^T.  (A wave's LDS accesses happen in their order, so between its writes
    // and reads only the compiler has to be kept from another one.)
    const uint16_t *tr = lv + (4 * lg + (lr >> 2)) * VP + 4 * (lr & 3);
    u32x2 a0[MB], a1[MB];
    wave_fence();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) a0[mb] = lds_transposed(tr + 16 * mb);
    if (VH == 2) {
      wave_fence();
      stage(1);
      wave_fence();
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) a1[mb] = lds_transposed(tr + 16 * mb + (VH == 2 ? 0 : 16 * VP));
    wave_fence();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const bf16x8 a = as_bf16x8(u32x4{a0[mb].x, a0[mb].y, a1[mb].x, a1[mb].y});
#pragma unroll
      for (int y = 0; y < 3; ++y) O[mb] = mfma_bf16(a, as_bf16x8(part[y]), O[mb]);
    }
  }
  // The masses that are added to at the end, requested already.
  constexpr int WAS = 4;
  const int near = min(emax, here);
  float was[WAS];
#pragma unroll
  for (int i = 0; i < WAS; ++i) was[i] = ldg(p.c.mass + x.off + min(tid + NT * i, emax - 1));
  l = sum_halves(l + swap16(l));
  if (lg == 0) sm.ml[w][lr] = make_float2(m, l);
  if (p.append && j == np - 1) append_rest<D, NT>(p, x, u, emax, tid);
  __threadfence_block();  // the logits in the workspace, for this workgroup
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();  // the values are read, the rows without finite values known
  if (drafts) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (sm.bad[16 * mb + 4 * lg + i] < end) O[mb][i] = __builtin_nanf("");
  }
  // The column's maximum and sum over all waves, and the waves' O relative to it.  (Without a
  // maximum there are no rows, all zeros, or only NaN, which stay.)
  float M = kNegInf, L = 0.f;
#pragma unroll
  for (int y = 0; y < NW; ++y) M = fmaxf(M, sm.ml[y][lr].x);
  const float ref = M == kNegInf ? 0.f : M;
#pragma unroll
  for (int y = 0; y < NW; ++y) L += fast_exp2(sm.ml[y][lr].x - ref) * sm.ml[y][lr].y;
  {
    const float f = fast_exp2(m - ref);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) O[mb] *= f;
  }
  float(*wo)[16][D + 4] = reinterpret_cast<float(*)[16][D + 4]>(sm.buf);
  if (NW == 8) {
    if (w >= 4) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) *reinterpret_cast<f32x4 *>(&wo[w & 3][lr][16 * mb + 4 * lg]) = O[mb];
    }
    __syncthreads();
    if (w < 4) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) O[mb] += *reinterpret_cast<const f32x4 *>(&wo[w][lr][16 * mb + 4 * lg]);
    }
  }
  if (w < 4) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) *reinterpret_cast<f32x4 *>(&wo[w & 3][lr][16 * mb + 4 * lg]) = O[mb];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int64_t slot = (int64_t)u * p.npmax + j;
  if (tid < cols) {  // (lr is the column)
    sm.stat[tid] = make_float2(ref, inv);
    if (np > 1) stg(p.part_ml + slot * 16 + tid, make_float2(M, L));
  }
  __syncthreads();
  const int ch = tid % D;
  for (int col = tid / D; col < cols; col += NT / D) {
    const float o = (wo[0][col][ch] + wo[1][col][ch]) + (wo[2][col][ch] + wo[3][col][ch]);
    const float y = sm.stat[col].y;
    if (np == 1)
      put(p, mass_col(p, p.out, u, col) + ch, y == 0.f ? 0.f : o * y);
    else
      stg(p.part_o + (slot * 16 + col) * D + ch, o);
  }
  if (tid == 0) {
    // The length: by the second launch where there is one, since other pieces read it.
    if (p.npmax == 1) {
      if (p.append) stg(p.c.len + u, x.held);
    } else if (j == np - 1) {
      st16(p.state + u, u32x4{(uint32_t)x.len0, (uint32_t)x.held, (uint32_t)x.cnt, (uint32_t)np});
    }
  }
  if (np > 1) return;
  const int fades = fading_rows(p, x);
  auto row_mass = [&](int r, float before) {
    const float *s = sm.logits + r * pitch;
    float got = 0.f;
    for (int c0 = 0; c0 < cols; c0 += 8) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = s[min(c0 + i, cols - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) got += weight_of(p, c0 + i < cols ? y[i] : kNegInf, sm.stat[(c0 + i) & 15]);
    }
    stg(p.c.mass + x.off + r, r < fades ? fmaf(p.decay, before, got) : got);
  };
#pragma unroll
  for (int i = 0; i < WAS; ++i)
    if (tid + NT * i < near) row_mass(tid + NT * i, was[i]);
  for (int r = tid + NT * WAS; r < near; r += NT) row_mass(r, ldg(p.c.mass + x.off + r));
  const float *lu = p.logits + (int64_t)u * p.cols * p.ldr;
  for (int r = here + 4 * tid; r < emax; r += 4 * NT) {
    MassRows<4> y;
    y.request(p, x, lu - here, cols, r, emax);
    y.finish(p, x, lu - here, sm.stat, cols, r, emax);
  }
}

// Workgroup (unit, chunk of rows) of a unit in several pieces: the columns that fall to
// the chunk from their pieces, 1024 / d at a time, and the chunk's masses.  Bound by
// latency, so all that it reads is requested at once, as soon as the unit is known.
template <int D, int R>
__global__ __launch_bounds__(kMassChunk) void k_finish(MassAttn p) {
  constexpr int NC = kMassChunk / D, U = 8;  // columns at a time, pieces in flight
  constexpr int kRows = kMassChunk * R;      // of a chunk
  __shared__ float2 ml[16];  // maximum and 1 / sum
  const int u = unit_of(p, (int)(blockIdx.x % (uint32_t)p.units)), ch = (int)(blockIdx.x / (uint32_t)p.units);
  if (u < 0) return;  // (nothing has written what its pieces leave)
  const int tid = threadIdx.x;
  const int cnt_ = p.count ? ldg(p.count + u / p.Hkv % p.B) : p.n;
  MassUnit x;
  x.off = ldg(p.c.row_off + u);
  const u32x4 st = ld16(p.state + u);
  if (cnt_ <= 0) return;  // (its pieces wrote nothing)
  x.len0 = (int)st.x, x.held = (int)st.y, x.cnt = (int)st.z;
  const int np = (int)st.w;
  if (ch == 0 && tid == 0 && p.append) stg(p.c.len + u, x.held);
  if (np <= 1) return;
  const int cols = x.cnt * p.G, emax = min(x.held, p.max_rows), nch = (emax - 1) / kRows + 1;
  if (ch >= nch) return;
  const int64_t slot = (int64_t)u * p.npmax;
  const float2 *pm = p.part_ml + slot * 16;
  const float *lu = p.logits + (int64_t)u * p.cols * p.ldr;
  const int r = ch * kRows + R * tid, rc = min(r, (emax - 1) / R * R);
  // Column tid / 16's pieces tid % 16, + 16, ...
  const int mc = min(tid / 16, cols - 1), m0 = tid % 16;
  const float2 a = ldg(pm + min(m0, np - 1) * 16 + mc);
  const int c = tid % D, col0 = ch + nch * (tid / D);
  float2 pa[U];
  float po[U];
  auto pieces = [&](int col, int y0) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int y = min(y0 + k, np - 1);
      pa[k] = ldg(pm + y * 16 + col);
      po[k] = ldg(p.part_o + ((slot + y) * 16 + col) * D + c);
    }
  };
  pieces(min(col0, cols - 1), 0);
  MassRows<R> rows;
  rows.request(p, x, lu, cols, rc, emax);
  if (tid < 256) {
    float M = m0 < np ? a.x : kNegInf, s = m0 < np ? a.y : 0.f;
    auto add = [&](float bm, float bs) {
      const float Mn = fmaxf(M, bm), ref = Mn == kNegInf ? 0.f : Mn;
      s = fast_exp2(M - ref) * s + fast_exp2(bm - ref) * bs;
      M = Mn;
    };
    for (int y = m0 + 16; y < np; y += 16) {
      const float2 b = ldg(pm + y * 16 + mc);
      add(b.x, b.y);
    }
#pragma unroll
    for (int y = 1; y < 16; y *= 2) add(shfl_xor(M, y), shfl_xor(s, y));
    if (m0 == 0 && tid / 16 < cols) ml[mc] = make_float2(M == kNegInf ? 0.f : M, s == 0.f ? 0.f : 1.f / s);
  }
  __syncthreads();
  for (int col = col0; col < cols; col += nch * NC) {
    const float2 b = ml[col];
    float o = 0.f;
    for (int y0 = 0; y0 < np; y0 += U) {
      if (col > col0 || y0 > 0) pieces(col, y0);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const float f = fast_exp2(pa[k].x - b.x) * po[k];
        o += y0 + k < np ? f : 0.f;
      }
    }
    put(p, mass_col(p, p.out, u, col) + c, b.y == 0.f ? 0.f : o * b.y);
  }
  if (r < emax) rows.finish(p, x, lu, ml, cols, r, emax);
}

template <int D>
hipError_t launch(const MassAttn &p, hipStream_t st) {
  if (p.waves == 8)
    hipLaunchKernelGGL((k_token<D, 8>), dim3((uint32_t)p.wgs), dim3(512), 0, st, p);
  else
    hipLaunchKernelGGL((k_token<D, 4>), dim3((uint32_t)p.wgs), dim3(256), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.npmax == 1) return e;
  if (p.finish == 4)
    hipLaunchKernelGGL((k_finish<D, 4>), dim3((uint32_t)p.finish_wgs), dim3(kMassChunk), 0, st, p);
  else
    hipLaunchKernelGGL((k_finish<D, 1>), dim3((uint32_t)p.finish_wgs), dim3(kMassChunk), 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mass_token(const MassAttn &p, hipStream_t st) {
  return p.d == 128 ? launch<128>(p, st) : launch<64>(p, st);
}

}  // namespace vc
