// k_mass_token.hip -- attention over a bf16 cache for single tokens (up to 16 (token,
// query head) columns per kv head) that also adds what every row was given to the
// row's mass, and appends the tokens' own rows on its way.
//
// A row's weight, exp(s - m) / l, is known only after the last row, and to compute the
// logits again would read the keys again.  So the logits, 4 bytes a column and row
// beside the row's 4 d, wait in the workspace until the maximum and the sum are known.
// Where a unit is one workgroup's the same workgroup comes back to them; where it is
// cut, a second launch joins the outputs and adds the weights up.
//
// Bound by memory: a wave takes tiles of 32 rows, keys straight into the A operands of
//   S^T = K Q^T,  O^T = V^T P^T  (16x16x32),
// values through LDS, read back transposed; the next tile is requested as soon as a
// tile's registers are free.  P enters in three bf16 parts, cut and not rounded, which
// hold all 24 bits of a weight; logits, sums, O and masses are fp32.
#include "vc_mass_device.h"

namespace vc {

namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr int kWaves = 4;

template <int D>
struct Smem {
  static constexpr int VP = D + 16;  // pitch of the values: conflict-free transposing reads
  static constexpr size_t kO = sizeof(float) * kWaves * 16 * (D + 4);
  static constexpr size_t kT = sizeof(uint16_t) * kWaves * kMassTile * VP;
  uint8_t buf[kO > kT ? kO : kT] __attribute__((aligned(16)));  // the waves' values, then their O
  float2 ml[kWaves][16];
  float2 stat[16];  // maximum and 1 / sum of each column
  int32_t bad[D];   // (without_nonfinite)
};

__device__ __forceinline__ void put(const MassAttn &p, int64_t at, float v) {
  if (p.fp32)
    stg(reinterpret_cast<float *>(p.out.base) + at, v);
  else
    stg(reinterpret_cast<uint16_t *>(p.out.base) + at, (uint16_t)pack_bf16(v, 0.f));
}

// What row t of a unit was given by all columns, from their logits.  (A logit of -inf
// is a row that its column does not see, also where the column's sum is NaN.)
__device__ __forceinline__ float row_weight(const MassAttn &p, const float *logits, const float2 *stat, int cols, int t) {
  float got = 0.f;
  for (int c = 0; c < cols; ++c) {
    const float s = ldg(logits + (int64_t)c * p.ldr + t);
    const float2 st = stat[c];
    got += s == kNegInf ? 0.f : fast_exp2(fmaf(s, p.sc, -st.x)) * st.y;
  }
  return got;
}

__device__ __forceinline__ void add_mass(const MassAttn &p, const MassUnit &x, int t, float got) {
  float *m = p.c.mass + x.off + t;
  stg(m, t < x.len0 ? fmaf(p.decay, ldg(m), got) : got);
}

// New rows from `first` on into the pools: those past the row bound, whose mass starts at 0.
template <int D>
__device__ __forceinline__ void append_rest(const MassAttn &p, const MassUnit &x, int u, int first, int tid) {
  const uint16_t *kn = new_rows(p, p.k, u), *vn = new_rows(p, p.v, u);
  const int n = x.held - max(first, x.len0);
  for (int e = tid; e < n * (D / 8); e += 64 * kWaves) {
    const int row = max(first, x.len0) + e / (D / 8), c = e % (D / 8);
    const int64_t to = (x.off + row) * D + 8 * c;
    st16(p.c.kp + to, ld16(kn + (int64_t)(row - x.len0) * p.k.token + 8 * c));
    st16(p.c.vp + to, ld16(vn + (int64_t)(row - x.len0) * p.v.token + 8 * c));
    if (c == 0) stg(p.c.mass + x.off + row, 0.f);
  }
}

// Workgroup (unit, piece): tiles [j piece, (j + 1) piece) of the unit, dealt to the four
// waves in turn.
template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void k_token(MassAttn p) {
  constexpr int KS = D / 32, MB = D / 16, CPR = D / 8, VIT = kMassTile * CPR / 64, VP = Smem<D>::VP;
  __shared__ Smem<D> sm;
  const int u = (int)(blockIdx.x % (uint32_t)p.units), j = (int)(blockIdx.x / (uint32_t)p.units);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const MassUnit x = mass_unit(p, u);
  const int cols = x.cnt * p.G;
  const int emax = min(x.held, p.max_rows);
  const int nt = (emax + kMassTile - 1) / kMassTile;
  const int np = max((nt + p.piece - 1) / p.piece, 1);
  if (j >= np || cols == 0) return;
  // Rows this lane's column sees, and the fewest any column does.
  auto sees = [&](int i) { return max(min(x.base + i + 1, emax), 0); };
  const int end = sees(min(lr, cols - 1) / p.G), emin = sees(0);
  const int t0 = j * p.piece, t1 = min(nt, t0 + p.piece);
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
  u32x4 k[2][KS], v[VIT];
  auto load_k = [&](int t) {
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      const int row = min(t * kMassTile + 16 * rb + lr, emax - 1);
      const uint16_t *src = row < x.len0 ? kp + (int64_t)row * D : kn + row * kst;
#pragma unroll
      for (int s = 0; s < KS; ++s) k[rb][s] = ld16(src + 32 * s + 8 * lg);
    }
  };
  auto load_v = [&](int t) {
#pragma unroll
    for (int it = 0; it < VIT; ++it) {
      const int e = lane + 64 * it, row = min(t * kMassTile + e / CPR, emax - 1);
      v[it] = ld16((row < x.len0 ? vp + (int64_t)row * D : vn + row * vst) + 8 * (e % CPR));
    }
  };
  int t = t0 + w;
  if (t < t1) {
    load_k(t);
    load_v(t);
  }
  const bool drafts = emin < emax;  // some column does not see every row
  if (drafts) {
    for (int c = tid; c < D; c += 64 * kWaves) sm.bad[c] = INT32_MAX;
    __syncthreads();
  }
  float m = kNegInf, l = 0.f;
  f32x4 O[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) O[mb] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint16_t *lv = reinterpret_cast<uint16_t *>(sm.buf) + w * kMassTile * VP;
  float *lo_ = p.logits + ((int64_t)u * p.cols + min(lr, cols - 1)) * p.ldr + 4 * lg;
  for (; t < t1; t += kWaves) {
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
    const int tn = min(t + kWaves, t1 - 1);  // the last tile again where there is no next (never used)
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
#pragma unroll
    for (int it = 0; it < VIT; ++it) {
      const int e = lane + 64 * it;
      *reinterpret_cast<u32x4 *>(lv + (e / CPR) * VP + 8 * (e % CPR)) = v[it];
    }
    load_v(tn);
    if (lr < cols) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
        st16(lo_ + r0 + 16 * rb, u32x4{__float_as_uint(S[rb][0]), __float_as_uint(S[rb][1]), __float_as_uint(S[rb][2]),
                                       __float_as_uint(S[rb][3])});
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
    for (int i = 0; i < 8; ++i) {
      pr[i] = fast_exp2(fmaf(S[i / 4][i % 4], p.sc, -ref));
      l += pr[i];
    }
    u32x4 part[3];
#pragma unroll
    for (int y = 0; y < 3; ++y) {
      part[y] = u32x4{tops(pr[0], pr[1]), tops(pr[2], pr[3]), tops(pr[4], pr[5]), tops(pr[6], pr[7])};
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] -= top_of(pr[i]);  // exact
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's LDS writes landed
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const uint16_t *base = lv + (4 * lg + (lr >> 2)) * VP + 16 * mb + 4 * (lr & 3);
      const u32x2 a0 = lds_transposed(base), a1 = lds_transposed(base + 16 * VP);
      const bf16x8 a = as_bf16x8(u32x4{a0.x, a0.y, a1.x, a1.y});
#pragma unroll
      for (int y = 0; y < 3; ++y) O[mb] = mfma_bf16(a, as_bf16x8(part[y]), O[mb]);
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // reads done before the next tile's writes
    __builtin_amdgcn_wave_barrier();
  }
  l = sum_halves(l + swap16(l));
  __syncthreads();  // the values are read, the rows without finite values known
  if (drafts) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (sm.bad[16 * mb + 4 * lg + i] < end) O[mb][i] = __builtin_nanf("");
  }
  float(*wo)[16][D + 4] = reinterpret_cast<float(*)[16][D + 4]>(sm.buf);
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) *reinterpret_cast<f32x4 *>(&wo[w][lr][16 * mb + 4 * lg]) = O[mb];
  if (lg == 0) sm.ml[w][lr] = make_float2(m, l);
  if (p.append && j == np - 1) append_rest<D>(p, x, u, emax, tid);
  __threadfence_block();  // the logits, for this workgroup
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  const int ch = tid % D;
  const int64_t slot = (int64_t)u * p.npmax + j;
  for (int col = tid / D; col < cols; col += 64 * kWaves / D) {
    float M = kNegInf;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) M = fmaxf(M, sm.ml[y][col].x);
    // (Without a maximum there are no rows, all zeros, or only NaN, which stay.)
    const float ref = M == kNegInf ? 0.f : M;
    float o = 0.f, s = 0.f;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
      const float f = fast_exp2(sm.ml[y][col].x - ref);
      o += f * wo[y][col][ch];
      s += f * sm.ml[y][col].y;
    }
    if (np == 1) {
      const float inv = s == 0.f ? 0.f : 1.f / s;
      put(p, mass_col(p, p.out, u, col) + ch, s == 0.f ? 0.f : o * inv);
      if (ch == 0) sm.stat[col] = make_float2(ref, inv);
    } else {
      stg(p.part_o + (slot * 16 + col) * D + ch, o);
      if (ch == 0) stg(p.part_ml + slot * 16 + col, make_float2(M, s));
    }
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
  __syncthreads();
  const float *lu = p.logits + (int64_t)u * p.cols * p.ldr;
  for (int r = tid; r < emax; r += 64 * kWaves) add_mass(p, x, r, row_weight(p, lu, sm.stat, cols, r));
}

// Workgroup (unit, chunk of rows) of a unit in several pieces: the columns that fall to
// the chunk from their pieces, and the chunk's masses.
template <int D>
__global__ __launch_bounds__(256) void k_finish(MassAttn p) {
  constexpr int NG = 256 / D;
  __shared__ float2 ml[16];  // maximum and 1 / sum
  __shared__ float red[NG][D];
  const int u = (int)(blockIdx.x % (uint32_t)p.units), ch = (int)(blockIdx.x / (uint32_t)p.units);
  const int tid = threadIdx.x;
  const int cnt_ = p.count ? ldg(p.count + u / p.Hkv % p.B) : p.n;
  if (cnt_ <= 0) return;  // (its pieces wrote nothing)
  MassUnit x;
  x.off = ldg(p.c.row_off + u);
  const u32x4 st = ld16(p.state + u);
  x.len0 = (int)st.x, x.held = (int)st.y, x.cnt = (int)st.z;
  const int np = (int)st.w;
  if (ch == 0 && tid == 0 && p.append) stg(p.c.len + u, x.held);
  if (np <= 1) return;
  const int cols = x.cnt * p.G, emax = min(x.held, p.max_rows), nch = (emax + kMassChunk - 1) / kMassChunk;
  if (ch >= nch) return;
  const int64_t slot = (int64_t)u * p.npmax;
  const float2 *pm = p.part_ml + slot * 16;
  {
    const int col = min(tid / 16, cols - 1);
    float M = kNegInf, s = 0.f;
    for (int y = tid % 16; y < np; y += 16) M = fmaxf(M, ldg(pm + y * 16 + col).x);
#pragma unroll
    for (int y = 1; y < 16; y *= 2) M = fmaxf(M, shfl_xor(M, y));
    const float ref = M == kNegInf ? 0.f : M;
    for (int y = tid % 16; y < np; y += 16) {
      const float2 a = ldg(pm + y * 16 + col);
      s += fast_exp2(a.x - ref) * a.y;
    }
#pragma unroll
    for (int y = 1; y < 16; y *= 2) s += shfl_xor(s, y);
    if (tid % 16 == 0 && tid / 16 < cols) ml[col] = make_float2(ref, s == 0.f ? 0.f : 1.f / s);
  }
  __syncthreads();
  const int c = tid % D, grp = tid / D;
  for (int col = ch; col < cols; col += nch) {  // uniform
    const float2 a = ml[col];
    float o = 0.f;
#pragma unroll 4
    for (int y = grp; y < np; y += NG)
      o += fast_exp2(ldg(pm + y * 16 + col).x - a.x) * ldg(p.part_o + ((slot + y) * 16 + col) * D + c);
    red[grp][c] = o;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int y = 1; y < NG; ++y) o += red[y][c];
      put(p, mass_col(p, p.out, u, col) + c, a.y == 0.f ? 0.f : o * a.y);
    }
    __syncthreads();
  }
  const float *lu = p.logits + (int64_t)u * p.cols * p.ldr;
  const int last = min(emax, (ch + 1) * kMassChunk);
  for (int r = ch * kMassChunk + tid; r < last; r += 256) add_mass(p, x, r, row_weight(p, lu, ml, cols, r));
}

template <int D>
hipError_t launch(const MassAttn &p, hipStream_t st) {
  hipLaunchKernelGGL((k_token<D>), dim3((uint32_t)p.wgs), dim3(64 * kWaves), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.npmax == 1) return e;
  const int64_t chunks = ((int64_t)p.max_rows + kMassChunk - 1) / kMassChunk;
  hipLaunchKernelGGL((k_finish<D>), dim3((uint32_t)(p.units * chunks)), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mass_token(const MassAttn &p, hipStream_t st) {
  return p.d == 128 ? launch<128>(p, st) : launch<64>(p, st);
}

}  // namespace vc
