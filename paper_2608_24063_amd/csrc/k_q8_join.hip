// k_q8_join.hip -- joins the partial results (max, sum, O) that an attention
// over the 8-bit cache leaves for a column whose rows went to several
// workgroups.
//
// Bound by latency: a column's parts are dealt to groups of D / 4 lanes, four
// parts in flight each, so that a unit cut into many parts costs few round
// trips.  A launch of its own costs less than the last workgroup's joining them
// in the attention's launch did: there the partials need device-coherent
// stores, a wait for them and an atomic, and one workgroup joins a whole unit
// (4 units of 12544 rows, about 49 parts each: 18.5 us in one launch, 13.0 in two;
// units of few parts were not timed in one).  After a step it
// also advances the lengths, which every piece of a unit reads.
#include "vc_q8_device.h"

namespace vc {

namespace {

constexpr float kNegInf = -__builtin_inff();

struct Part {
  float M, l, o[4];
};

// What the parts' maxima are taken against: anything finite where there are no rows
// (their sums are zeros, or NaN, which stay).
__device__ __forceinline__ float against(float M) { return M == kNegInf ? 0.f : M; }

// b into a.
__device__ __forceinline__ void add(Part &a, const Part &b) {
  const float M = fmaxf(a.M, b.M), r = against(M);
  const float fa = fast_exp2(a.M - r), fb = fast_exp2(b.M - r);
  a.M = M;
  a.l = fa * a.l + fb * b.l;
#pragma unroll
  for (int i = 0; i < 4; ++i) a.o[i] = fa * a.o[i] + fb * b.o[i];
}

// WPC waves take a column: four where columns are few and parts many, one
// where the columns fill the chip.
template <int D, int WPC>
__global__ __launch_bounds__(256) void k_join(Q8Attn p) {
  constexpr int TPG = D / 4, GPW = 64 / TPG, NG = GPW * WPC, U = 4;
  __shared__ Part sp[WPC][TPG];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t cg = (int64_t)blockIdx.x * (4 / WPC) + w / WPC;
  const int i = (int)min(cg / p.cols, (int64_t)p.units - 1), col = (int)(cg % p.cols);
  // The units that the attention's launch took: nothing has written the parts of one
  // that its order leaves out.  (Prompts take all.)
  const int u = p.npmax > 1 && p.c.order ? ldg(p.c.order + i) : i;
  if (u < 0 || u >= p.units) return;
  const int grp = w % WPC * GPW + lane / TPG, ch = lane % TPG * 4;
  const int g = u % p.Hkv, lb = u / p.Hkv, b = lb % p.B;
  const int cnt_ = p.count ? ldg(p.count + b) : p.n;
  if (cg >= (int64_t)p.units * p.cols || col >= min(max(cnt_, 0), p.n) * p.G) return;
  int64_t at;  // part 0 of the column
  int ns;
  if (p.npmax > 1) {  // pieces: as many as the unit's rows make; a single one wrote its output
    if (p.step) {
      const int v = ldg(p.np + u);
      ns = v & 0x3FFFFFFF;
      if (col == 0 && (v >> 30) && lane == 0 && w % WPC == 0) stg(p.c.len + u, ldg(p.c.len + u) + 1);
    } else {
      const int rows = min(rows_held(ldg(p.c.len + u), ldg(p.c.cap + u)), p.max_rows);
      ns = ((rows + kQ8Block - 1) / kQ8Block + p.piece - 1) / p.piece;
    }
    at = (int64_t)u * p.npmax * p.qcols + col;
  } else {
    const u32x2 v = ld8(reinterpret_cast<const uint32_t *>(p.np) + 2 * (u * p.nqt + col / p.qcols));
    ns = (int)v.y;
    at = (int64_t)v.x * p.qcols + col % p.qcols;
  }
  if (ns <= 1) return;  // written already
  Part t{kNegInf, 0.f, {0.f, 0.f, 0.f, 0.f}};
  for (int s0 = grp; s0 < ns; s0 += NG * U) {
    float2 ml[U];
    float x[U][4];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t a = at + (int64_t)min(s0 + k * NG, ns - 1) * p.qcols;
      ml[k] = ldg(p.part_ml + a);
      const u32x4 v = ld16(p.part_o + a * D + ch);
      x[k][0] = __uint_as_float(v.x);
      x[k][1] = __uint_as_float(v.y);
      x[k][2] = __uint_as_float(v.z);
      x[k][3] = __uint_as_float(v.w);
    }
    float M = t.M;
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (s0 + k * NG < ns) M = fmaxf(M, ml[k].x);
    const float r = against(M), f0 = fast_exp2(t.M - r);
    t.M = M;
    t.l *= f0;
#pragma unroll
    for (int i = 0; i < 4; ++i) t.o[i] *= f0;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (s0 + k * NG >= ns) continue;
      const float f = fast_exp2(ml[k].x - r);
      t.l += f * ml[k].y;
#pragma unroll
      for (int i = 0; i < 4; ++i) t.o[i] += f * x[k][i];
    }
  }
  // The groups of a wave, then the waves.
#pragma unroll
  for (int d = TPG; d < 64; d *= 2) {
    Part y;
    y.M = shfl_xor(t.M, d);
    y.l = shfl_xor(t.l, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) y.o[i] = shfl_xor(t.o[i], d);
    add(t, y);
  }
  if (WPC > 1) {
    if (lane < TPG) sp[w][lane] = t;
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int k = 1; k < WPC; ++k) add(t, sp[k][lane % TPG]);
  }
  if (lane >= TPG) return;
  const float inv = t.l == 0.f ? 0.f : 1.f / t.l;
  const int64_t to = (int64_t)(lb / p.B) * p.out.layer + (int64_t)b * p.out.seq + (int64_t)(col / p.G) * p.out.token +
                     (int64_t)(g * p.G + col % p.G) * p.out.head + ch;
  const float v[4] = {t.o[0] * inv, t.o[1] * inv, t.o[2] * inv, t.o[3] * inv};
  if (p.fp32)
    st16(reinterpret_cast<float *>(p.out.base) + to,
         u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
  else
    st8(reinterpret_cast<uint16_t *>(p.out.base) + to, u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])});
}

template <int D>
void launch(const Q8Attn &p, hipStream_t st) {
  const int64_t cols = (int64_t)p.units * p.cols;
  // 1024 columns and more are a wave each: 5460 columns of 12 parts take 13.2 us
  // in four waves, 6.9 in one; 28 columns of 49 to 125 parts need the four.
  if (cols >= 1024)
    hipLaunchKernelGGL((k_join<D, 1>), dim3((uint32_t)((cols + 3) / 4)), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((k_join<D, 4>), dim3((uint32_t)cols), dim3(256), 0, st, p);
}

}  // namespace

hipError_t launch_q8_join(const Q8Attn &p, hipStream_t st) {
  if (p.d == 128)
    launch<128>(p, st);
  else
    launch<64>(p, st);
  return hipGetLastError();
}

}  // namespace vc
