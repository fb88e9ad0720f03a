// k_mass_evict.hip -- eviction by mass: unit u keeps k = keep[u] of its n rows, the first
// `sinks`, the last `recent` and of the others those of the largest mass (ties to the
// lower index, NaN behind every number), in order, in place or into another cache.
//
// k_choose, a workgroup a unit, finds the threshold exactly: a most-significant-digit radix
// select over the masses' bits (digits of 11, 11 and 10 bits, counted in LDS), then one
// pass that gives every kept row its place by ballots and prefix sums.  A chain of LDS
// round trips bounds it (us: 8 units of 200 rows 6, 112 of 2400 to 3136 rows 7.4, 896 of
// 2300 to 5800 19.5; with every pass reading the masses again 6, 9.4, 43).
//
// k_move copies the rows, a workgroup 32 KB of keys and 32 of values, and is bound by
// memory: half of those 896 units into another cache 446 us (5.7 TB/s read and written);
// 0.6 of the 112 in place 47 (4.5 TB/s).
//
// In place a row's new place may hold a row that has yet to move.  Rows only move down and
// keep their order, so the rows of a chunk of new places come from that chunk or later
// ones, and what a chunk writes over is read by itself and by earlier chunks of its unit
// alone.  So a workgroup reads its rows into registers, says so, waits until all earlier
// chunks of the unit have said so, and writes.  A unit's chunks are handed out by a counter
// of its own: a workgroup that waits was handed a later chunk than those it waits for,
// which were handed to workgroups that run already and say so without waiting for
// anything.  (One counter for all units takes 14 ns a workgroup, which follow one another:
// 83 us against 56 for the 112 units, in chunks of 16 KB.)
#include <algorithm>

#include "vc_mass_device.h"

namespace vc {

namespace {

// (us of the 112 units in place and the 896 into another cache, chunks of 16 KB by 256
// threads 56 -, 32 KB by 512 47 446, 64 KB by 1024 44 467.)
constexpr int kMoveThreads = 512;

// A mass as a key that orders like it: NaN lowest, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float m) {
  if (m != m) return 0u;
  const uint32_t x = __float_as_uint(m + 0.f);
  return (x & 0x80000000u) ? ~x : x | 0x80000000u;
}

template <int NT>
__global__ __launch_bounds__(NT) void k_choose(EvictPlan p) {
  constexpr int kWaves = NT / 64, kBins = 2048;
  __shared__ __attribute__((aligned(16))) uint32_t hist[kBins];
  __shared__ uint32_t found[2], tot[2][kWaves][2];
  const int u = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len_ = ldg(p.c.len + u), cap_ = ldg(p.c.cap + u), keep_ = ldg(p.keep + u);
  const int room = p.inplace ? INT32_MAX : ldg(p.to.cap + u);
  const float *mass = p.c.mass + ldg(p.c.row_off + u);
  const int n = max(min(min(len_, cap_), p.max_rows), 0);
  const int k = max(min(min(keep_, n), room), 0);
  const int a = min(p.sinks, k), z = min(p.recent, k - a), mid = n - z;  // rows a .. mid - 1 compete
  uint32_t T = 0u, left = (uint32_t)(k - a - z);  // the threshold; rows wanted among those equal to it
  if (left == 0u) T = ~0u;  // above every key
  // For the launch after this one: nobody has read a row, no chunk is handed out.
  if (p.inplace) {
    for (int i = tid; i < p.chunks; i += NT) stg(p.flags + (int64_t)u * p.chunks + i, 0u);
    if (tid == 0) stg(p.ticket + u, 0u);
  }
  // A wave takes 256 rows of a tile of 4 NT, 64 at a time.  The keys of two tiles stay in
  // registers, further ones are read again in each pass.
  constexpr int kTile = 4 * NT, kHeld = 2;
  const int mine = 256 * w + lane;  // the lane's first row in a tile
  uint32_t held[kHeld][4];
  auto keys = [&](int t0, uint32_t (&x)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = key_of(ldg(mass + min(t0 + mine + 64 * j, n - 1)));
  };
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (h * kTile < n) keys(h * kTile, held[h]);  // uniform
  if (left > 0u && left < (uint32_t)(mid - a)) {  // uniform
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int sh = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t bins = pass == 2 ? 1024u : 2048u, known = pass == 0 ? 0u : ~0u << (pass == 1 ? 21 : 10);
      for (int i = 4 * tid; i < kBins; i += 4 * NT) *reinterpret_cast<u32x4 *>(hist + i) = u32x4{0u, 0u, 0u, 0u};
      __syncthreads();
      auto count = [&](int t0, const uint32_t (&x)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = t0 + mine + 64 * j;
          if (t >= a && t < mid && (x[j] & known) == T) atomicAdd(&hist[x[j] >> sh & (bins - 1u)], 1u);
        }
      };
#pragma unroll
      for (int h = 0; h < kHeld; ++h)
        if (h * kTile < n) count(h * kTile, held[h]);
      for (int t0 = kHeld * kTile; t0 < n; t0 += kTile) {
        uint32_t x[4];
        keys(t0, x);
        count(t0, x);
      }
      __syncthreads();
      if (w == 0) {  // the bin that holds rank `left` from the top: lane l sums bins of 32 in descending order
        uint32_t sum = 0u;
        for (int i = 0; i < kBins / 64; i += 4) {
          const u32x4 h = *reinterpret_cast<const u32x4 *>(hist + kBins - kBins / 64 * (lane + 1) + i);
          sum += (h.x + h.y) + (h.z + h.w);
        }
        const uint32_t incl = wave_incl_scan(sum);
        const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(incl - sum < left && left <= incl));
        const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)(incl - sum), src);
        const int bin = kBins - 1 - kBins / 64 * src - lane;
        const uint32_t h = lane < kBins / 64 ? hist[max(bin, 0)] : 0u;
        const uint32_t in2 = wave_incl_scan(h) + before;
        const uint64_t hit = __builtin_amdgcn_ballot_w64(in2 - h < left && left <= in2);
        if (lane == __builtin_ctzll(hit)) {
          found[0] = (uint32_t)bin;
          found[1] = left - (in2 - h);
        }
      }
      __syncthreads();
      T |= found[0] << sh;
      left = found[1];
    }
  }
  // Every kept row's place.
  int32_t *list = p.list + (int64_t)u * p.ldl;
  int32_t *index = p.index ? p.index + (int64_t)u * p.index_rows : nullptr;
  uint32_t kept = 0u, equal = 0u;  // before the tile
  auto places = [&](int t0, int it, const uint32_t (&x)[4]) {
    uint64_t sure[4], tie[4];
    uint32_t ns = 0u, ne = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = t0 + mine + 64 * j;
      const bool in = t >= a && t < mid;
      sure[j] = __builtin_amdgcn_ballot_w64(t < n && (!in || x[j] > T));
      tie[j] = __builtin_amdgcn_ballot_w64(in && x[j] == T);
      ns += (uint32_t)__builtin_popcountll(sure[j]);
      ne += (uint32_t)__builtin_popcountll(tie[j]);
    }
    if (lane == 0) tot[it][w][0] = ns, tot[it][w][1] = ne;
    __syncthreads();
    uint32_t bs = kept, be = equal;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
      const uint32_t s = tot[it][y][0], e = tot[it][y][1];
      if (y < w) bs += s, be += e;
      kept += s, equal += e;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t below = ((uint64_t)1 << lane) - 1;
      const uint32_t s = bs + (uint32_t)__builtin_popcountll(sure[j] & below);
      const uint32_t e = be + (uint32_t)__builtin_popcountll(tie[j] & below);
      const bool is = sure[j] >> lane & 1, ie = (tie[j] >> lane & 1) && e < left;
      const uint32_t at = s + min(e, left);
      if ((is || ie) && at < (uint32_t)k) {
        const int t = t0 + mine + 64 * j;
        stg(list + at, t);
        if (index && at < (uint32_t)p.index_rows) stg(index + at, t);
      }
      bs += (uint32_t)__builtin_popcountll(sure[j]);
      be += (uint32_t)__builtin_popcountll(tie[j]);
    }
  };
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (h * kTile < n) places(h * kTile, h & 1, held[h]);
  for (int t0 = kHeld * kTile, it = 0; t0 < n; t0 += kTile, it ^= 1) {
    uint32_t x[4];
    keys(t0, x);
    places(t0, it, x);
  }
  if (tid == 0) {
    stg(p.count + u, k);
    stg((p.inplace ? p.c.len : p.to.len) + u, k);
  }
}

template <int D, bool INPLACE>
__global__ __launch_bounds__(kMoveThreads) void k_move(EvictPlan p) {
  constexpr int CPR = D / 8, R = kEvictBytes / (2 * D), IT = R * CPR / kMoveThreads;  // rows of a chunk
  __shared__ uint32_t mine;
  __shared__ int32_t from[R];
  const int tid = threadIdx.x;
  const int u = (int)(blockIdx.x / (uint32_t)p.chunks);
  int c = (int)(blockIdx.x % (uint32_t)p.chunks);
  const int k = ldg(p.count + u);
  if (INPLACE) {
    if (c * R >= k) return;  // as many stay as there are chunks
    if (tid == 0) mine = __hip_atomic_fetch_add(p.ticket + u, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    c = (int)mine;
  }
  const int j0 = c * R;
  if (j0 >= k) return;
  const int nr = min(R, k - j0);
  const int64_t src = ldg(p.c.row_off + u), dst = INPLACE ? src : ldg(p.to.row_off + u);
  for (int i = tid; i < R; i += kMoveThreads) from[i] = ldg(p.list + (int64_t)u * p.ldl + j0 + min(i, nr - 1));
  __syncthreads();
  u32x4 kr[IT], vr[IT];
  float m = 0.f;
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int e = tid + kMoveThreads * it;
    const int64_t at = (src + from[e / CPR]) * D + 8 * (e % CPR);
    kr[it] = ld16_stream(p.c.kp + at);
    vr[it] = ld16_stream(p.c.vp + at);
  }
  if (tid < nr) m = ldg(p.c.mass + src + from[tid]);
  if (INPLACE) {
    // The rows are in registers before the barrier: what uses them here waits for them.
#pragma unroll
    for (int it = 0; it < IT; ++it) asm volatile("" : "+v"(kr[it]), "+v"(vr[it]) : : "memory");
    asm volatile("" : "+v"(m) : : "memory");
    __syncthreads();
    uint32_t *flag = p.flags + (int64_t)u * p.chunks;
    if (tid == 0) __hip_atomic_store(flag + c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i = tid; i < c; i += kMoveThreads)
      while (__hip_atomic_load(flag + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0u) __builtin_amdgcn_s_sleep(1);
    __syncthreads();
  }
  const MassPool &to = INPLACE ? p.c : p.to;
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int e = tid + kMoveThreads * it, i = e / CPR;
    if (i >= nr || (INPLACE && from[i] == j0 + i)) continue;
    const int64_t at = (dst + j0 + i) * D + 8 * (e % CPR);
    st16_stream(to.kp + at, kr[it]);
    st16_stream(to.vp + at, vr[it]);
  }
  if (tid < nr) stg(to.mass + dst + j0 + tid, m);
}

template <int D>
void launch_move(const EvictPlan &p, hipStream_t st) {
  const dim3 grid((uint32_t)(p.units * p.chunks));
  if (p.inplace)
    hipLaunchKernelGGL((k_move<D, true>), grid, dim3(kMoveThreads), 0, st, p);
  else
    hipLaunchKernelGGL((k_move<D, false>), grid, dim3(kMoveThreads), 0, st, p);
}

}  // namespace

hipError_t launch_mass_evict(const EvictPlan &p, hipStream_t st) {
  // More threads where few units are long.  (us, 512 and 1024 threads: 8 units of 25000 rows
  // 34.4 28.0, 64 of 12000 17.8 14.4, 112 of 3000 7.4 7.1, 256 of 5000 10.8 11.2, 504 of 2500
  // 10.7 13.8, 600 of 3000 13.5 19.5, 912 of 12000 43 56; 256 and 512: 112 of 3000 11.0 7.4.)
  const dim3 grid((uint32_t)p.units);
  if (p.max_rows <= 2048)
    hipLaunchKernelGGL((k_choose<256>), grid, dim3(256), 0, st, p);
  else if (p.max_rows <= 8192 || p.units > 256)
    hipLaunchKernelGGL((k_choose<512>), grid, dim3(512), 0, st, p);
  else
    hipLaunchKernelGGL((k_choose<1024>), grid, dim3(1024), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.chunks == 0) return e;
  if (p.d == 128)
    launch_move<128>(p, st);
  else
    launch_move<64>(p, st);
  return hipGetLastError();
}

}  // namespace vc
