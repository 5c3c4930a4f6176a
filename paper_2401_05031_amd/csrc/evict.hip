// Eviction from the cache: which entries stay (one workgroup a query), then the moves (many).
#include "common.h"
#include "decode_kernels.h"
#include "plan_args.h"

namespace otas {

// ------------------------------------------------------------------------------------------------- which entries stay
// Scores become unsigned numbers in the same order (NaN lowest, protected entries highest and alike), which stay in LDS up to 32768 entries
// (beyond that they are formed again in every pass).  The keep-th largest of them is found by 11, 11 and 10 bits, highest first: a
// histogram of the bits over the entries that agree with those found so far (integer counts: any order gives the same), and a
// scan from its top.  Bytes would take a fourth pass, and the highest of them is little but the exponent: weights of one
// order of magnitude would all meet in one counter.  Of the entries equal to the keep-th the lowest stay.  Then every wave goes
// through a run of its own of the entries twice, counting and then writing the places below keep that fall free and the entries above
// that move there, in rising order.
//   One workgroup's LDS reads, barriers and ballots: 7.2 us for 1000 entries, 21.8 for 16 queries of 16000 (2 of them the loads, 7 the
// three passes, 8 the two walks at the end).  Sums over the waves in one step in place of a loop, one walk of counting in place of
// two and the waves' numbers in scalars took 1.1 and 2.4 us off.  Past 32768 entries the one workgroup
// reads them five times: a cache of 500000 entries cut by a fiftieth takes 670 us, 33000 51 us, 32000 40.
constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64, kEvictBins = 2048, kEvictInLds = 32768;

struct EvictQuery {
  const float* mass;
  const int32_t* positions;
  int n, keep, lead, recent_from;
  bool has_recent;
  __device__ uint32_t rank(int j) const {   // both loads at once, no branch
    const float m = mass[j] + 0.f;          // -0 and 0 are equal
    const int p = positions[j];
    const uint32_t b = __float_as_uint(m), sign = (uint32_t)((int)b >> 31);
    const uint32_t r = m != m ? 0u : b ^ (sign | 0x80000000u);   // -inf: 0x007FFFFF, inf: 0xFF800000
    return (j < lead) | (has_recent & (p >= recent_from)) ? 0xFFFFFFFFu : r;
  }
};

// The sum over every 16 lanes, in all of them; the sum over those up to the lane's.
template <int ROTATION> __device__ __forceinline__ int rotated16(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + ROTATION, 0xF, 0xF, false); }
__device__ __forceinline__ int sum16(int x) {
  x += rotated16<8>(x); x += rotated16<4>(x); x += rotated16<2>(x);
  return x + rotated16<1>(x);
}
__device__ __forceinline__ int upto16(int x, int lane) {
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    const int y = __shfl_up(x, d, 16);
    if ((lane & 15) >= d) x += y;
  }
  return x;
}
static_assert(kEvictWaves == 16, "a lane of 16 for every wave");

template <bool IN_LDS, typename P>
__global__ __launch_bounds__(kEvictThreads) void cache_evict_select_kernel(CacheRef c, P plan, int B, int lead, bool has_recent,
                                                                           int32_t* __restrict__ lists) {
  extern __shared__ __attribute__((aligned(16))) uint32_t ranks[];   // [n] where they fit
  __shared__ int hist[kEvictBins];
  __shared__ uint32_t found;
  __shared__ int above;
  __shared__ int sums[4][kEvictWaves];
  const int q = (int)blockIdx.x, tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int64_t slot = plan[q];
  const int n = plan[B + q], keep = plan[2 * B + q];
  if (keep >= n || keep == 0) {   // workgroup-uniform
    if (tid == 0) lists[q] = 0;
    return;
  }
  const EvictQuery eq{c.mass + slot * c.capacity, c.positions + slot * c.capacity, n, keep, lead, plan[3 * B + q], has_recent};
  if (IN_LDS) {
#pragma unroll 4
    for (int j = tid; j < n; j += kEvictThreads) ranks[j] = eq.rank(j);
  }
  auto rank = [&](int j) { return IN_LDS ? ranks[j] : eq.rank(j); };
  if (tid == 0) { found = 0; above = 0; }
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
    const uint32_t agree = pass == 0 ? 0u : pass == 1 ? ~0u << 21 : ~0u << 10;
    for (int i = tid; i < bins; i += kEvictThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t prefix = found;
    const int had = above;
#pragma unroll 4
    for (int j = tid; j < n; j += kEvictThreads) {
      const uint32_t r = rank(j);
      if ((r & agree) == prefix) atomicAdd(&hist[(r >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    // The bin of the keep-th largest: as many as possible above it, fewer than keep.  Thread t has the two bins 2 t from the top.
    const bool has = 2 * tid < bins;
    const int hi = has ? hist[bins - 1 - 2 * tid] : 0, lo = has ? hist[bins - 2 - 2 * tid] : 0;
    int upto = hi + lo;
    for (int d = 1; d < 64; d <<= 1) {
      const int x = __shfl_up(upto, d);
      if (lane >= d) upto += x;
    }
    if (lane == 63) sums[0][wave] = upto;
    __syncthreads();
    upto += sum16((lane & 15) < wave ? sums[0][lane & 15] : 0);
    const int before = had + upto - hi - lo;
    if (has && before < keep && had + upto >= keep) {   // one thread
      const bool low = before + hi < keep;
      above = low ? before + hi : before;
      found = prefix | ((uint32_t)(bins - 1 - 2 * tid - (low ? 1 : 0)) << shift);
    }
    __syncthreads();
  }
  const uint32_t edge = found;
  const int equal_kept = keep - above;   // >= 1 of those equal to the edge stay
  // Every wave's run of whole blocks of 64 entries.  Counted: those equal to the edge, those of them below keep, the smaller ones below
  // keep and the larger ones above.
  const int blocks = (n + 63) >> 6, per = (blocks + kEvictWaves - 1) / kEvictWaves;
  const int b0 = wave * per, b1 = min(blocks, b0 + per);
  constexpr int AT_ONCE = 4;
  auto walk = [&](auto f) {   // f(entry, rank, entries of the block below keep, lanes past the end)
    for (int b = b0; b < b1; b += AT_ONCE) {
      uint32_t r[AT_ONCE];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) r[u] = rank(min((b + u) * 64 + lane, n - 1));
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u)
        if (b + u < b1) {
          const int first = (b + u) * 64, low = keep - first, in = n - first;
          f(first + lane, r[u], low >= 64 ? ~0ull : low <= 0 ? 0ull : (1ull << low) - 1, in >= 64 ? ~0ull : (1ull << in) - 1);
        }
    }
  };
  int same = 0, same_low = 0, less_low = 0, more_high = 0;
  walk([&](int, uint32_t r, uint64_t low, uint64_t in) {
    const uint64_t ties = __ballot(r == edge) & in;
    same += __popcll(ties);
    same_low += __popcll(ties & low);
    less_low += __popcll(__ballot(r < edge) & low);
    more_high += __popcll(__ballot(r > edge) & in & ~low);
  });
  if (lane == 0) { sums[0][wave] = same; sums[1][wave] = same_low; sums[2][wave] = less_low; sums[3][wave] = more_high; }
  __syncthreads();
  // Lane w has wave w's counts: of its ties the first stay, those below keep first.
  const int lw = lane & 15, ties_w = sums[0][lw], low_w = sums[1][lw], ties_before = upto16(ties_w, lane) - ties_w;
  const int stay_w = min(max(equal_kept - ties_before, 0), ties_w), stay_low = min(stay_w, low_w);
  const int places_w = sums[2][lw] + low_w - stay_low, sources_w = sums[3][lw] + stay_w - stay_low;
  const int places_upto = upto16(places_w, lane), sources_upto = upto16(sources_w, lane);
  int n_ties = __builtin_amdgcn_readlane(ties_before, wave);
  int n_place = __builtin_amdgcn_readlane(places_upto - places_w, wave), n_source = __builtin_amdgcn_readlane(sources_upto - sources_w, wave);
  const int base = plan[4 * B + q], bound = min(keep, n - keep);
  int32_t* place = lists + B + base;
  int32_t* source = place + bound;
  const uint64_t below = (1ull << lane) - 1;
  walk([&](int j, uint32_t r, uint64_t low, uint64_t in) {
    const uint64_t ties = __ballot(r == edge) & in;
    const bool stays = r > edge || (r == edge && n_ties + __popcll(ties & below) < equal_kept);
    n_ties += __popcll(ties);
    const uint64_t stay = __ballot(stays) & in, pl = ~stay & low, sr = stay & ~low;
    if (pl >> lane & 1) place[n_place + __popcll(pl & below)] = j;
    if (sr >> lane & 1) source[n_source + __popcll(sr & below)] = j;
    n_place += __popcll(pl);
    n_source += __popcll(sr);
  });
  if (tid == kEvictWaves - 1) lists[q] = places_upto;   // of all waves
}

// ------------------------------------------------------------------------------------------------------------ the moves
// Places lie below keep and sources from keep on: no move reads what another writes.  A workgroup has four moves.  Bound by HBM: 72 us
// for 16 queries of 12800 .. 16000 cut by a quarter (8 key and 8 value heads of 128 bf16 elements an entry, 360 MB read and written).
constexpr int kMovesPerGroup = 4;
template <typename T, int V, typename P>
__global__ __launch_bounds__(256) void cache_evict_move_kernel(CacheRef c, P plan, int B, const int32_t* __restrict__ lists) {
  struct alignas(V * sizeof(T)) C { T x[V]; };
  const int q = (int)blockIdx.y, m0 = (int)blockIdx.x * kMovesPerGroup;
  const int moves = lists[q];
  if (m0 >= moves) return;
  const int64_t slot = plan[q];
  const int n = plan[B + q], keep = plan[2 * B + q];
  const int32_t* place = lists + B + plan[4 * B + q];
  const int32_t* source = place + min(keep, n - keep);
  const int per_head = c.dh / V, per_move = 2 * c.KV * per_head, nm = min(kMovesPerGroup, moves - m0);
  for (int u = (int)threadIdx.x; u < nm * per_move; u += 256) {
    const int m = u / per_move, w = u - m * per_move, h = w / per_head, e = (w - h * per_head) * V;
    T* head = (T*)(h < c.KV ? c.k : c.v) + (slot * c.KV + (h < c.KV ? h : h - c.KV)) * c.capacity * c.dh + e;
    *reinterpret_cast<C*>(head + (int64_t)place[m0 + m] * c.dh) = *reinterpret_cast<const C*>(head + (int64_t)source[m0 + m] * c.dh);
  }
  if ((int)threadIdx.x < nm) {
    const int64_t at = slot * c.capacity, to = at + place[m0 + threadIdx.x], from = at + source[m0 + threadIdx.x];
    c.positions[to] = c.positions[from];
    c.mass[to] = c.mass[from];
  }
}

hipError_t launch_cache_evict(int dtype, const CacheRef& c, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int max_len,
                              int max_moves, int lead, bool has_recent, int32_t* lists, hipStream_t s) {
  if (max_moves <= 0) return hipSuccess;   // nothing is to go, or nothing stays
  return with_plan(plan, count, d_plan, [&](auto p) {
    typedef decltype(p) P;
    if (max_len <= kEvictInLds) {
      const hipError_t e = set_max_dynamic_lds((const void*)cache_evict_select_kernel<true, P>, kEvictInLds * (int)sizeof(uint32_t));
      if (e != hipSuccess) return e;
      cache_evict_select_kernel<true, P><<<dim3(B), dim3(kEvictThreads), (size_t)max_len * sizeof(uint32_t), s>>>(c, p, B, lead, has_recent, lists);
    } else {
      cache_evict_select_kernel<false, P><<<dim3(B), dim3(kEvictThreads), 0, s>>>(c, p, B, lead, has_recent, lists);
    }
    const dim3 grid((max_moves + kMovesPerGroup - 1) / kMovesPerGroup, B), block(256);
    if (dtype == 0) cache_evict_move_kernel<float, 4, P><<<grid, block, 0, s>>>(c, p, B, lists);
    else if (c.dh % 8 == 0) cache_evict_move_kernel<bf16_t, 8, P><<<grid, block, 0, s>>>(c, p, B, lists);
    else cache_evict_move_kernel<bf16_t, 4, P><<<grid, block, 0, s>>>(c, p, B, lists);
    return hipGetLastError();
  });
}

}  // namespace otas
