// Eviction from the cache: which entries stay (one workgroup a query), then the moves (many).
#include "common.h"
#include "decode_kernels.h"
#include "plan_args.h"

namespace otas {

// ------------------------------------------------------------------------------------------------- which entries stay
// Scores become unsigned numbers in the same order (NaN lowest, protected entries highest), which stay in LDS up to 32768 entries
// (beyond that they are formed again in every pass).  The keep-th largest of them is found by 11, 11 and 10 bits, highest first: a
// histogram of the bits over the entries that agree with those found so far (integer counts: any order gives the same), and a
// scan from its top.  Bytes would take a fourth pass, and the highest of them is little but the exponent: weights of one
// order of magnitude would all meet in one counter.  Of the entries equal to the keep-th the lowest stay.  Then every wave goes
// through a run of its own of the entries twice, counting and writing the places below keep that fall free and the entries above
// that move there, in rising order.
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

template <bool IN_LDS, typename P>
__global__ __launch_bounds__(kEvictThreads) void cache_evict_select_kernel(CacheRef c, P plan, int B, int lead, bool has_recent,
                                                                           int32_t* __restrict__ lists) {
  extern __shared__ __attribute__((aligned(16))) uint32_t ranks[];   // [n] where they fit
  __shared__ int hist[kEvictBins];
  __shared__ uint32_t found;
  __shared__ int above;
  __shared__ int sums[3][kEvictWaves];
  const int q = (int)blockIdx.x, tid = (int)threadIdx.x, wave = tid >> 6, lane = tid & 63;
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
    for (int w = 0; w < wave; ++w) upto += sums[0][w];
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
  // Every wave's run of whole blocks of 64 entries.
  const int blocks = (n + 63) >> 6, per = (blocks + kEvictWaves - 1) / kEvictWaves;
  const int b0 = wave * per, b1 = min(blocks, b0 + per);
  int eqs = 0;
  for (int b = b0; b < b1; ++b) {
    const int j = b * 64 + lane;
    eqs += __popcll(__ballot(j < n && rank(j) == edge));
  }
  if (lane == 0) sums[0][wave] = eqs;
  __syncthreads();
  int eq_before = 0;
  for (int w = 0; w < wave; ++w) eq_before += sums[0][w];
  const int base = plan[4 * B + q], bound = min(keep, n - keep);
  int32_t* place = lists + B + base;
  int32_t* source = place + bound;
  int n_place = 0, n_source = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int eqr = eq_before;
    for (int b = b0; b < b1; ++b) {
      const int j = b * 64 + lane;
      const uint32_t r = j < n ? rank(j) : 0u;
      const bool same = j < n && r == edge;
      const uint64_t ties = __ballot(same), below = (1ull << lane) - 1;
      const bool stays = j < n && (r > edge || (same && eqr + __popcll(ties & below) < equal_kept));
      eqr += __popcll(ties);
      const uint64_t pl = __ballot(j < keep && !stays), sr = __ballot(j >= keep && stays);
      if (pass == 1) {
        if (pl >> lane & 1) place[n_place + __popcll(pl & below)] = j;
        if (sr >> lane & 1) source[n_source + __popcll(sr & below)] = j;
      }
      n_place += __popcll(pl);
      n_source += __popcll(sr);
    }
    if (pass == 0) {
      if (lane == 0) { sums[1][wave] = n_place; sums[2][wave] = n_source; }
      __syncthreads();
      n_place = n_source = 0;
      for (int w = 0; w < wave; ++w) { n_place += sums[1][w]; n_source += sums[2][w]; }
    }
  }
  if (tid == 0) {
    int moves = 0;
    for (int w = 0; w < kEvictWaves; ++w) moves += sums[1][w];
    lists[q] = moves;
  }
}

// ------------------------------------------------------------------------------------------------------------ the moves
// Places lie below keep and sources from keep on: no move reads what another writes.  A workgroup has four moves.
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
