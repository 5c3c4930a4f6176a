// Eviction from the cache: which entries stay (one workgroup a query), then the moves (many).
#include "common.h"
#include "decode_kernels.h"
#include "plan_args.h"

namespace otas {

// ------------------------------------------------------------------------------------------------- which entries stay
// Scores become unsigned numbers in the same order (NaN lowest, protected entries highest); the keep-th largest of them is found by
// its four bytes, highest first: a histogram of the byte over the entries that agree with the bytes found so far, counted
// per wave in LDS (integer counts: any order gives the same), and a walk from its top.  Of the entries equal to it the lowest stay.
// Then every wave goes through a run of its own of the entries twice, counting and writing the places below keep that fall
// free and the entries above that move there, in rising order.  A few passes over 8 n bytes that sit in the L2: latency.
constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

struct EvictQuery {
  const float* mass;
  const int32_t* positions;
  int n, keep, lead, recent_from;
  bool has_recent;
  __device__ uint32_t rank(int j) const {
    if (j < lead || (has_recent && positions[j] >= recent_from)) return 0xFFFFFFFFu;
    const float m = mass[j] + 0.f;   // -0 and 0 are equal
    if (m != m) return 0u;
    const uint32_t b = __float_as_uint(m);
    return b & 0x80000000u ? ~b : b | 0x80000000u;   // -inf: 0x007FFFFF, inf: 0xFF800000
  }
};

template <typename P>
__global__ __launch_bounds__(kEvictThreads) void cache_evict_select_kernel(CacheRef c, P plan, int B, int lead, bool has_recent,
                                                                           int32_t* __restrict__ lists) {
  __shared__ int hist[kEvictWaves][256];
  __shared__ int total[256];
  __shared__ uint32_t found;
  __shared__ int above;
  __shared__ int sums[3][kEvictWaves];
  const int q = (int)blockIdx.x, tid = (int)threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t slot = plan[q];
  const int n = plan[B + q], keep = plan[2 * B + q];
  if (keep >= n) {   // workgroup-uniform
    if (tid == 0) lists[q] = 0;
    return;
  }
  if (keep == 0) {
    if (tid == 0) lists[q] = 0;
    return;
  }
  const EvictQuery eq{c.mass + slot * c.capacity, c.positions + slot * c.capacity, n, keep, lead, plan[3 * B + q], has_recent};
  if (tid == 0) { found = 0; above = 0; }
  for (int byte = 3; byte >= 0; --byte) {
    for (int i = tid; i < kEvictWaves * 256; i += kEvictThreads) (&hist[0][0])[i] = 0;
    __syncthreads();
    const uint32_t prefix = found, mask = byte == 3 ? 0u : ~0u << (8 * (byte + 1));
    for (int j = tid; j < n; j += kEvictThreads) {
      const uint32_t r = eq.rank(j);
      if ((r & mask) == prefix) atomicAdd(&hist[wave][(r >> (8 * byte)) & 255], 1);
    }
    __syncthreads();
    if (tid < 256) {
      int v = 0;
      for (int w = 0; w < kEvictWaves; ++w) v += hist[w][tid];
      total[tid] = v;
    }
    __syncthreads();
    if (wave == 0) {   // the byte of the keep-th largest: as many as possible above it, fewer than keep
      int v[4], sum = 0;
      for (int i = 0; i < 4; ++i) sum += v[i] = total[255 - 4 * lane - i];   // lane 0 has the highest four
      int upto = sum;
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
      }
      int a = above + upto - sum;
      if (a < keep && above + upto >= keep) {   // one lane: all entries that agree so far are more than are still wanted
        int i = 0;
        while (a + v[i] < keep) a += v[i++];
        above = a;
        found = prefix | ((uint32_t)(255 - 4 * lane - i) << (8 * byte));
      }
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
    eqs += __popcll(__ballot(j < n && eq.rank(j) == edge));
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
      const uint32_t r = j < n ? eq.rank(j) : 0u;
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
  (void)max_len;
  if (max_moves <= 0) return hipSuccess;   // nothing is to go, or nothing stays
  return with_plan(plan, count, d_plan, [&](auto p) {
    typedef decltype(p) P;
    cache_evict_select_kernel<P><<<dim3(B), dim3(kEvictThreads), 0, s>>>(c, p, B, lead, has_recent, lists);
    const dim3 grid((max_moves + kMovesPerGroup - 1) / kMovesPerGroup, B), block(256);
    if (dtype == 0) cache_evict_move_kernel<float, 4, P><<<grid, block, 0, s>>>(c, p, B, lists);
    else if (c.dh % 8 == 0) cache_evict_move_kernel<bf16_t, 8, P><<<grid, block, 0, s>>>(c, p, B, lists);
    else cache_evict_move_kernel<bf16_t, 4, P><<<grid, block, 0, s>>>(c, p, B, lists);
    return hipGetLastError();
  });
}

}  // namespace otas
