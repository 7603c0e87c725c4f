// Eviction from the 4-bit cache by accumulated attention weight.
//
// Each (sequence, key/value head) keeps `budget` of its slots: those whose position is below
// `sink` or among the newest `recent`, then the others by (weight descending, position
// ascending).  Attention does not depend on the order of the slots, so nothing is shifted:
// the i-th slot below the budget that was not kept takes the i-th kept slot at or above it.
// What moves is the smaller side, in steady state one row per appended token.
//
// A cluster of one to eight blocks handles one (sequence, head), a run of its slots each.  The
// weight of the last slot kept is found by radix selection on the weights' order-preserving
// integers (11 + 11 + 10 bits): every block counts its slots' digits in its shared memory and
// adds up all blocks' counts; ties by the same selection on the positions.  Weights and
// positions are read once and stay in shared memory where they fit.  Then every slot's fate is
// one bit, the i-th set bit is found by binary search over the words' prefix sums (in whichever
// block's shared memory it lies), and the moves are dealt out to all blocks, eight lanes each.
#include <cooperative_groups.h>

#include "kv.cuh"

namespace cg = cooperative_groups;

namespace oilbird {

constexpr int kEvThreads = 512, kEvWarps = 16, kEvBins = 2048, kEvMaxCluster = 8;

// Order-preserving integer of a weight; NaN below everything, -0 as +0.
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (!(w == w)) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

struct EvictShared {
  uint32_t hist[kEvBins];
  uint2 moves[kEvThreads];           // source and destination slots
  uint32_t warp_sum[kEvWarps];
  uint32_t digit, below, count;
  // what the other blocks of the cluster read: safe slots; kept for sure, ties; holes, movers
  uint32_t safe, sure, ties, holes, movers;
};

// Finds the digit d with  sum of hist[> d] < want <= sum of hist[>= d]  (descending = true), or
// the same counted from the low end, over all blocks' counts; sh.below = the sum strictly in
// front of d, sh.count that of d.  All threads.
__device__ __forceinline__ void find_digit(EvictShared& sh, cg::cluster_group& cl, int n_blocks, uint32_t want, bool descending) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint4 c = make_uint4(0, 0, 0, 0);                      // four bins, in the order of counting
  const int b = descending ? kEvBins - 4 - 4 * tid : 4 * tid;
  for (int r = 0; r < n_blocks; ++r) {
    const uint4 x = *reinterpret_cast<const uint4*>(cl.map_shared_rank(sh.hist, r) + b);
    c.x += x.x; c.y += x.y; c.z += x.z; c.w += x.w;
  }
  if (descending) { uint32_t t = c.x; c.x = c.w; c.w = t; t = c.y; c.y = c.z; c.z = t; }
  const uint32_t mine = c.x + c.y + c.z + c.w;
  uint32_t x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh.warp_sum[warp] = x;
  __syncthreads();
  uint32_t before = x - mine;
  for (int w = 0; w < warp; ++w) before += sh.warp_sum[w];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t n = (&c.x)[i];
    if (before < want && want <= before + n) { sh.digit = descending ? b + 3 - i : b + i; sh.below = before; sh.count = n; }
    before += n;
  }
  __syncthreads();
}

// Position of the n-th set bit (from 0) of w.
__device__ __forceinline__ int nth_bit(uint32_t w, int n) {
  for (; n; --n) w &= w - 1;
  return __ffs(w) - 1;
}
// The first n set bits of w.
__device__ __forceinline__ uint32_t first_bits(uint32_t w, uint32_t n) {
  if (n >= (uint32_t)__popc(w)) return w;
  uint32_t out = 0;
  for (; n; --n) { out |= w & (0u - w); w &= w - 1; }
  return out;
}
__device__ __forceinline__ uint32_t warp_inclusive(uint32_t x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

__global__ void __launch_bounds__(kEvThreads)
kv_evict_kernel(const KvView c, const KvEvictArgs a, int groups) {
  extern __shared__ __align__(16) unsigned char smem[];
  cg::cluster_group cl = cg::this_cluster();
  const int n_blocks = (int)cl.num_blocks(), me = (int)cl.block_rank();
  EvictShared& sh = *reinterpret_cast<EvictShared*>(smem);
  uint32_t* keep = reinterpret_cast<uint32_t*>(smem + sizeof(EvictShared));   // a bit per slot of the run
  uint32_t* rank_h = keep + a.max_words;                 // holes, movers of the run in front of each word
  uint32_t* rank_m = rank_h + a.max_words;
  uint2* held = reinterpret_cast<uint2*>(rank_m + a.max_words);               // order and position, if a.held
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int it = blockIdx.x / n_blocks, s = it / c.n_kv, head = it % c.n_kv;
  const int page = 1 << c.page_shift;
  pdl_enter();
  const long long room = (long long)c.max_pages << c.page_shift;
  int len = c.seq_len[s];
  len = len < 0 ? 0 : (len > room ? (int)room : len);
  const int budget = a.budget;
  if (len > budget) {
    const int per = ((len + 31) / 32 + n_blocks - 1) / n_blocks;              // words a run
    const int w0 = min(me * per, (len + 31) / 32), words = min(per, (len + 31) / 32 - w0);
    const int first = w0 * 32, n = max(0, min(len - first, words * 32));      // the run's slots
    const int newest = c.n_pos[s] - a.recent;
    const int32_t* table = c.table + (size_t)s * c.max_pages;
    auto fetch = [&](int i) {                            // order and position of the run's slot i
      const int slot = first + i, p = table[slot >> c.page_shift];
      uint2 r = make_uint2(0u, 2147483647u);             // (no page: below everything)
      if ((uint32_t)p < (uint32_t)c.n_pages) {
        const size_t at = ((size_t)p * c.n_kv + head) * page + (slot & (page - 1));
        r = make_uint2(weight_order(c.weight[at]), (uint32_t)c.pos[at]);
      }
      return r;
    };
    if (tid == 0) sh.safe = 0;
    __syncthreads();
    uint32_t n_safe = 0;
    if (a.held) {
#pragma unroll 4
      for (int i = tid; i < n; i += kEvThreads) held[i] = fetch(i);
    }
    auto slot_at = [&](int i) { return a.held ? held[i] : fetch(i); };
    auto safe_at = [&](const uint2& x) { return x.y != 2147483647u && ((int)x.y < a.sink || (int)x.y >= newest); };
    // ---- radix selection ----
    uint32_t prefix = 0, mask = 0, want = 0;             // of the weights' order
    uint32_t ppre = 0, pmask = 0;                        // of the positions, among ties
    bool by_pos = false;
    for (int pass = 0; pass < 6; ++pass) {
      if (pass == 3) {
        // ties with the last kept weight: all of them, or the lowest positions
        if (sh.count == want) break;
        by_pos = true;
      }
      const int shift = pass % 3 == 0 ? 21 : pass % 3 == 1 ? 10 : 0;
      const uint32_t dmask = pass % 3 == 2 ? 1023u : 2047u;
      for (int i = tid; i < kEvBins; i += kEvThreads) sh.hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += kEvThreads) {
        const uint2 x = slot_at(i);
        const bool safe = safe_at(x);
        n_safe += safe;
        if (!safe && (x.x & mask) == prefix) {
          const uint32_t key = by_pos ? x.y ^ 0x80000000u : x.x;
          if (!by_pos || (key & pmask) == ppre) atomicAdd(&sh.hist[key >> shift & dmask], 1u);
        }
      }
      if (pass == 0) {
        n_safe = __reduce_add_sync(0xffffffffu, n_safe);
        if (lane == 0 && n_safe) atomicAdd(&sh.safe, n_safe);
      }
      cl.sync();
      if (pass == 0) {
        // positions are distinct, so at most sink + recent <= budget slots are safe; should a
        // caller's be not, the first ones in slot order stay
        uint32_t all = 0;
        for (int r = 0; r < n_blocks; ++r) all += *cl.map_shared_rank(&sh.safe, r);
        want = all >= (uint32_t)budget ? 0u : (uint32_t)budget - all;
        if (want == 0) break;
      }
      find_digit(sh, cl, n_blocks, want, !by_pos);
      want -= sh.below;
      if (by_pos) { ppre |= sh.digit << shift; pmask |= dmask << shift; }
      else { prefix |= sh.digit << shift; mask |= dmask << shift; }
      cl.sync();                                         // the counts may be cleared
    }
    // kept: safe, or order > prefix, or order == prefix and (position below ppre, or equal to it
    // and among the first `want`); without by_pos every tie is kept
    const bool none = mask == 0;                         // nothing but safe slots
    // ---- a bit per slot, in slot order ----
    if (tid == 0) { sh.sure = sh.ties = sh.holes = sh.movers = 0; }
    __syncthreads();
    uint32_t n_sure = 0, n_ties = 0;
    for (int i0 = 0; i0 < words * 32; i0 += kEvThreads) {
      const int i = i0 + tid;
      bool in = false, tie = false;
      if (i < n) {
        const uint2 x = slot_at(i);
        in = safe_at(x);
        if (!in && !none) {
          const uint32_t key = x.y ^ 0x80000000u;
          in = x.x > prefix || (x.x == prefix && (!by_pos || key < ppre));
          tie = by_pos && x.x == prefix && key == ppre;
        }
      }
      const uint32_t b = __ballot_sync(0xffffffffu, in), t = __ballot_sync(0xffffffffu, tie);
      if (lane == 0 && i / 32 < words) {
        keep[i / 32] = b;
        rank_h[i / 32] = t;
        n_sure += __popc(b);
        n_ties += __popc(t);
      }
    }
    if (lane == 0) { atomicAdd(&sh.sure, n_sure); atomicAdd(&sh.ties, n_ties); }
    cl.sync();
    // exact ties (equal weight and position) and an excess of safe slots: the first in slot order
    if (warp == 0) {
      uint32_t left = by_pos ? want : 0u, kept = 0;
      for (int r = 0; r < me; ++r) {
        const uint32_t t = min(left, *cl.map_shared_rank(&sh.ties, r));
        left -= t;
        kept += t + *cl.map_shared_rank(&sh.sure, r);
      }
      uint32_t holes = 0, movers = 0;
      for (int b0 = 0; b0 < words; b0 += 32) {
        const int w = b0 + lane;
        const uint32_t t = w < words && by_pos ? rank_h[w] : 0u, nt = __popc(t);
        const uint32_t xt = warp_inclusive(nt, lane), before = xt - nt;
        uint32_t k = (w < words ? keep[w] : 0u) | first_bits(t, before >= left ? 0u : left - before);
        left -= min(left, __shfl_sync(0xffffffffu, xt, 31));
        const uint32_t nk = __popc(k), xk = warp_inclusive(nk, lane), have = kept + xk - nk;
        k = first_bits(k, have >= (uint32_t)budget ? 0u : (uint32_t)budget - have);
        kept += __shfl_sync(0xffffffffu, xk, 31);
        // slots of the word below the budget, and below the length
        const int at = (w0 + w) * 32;
        const uint32_t low = at + 32 <= budget ? 0xffffffffu : at >= budget ? 0u : (1u << (budget - at)) - 1u;
        const uint32_t h = w < words ? ~k & low : 0u, m = w < words ? k & ~low : 0u;
        const uint32_t xh = warp_inclusive(__popc(h), lane), xm = warp_inclusive(__popc(m), lane);
        if (w < words) {
          keep[w] = k;
          rank_h[w] = holes + xh - __popc(h);
          rank_m[w] = movers + xm - __popc(m);
        }
        holes += __shfl_sync(0xffffffffu, xh, 31);
        movers += __shfl_sync(0xffffffffu, xm, 31);
      }
      if (lane == 0) { sh.holes = holes; sh.movers = movers; }
    }
    cl.sync();
    // ---- the moves ----
    uint32_t n_moves = 0;
    for (int r = 0; r < n_blocks; ++r) n_moves += *cl.map_shared_rank(&sh.holes, r);
    const size_t block = 2 * (size_t)kv_part_bytes(groups * kKvGroup, page);
    const int lane8 = tid & 7;
    // the slot with rank i among the holes or the movers
    auto find = [&](uint32_t i, bool hole) {
      int r = 0;
      for (;; ++r) {
        const uint32_t here = hole ? *cl.map_shared_rank(&sh.holes, r) : *cl.map_shared_rank(&sh.movers, r);
        if (i < here || r == n_blocks - 1) break;
        i -= here;
      }
      const uint32_t* rk = cl.map_shared_rank(hole ? rank_h : rank_m, r);
      const int base = r * per, nw = min(per, (len + 31) / 32 - base);
      int lo = 0, hi = nw - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (rk[mid] <= i) lo = mid; else hi = mid - 1;
      }
      const uint32_t k = cl.map_shared_rank(keep, r)[lo];
      const int at = (base + lo) * 32;
      const uint32_t low = at + 32 <= budget ? 0xffffffffu : at >= budget ? 0u : (1u << (budget - at)) - 1u;
      return at + nth_bit(hole ? ~k & low : k & ~low, (int)(i - rk[lo]));
    };
    for (uint32_t m0 = me; m0 < n_moves; m0 += n_blocks * kEvThreads) {
      const uint32_t i = m0 + (uint32_t)tid * n_blocks;
      if (i < n_moves) sh.moves[tid] = make_uint2(find(i, false), find(i, true));
      __syncthreads();
      const int count = (int)min((n_moves - m0 + n_blocks - 1) / n_blocks, (uint32_t)kEvThreads);
#pragma unroll 2
      for (int k = tid >> 3; k < count; k += kEvThreads / 8) {
        const int src = (int)sh.moves[k].x, dst = (int)sh.moves[k].y;
        const int ps = table[src >> c.page_shift], pd = table[dst >> c.page_shift];
        if ((uint32_t)ps >= (uint32_t)c.n_pages || (uint32_t)pd >= (uint32_t)c.n_pages) continue;
        const int is = src & (page - 1), id = dst & (page - 1);
        const unsigned char* bs = c.pages + ((size_t)ps * c.n_kv + head) * block;
        unsigned char* bd = c.pages + ((size_t)pd * c.n_kv + head) * block;
        // codes: 2 halves of 32 bytes for each of K, V and each group
        if (lane8 < 4 * groups) {
          const int kv = lane8 / (2 * groups), grp = lane8 / 2 % groups, half = (lane8 & 1) * 16;
          const size_t off = kv * (block / 2) + (size_t)grp * page * 32 + half;
          *reinterpret_cast<uint4*>(bd + off + id * 32) = *reinterpret_cast<const uint4*>(bs + off + is * 32);
        }
        if (lane8 < 2 * groups) {
          const int kv = lane8 / groups, grp = lane8 % groups;
          const size_t off = kv * (block / 2) + (size_t)groups * page * 32 + grp * 4;
          *reinterpret_cast<uint32_t*>(bd + off + id * groups * 4) = *reinterpret_cast<const uint32_t*>(bs + off + is * groups * 4);
        }
        const size_t as = ((size_t)ps * c.n_kv + head) * page + is, ad = ((size_t)pd * c.n_kv + head) * page + id;
        if (lane8 == 6) c.weight[ad] = c.weight[as];
        if (lane8 == 7) c.pos[ad] = c.pos[as];
      }
      __syncthreads();
    }
    cl.sync();                                           // (others may still read this block's bits)
  }
  // ---- the lengths, once nobody reads them any more ----
  __syncthreads();
  if (tid == 0) {
    KvWork* work = reinterpret_cast<KvWork*>(c.work);
    __threadfence();
    sh.count = atomicAdd(&work->arrivals, 1u) == gridDim.x - 1;
    if (sh.count) work->arrivals = 0u;
  }
  __syncthreads();
  if (sh.count)
    for (int i = tid; i < c.n_seq; i += kEvThreads)
      if (c.seq_len[i] > budget) c.seq_len[i] = budget;
}

// Blocks a cluster: runs of 2048 to 4096 slots are scanned in a few microseconds, and shorter
// ones do not pay for the cluster's barriers.
static int evict_cluster(long long slots) { return slots <= 4096 ? 1 : slots <= 8192 ? 2 : slots <= 16384 ? 4 : kEvMaxCluster; }
static constexpr long long run_words(long long slots, int blocks) { return ((slots + 31) / 32 + blocks - 1) / blocks; }
static constexpr size_t evict_smem(long long words, bool held) {
  return sizeof(EvictShared) + (size_t)(words + 3) / 4 * 4 * (12 + (held ? 32 * 8 : 0));
}
static_assert(evict_smem(run_words(OILBIRD_KV_MAX_EVICT_SLOTS, kEvMaxCluster), false) <= 224 * 1024, "does not fit a block's shared memory");

cudaError_t launch_kv_evict(const KvView& c, KvEvictArgs a, int head_dim, cudaStream_t st) {
  const long long slots = (long long)c.max_pages << c.page_shift;
  const int blocks = evict_cluster(slots);
  const long long words = run_words(slots, blocks);
  a.held = evict_smem(words, true) <= 100 * 1024;        // two blocks an SM
  a.max_words = (int)((words + 3) / 4 * 4);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(c.n_seq * c.n_kv * blocks));
  cfg.blockDim = dim3(kEvThreads);
  cfg.dynamicSmemBytes = evict_smem(words, a.held);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = !tl_pdl_off && pdl_process_ok() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kv_evict_kernel, c, a, head_dim / kKvGroup);
}
cudaError_t preload_kv_evict_kernels() { return preload_kernel(kv_evict_kernel, true); }

}  // namespace oilbird
