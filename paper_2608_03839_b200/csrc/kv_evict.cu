// Eviction from the 4-bit cache by accumulated attention weight.
//
// Each (sequence, key/value head) keeps `budget` of its slots: those whose position is below
// `sink` or among the newest `recent`, then the others by (weight descending, position
// ascending).  Attention does not depend on the order of the slots, so nothing is shifted:
// the i-th slot below the budget that was not kept takes the i-th kept slot at or above it.
// What moves is the smaller side, in steady state one row per appended token.  Slots whose page is
// none hold their places below the budget, for a slot moved there would be lost.
//
// A cluster of one to eight blocks handles one (sequence, head), a run of its slots each.  The
// weight of the last slot kept is found by radix selection on the weights' order-preserving
// integers (11 + 11 + 10 bits; slots that have to stay get an order above all): every block counts
// its slots' digits in its shared memory and adds up all blocks' counts; ties by the same
// selection on the positions.  Weights and positions are read once and stay in shared memory
// where they fit.  Then every slot's fate is one bit, the i-th set bit is found by binary search
// over the words' prefix sums (in whichever block's shared memory it lies), and the moves are
// dealt out to all blocks, eight lanes each.
//
// Measured, with 8 heads of 128: 8 sequences of 4,096 to 32,768 slots cut to 4,096 in 66 us
// (9.5 us at the copy rate; selection 28 us, moves 27 us: rows of 32-byte pieces);
// 16 sequences up to seven slots over a budget of 1,024 in 15 us: a launch, one reading, and a
// chain of barriers.
#include <cooperative_groups.h>

#include "kv.cuh"

namespace cg = cooperative_groups;

namespace oilbird {

constexpr int kEvThreads = 512, kEvWarps = 16, kEvBins = 2048, kEvMaxCluster = 8;
// Slots dropped one by one at most, in a block alone: a round takes about 0.2 us, the selection it
// replaces three to six passes of 1.9 us each (16 sequences seven slots over 1,024: 15 us one by
// one, 23 us by selection).
constexpr int kEvFew = 16;

// Order-preserving integer of a weight; NaN below everything, -0 as +0.
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (!(w == w)) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// The order of a slot that has to stay: above every weight's.
constexpr uint32_t kEvStays = 0xfffffffeu, kEvGone = 0xffffffffu;

struct EvictShared {
  uint32_t hist[kEvBins];
  int4 moves[kEvThreads];            // pages and slots in them: source, destination
  uint32_t warp_sum[kEvWarps];
  uint4 last[2][kEvWarps];           // the slot each warp would drop next
  uint32_t digit, below, count;
  // what the other blocks of the cluster read: slots that tie with the last one kept; holes, movers
  uint32_t ties, holes, movers;
  uint32_t all_holes[kEvMaxCluster], all_movers[kEvMaxCluster];    // every block's
};

// A block alone takes its own memory and its own barrier.
template <typename T> __device__ __forceinline__ T* of_block(cg::cluster_group& cl, int n_blocks, T* p, int r) {
  return n_blocks == 1 ? p : cl.map_shared_rank(p, r);
}
__device__ __forceinline__ void sync_blocks(cg::cluster_group& cl, int n_blocks) {
  if (n_blocks == 1) __syncthreads();
  else cl.sync();
}

// Finds the digit d with  sum of hist[> d] < want <= sum of hist[>= d]  (descending = true), or
// the same counted from the low end, over all blocks' counts; sh.below = the sum strictly in
// front of d, sh.count that of d.  All threads.
__device__ __forceinline__ void find_digit(EvictShared& sh, cg::cluster_group& cl, int n_blocks, uint32_t want, bool descending) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint4 c = make_uint4(0, 0, 0, 0);                      // four bins, in the order of counting
  const int b = descending ? kEvBins - 4 - 4 * tid : 4 * tid;
  uint4 x4[kEvMaxCluster];
#pragma unroll
  for (int r = 0; r < kEvMaxCluster; ++r)
    if (r < n_blocks) x4[r] = *reinterpret_cast<const uint4*>(of_block(cl, n_blocks, sh.hist, r) + b);
#pragma unroll
  for (int r = 0; r < kEvMaxCluster; ++r)
    if (r < n_blocks) { c.x += x4[r].x; c.y += x4[r].y; c.z += x4[r].z; c.w += x4[r].w; }
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

// The least (x, y, z) of the warp's, in lexical order.
__device__ __forceinline__ uint4 warp_least(const uint4& v) {
  const uint32_t x = __reduce_min_sync(0xffffffffu, v.x);
  const uint32_t y = __reduce_min_sync(0xffffffffu, v.x == x ? v.y : 0xffffffffu);
  return make_uint4(x, y, __reduce_min_sync(0xffffffffu, v.x == x && v.y == y ? v.z : 0xffffffffu), 0u);
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

__global__ void __launch_bounds__(kEvThreads, 2)
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
      const bool have = (uint32_t)p < (uint32_t)c.n_pages;
      const size_t at = ((size_t)(have ? p : 0) * c.n_kv + head) * page + (slot & (page - 1));
      const float w = c.weight[at];
      const int32_t x = c.pos[at];
      // No page: nothing can be moved there, so below the budget the slot holds its place, and above
      // it is behind everything.
      if (!have) return slot < budget ? make_uint2(kEvStays, 0x80000000u) : make_uint2(0u, 0x7fffffffu);
      return make_uint2(x < a.sink || x >= newest ? kEvStays : weight_order(w), (uint32_t)x);
    };
    if (a.held) {
#pragma unroll 8
      for (int i = tid; i < n; i += kEvThreads) held[i] = fetch(i);
    }
    auto slot_at = [&](int i) { return a.held ? held[i] : fetch(i); };
    uint32_t prefix = 0, mask = 0, want = budget;        // of the order; how many of it are kept
    uint32_t ppre = 0, pmask = 0;                        // of the positions, among ties
    bool by_pos = false;
    if (tid == 0) sh.ties = 0;
    if (n_blocks == 1 && a.held && len - budget <= kEvFew) {
      // ---- few over the budget: the last in order go one by one ----
      auto last_of = [&]() {
        uint4 v = make_uint4(kEvGone, 0u, 0u, 0u);
        for (int i = tid; i < n; i += kEvThreads) {
          const uint2 x = held[i];
          const uint32_t y = ~(x.y ^ 0x80000000u), z = ~(uint32_t)i;
          if (x.x < v.x || (x.x == v.x && (y < v.y || (y == v.y && z < v.z)))) v = make_uint4(x.x, y, z, 0u);
        }
        return v;
      };
      for (int w = tid; w < words; w += kEvThreads) {
        keep[w] = w * 32 + 32 <= n ? 0xffffffffu : (1u << (n - w * 32)) - 1u;
        rank_h[w] = 0u;
      }
      uint4 mine = last_of();
      for (int gone = 0; gone < len - budget; ++gone) {
        const uint4 v = warp_least(mine);
        if (lane == 0) sh.last[gone & 1][warp] = v;
        __syncthreads();
        const int i = (int)~warp_least(sh.last[gone & 1][lane & (kEvWarps - 1)]).z;
        if (i % kEvThreads == tid) {
          keep[i / 32] &= ~(1u << (i & 31));
          held[i].x = kEvGone;
          mine = last_of();
        }
      }
    } else {
      // ---- radix selection ----
      for (int pass = 0; pass < 6; ++pass) {
        if (pass == 3) {
          // ties with the last one kept: all of them, or the lowest positions
          if (sh.count == want) break;
          by_pos = true;
        }
        const int shift = pass % 3 == 0 ? 21 : pass % 3 == 1 ? 10 : 0;
        const uint32_t dmask = pass % 3 == 2 ? 1023u : 2047u;
        for (int i = tid; i < kEvBins; i += kEvThreads) sh.hist[i] = 0;
        __syncthreads();
        uint32_t n_stay = 0;                             // (many in one bin: not one by one)
        for (int i = tid; i < n; i += kEvThreads) {
          const uint2 x = slot_at(i);
          if (pass == 0 && x.x == kEvStays) ++n_stay;
          else if ((x.x & mask) == prefix) {
            const uint32_t key = by_pos ? x.y ^ 0x80000000u : x.x;
            if (!by_pos || (key & pmask) == ppre) atomicAdd(&sh.hist[key >> shift & dmask], 1u);
          }
        }
        if (pass == 0) {
          n_stay = __reduce_add_sync(0xffffffffu, n_stay);
          if (lane == 0 && n_stay) atomicAdd(&sh.hist[kEvStays >> 21], n_stay);
        }
        sync_blocks(cl, n_blocks);
        find_digit(sh, cl, n_blocks, want, !by_pos);
        want -= sh.below;
        if (by_pos) { ppre |= sh.digit << shift; pmask |= dmask << shift; }
        else { prefix |= sh.digit << shift; mask |= dmask << shift; }
        sync_blocks(cl, n_blocks);                       // the counts may be cleared
      }
      // kept: order > prefix, or order == prefix and (position below ppre, or equal to it and among
      // the first `want`); without by_pos every tie is kept
      // ---- a bit per slot, in slot order ----
      uint32_t n_ties = 0;
      for (int i0 = 0; i0 < words * 32; i0 += kEvThreads) {
        const int i = i0 + tid;
        bool in = false, tie = false;
        if (i < n) {
          const uint2 x = slot_at(i);
          const uint32_t key = x.y ^ 0x80000000u;
          in = x.x > prefix || (x.x == prefix && (!by_pos || key < ppre));
          tie = by_pos && x.x == prefix && key == ppre;
        }
        const uint32_t b = __ballot_sync(0xffffffffu, in), t = __ballot_sync(0xffffffffu, tie);
        if (lane == 0 && i / 32 < words) {
          keep[i / 32] = b;
          rank_h[i / 32] = t;
          n_ties += __popc(t);
        }
      }
      if (lane == 0 && n_ties) atomicAdd(&sh.ties, n_ties);
    }
    sync_blocks(cl, n_blocks);
    uint32_t ties = 0, left = want;                      // ties of all blocks; what is left for this one's
    for (int r = 0; r < n_blocks; ++r) {
      const uint32_t t = *of_block(cl, n_blocks, &sh.ties, r);
      ties += t;
      if (r < me) left -= min(left, t);
    }
    if (warp == 0 && by_pos && ties > want)
      // equal in order and position, which a cache's slots are not: the first in slot order stay
      for (int b0 = 0; b0 < words; b0 += 32) {
        const int w = b0 + lane;
        const uint32_t t = w < words ? rank_h[w] : 0u;
        const uint32_t x = warp_inclusive(__popc(t), lane), before = x - __popc(t);
        if (w < words) rank_h[w] = first_bits(t, before >= left ? 0u : left - before);
        left -= min(left, __shfl_sync(0xffffffffu, x, 31));
      }
    __syncthreads();
    // the ranks: a word a thread, holes in the low and movers in the high half of what the warps
    // add up (512 words of 32 slots at a time: below 2^15 each)
    uint32_t holes = 0, movers = 0;
    for (int b0 = 0; b0 < words; b0 += kEvThreads) {
      const int w = b0 + tid, at = (w0 + w) * 32;
      const uint32_t low = at + 32 <= budget ? 0xffffffffu : at >= budget ? 0u : (1u << (budget - at)) - 1u;
      const uint32_t k = w < words ? keep[w] | rank_h[w] : 0u;
      const uint32_t mine = w < words ? __popc(~k & low) + (__popc(k & ~low) << 16) : 0u;
      const uint32_t x = warp_inclusive(mine, lane);
      if (lane == 31) sh.warp_sum[warp] = x;
      __syncthreads();
      uint32_t before = x - mine, all = 0;
#pragma unroll
      for (int v = 0; v < kEvWarps; ++v) {
        const uint32_t y = sh.warp_sum[v];
        if (v < warp) before += y;
        all += y;
      }
      if (w < words) {
        keep[w] = k;
        rank_h[w] = holes + (before & 0xffffu);
        rank_m[w] = movers + (before >> 16);
      }
      holes += all & 0xffffu;
      movers += all >> 16;
      __syncthreads();
    }
    if (tid == 0) { sh.holes = holes; sh.movers = movers; }
    sync_blocks(cl, n_blocks);
    // ---- the moves ----
    if (tid < n_blocks) {
      sh.all_holes[tid] = *of_block(cl, n_blocks, &sh.holes, tid);
      sh.all_movers[tid] = *of_block(cl, n_blocks, &sh.movers, tid);
    }
    // every block's bits and ranks, where they fit beside one another
    const int all_words = (len + 31) / 32;
    uint32_t* every = reinterpret_cast<uint32_t*>(held + (a.held ? a.max_words * 32 : 0));
    if (a.gather)
      for (int w = tid; w < all_words; w += kEvThreads) {
        const int r = w / per, i = w - r * per;
        every[w] = of_block(cl, n_blocks, keep, r)[i];
        every[a.gather + w] = of_block(cl, n_blocks, rank_h, r)[i];
        every[2 * a.gather + w] = of_block(cl, n_blocks, rank_m, r)[i];
      }
    __syncthreads();
    uint32_t n_moves = 0;
    for (int r = 0; r < n_blocks; ++r) n_moves += sh.all_holes[r];
    const size_t block = 2 * (size_t)kv_part_bytes(groups * kKvGroup, page);
    const int lane8 = tid & 7;
    // the slot with rank i among the holes or the movers
    auto find = [&](uint32_t i, bool hole) {
      int r = 0;
      for (;; ++r) {
        const uint32_t here = hole ? sh.all_holes[r] : sh.all_movers[r];
        if (i < here || r == n_blocks - 1) break;
        i -= here;
      }
      const int base = r * per, nw = min(per, all_words - base);
      const uint32_t* rk = a.gather ? every + (hole ? a.gather : 2 * a.gather) + base : of_block(cl, n_blocks, hole ? rank_h : rank_m, r);
      int lo = 0, hi = nw - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (rk[mid] <= i) lo = mid; else hi = mid - 1;
      }
      const uint32_t k = a.gather ? every[base + lo] : of_block(cl, n_blocks, keep, r)[lo];
      const int at = (base + lo) * 32;
      const uint32_t low = at + 32 <= budget ? 0xffffffffu : at >= budget ? 0u : (1u << (budget - at)) - 1u;
      return at + nth_bit(hole ? ~k & low : k & ~low, (int)(i - rk[lo]));
    };
    for (uint32_t m0 = me; m0 < n_moves; m0 += n_blocks * kEvThreads) {
      const uint32_t i = m0 + (uint32_t)tid * n_blocks;
      if (i < n_moves) {
        const int src = find(i, false), dst = find(i, true);
        const int ps = table[src >> c.page_shift], pd = table[dst >> c.page_shift];
        const bool ok = (uint32_t)ps < (uint32_t)c.n_pages && (uint32_t)pd < (uint32_t)c.n_pages;
        sh.moves[tid] = make_int4(ok ? ps : -1, src & (page - 1), pd, dst & (page - 1));
      }
      __syncthreads();
      const int count = (int)min((n_moves - m0 + n_blocks - 1) / n_blocks, (uint32_t)kEvThreads);
      // lanes 0..7: 16 bytes of codes (two for each 32 of K, V and each group), a word of meta, the
      // weight and the position; three moves' loads on their way together
      const int part = groups * page * 36;
      const int kv = lane8 / (2 * groups), c_off = kv * part + (lane8 / 2 % groups) * page * 32 + (lane8 & 1) * 16;
      const int m_off = lane8 / groups * part + groups * page * 32 + lane8 % groups * 4;
      constexpr int kAtOnce = 3;
      for (int k0 = tid >> 3; k0 < count; k0 += kAtOnce * (kEvThreads / 8)) {
        int4 mv[kAtOnce];
        uint4 code[kAtOnce];
        uint32_t meta[kAtOnce], side[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
          const int k = k0 + q * (kEvThreads / 8);
          mv[q] = k < count ? sh.moves[k] : make_int4(-1, 0, 0, 0);
          if (mv[q].x >= 0) {
            const size_t at = (size_t)mv[q].x * c.n_kv + head;
            const unsigned char* bs = c.pages + at * block;
            if (lane8 < 4 * groups) code[q] = *reinterpret_cast<const uint4*>(bs + c_off + mv[q].y * 32);
            if (lane8 < 2 * groups) meta[q] = *reinterpret_cast<const uint32_t*>(bs + m_off + mv[q].y * groups * 4);
            if (lane8 == 6) side[q] = reinterpret_cast<const uint32_t*>(c.weight)[at * page + mv[q].y];
            if (lane8 == 7) side[q] = reinterpret_cast<const uint32_t*>(c.pos)[at * page + mv[q].y];
          }
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q)
          if (mv[q].x >= 0) {
            const size_t at = (size_t)mv[q].z * c.n_kv + head;
            unsigned char* bd = c.pages + at * block;
            if (lane8 < 4 * groups) *reinterpret_cast<uint4*>(bd + c_off + mv[q].w * 32) = code[q];
            if (lane8 < 2 * groups) *reinterpret_cast<uint32_t*>(bd + m_off + mv[q].w * groups * 4) = meta[q];
            if (lane8 == 6) reinterpret_cast<uint32_t*>(c.weight)[at * page + mv[q].w] = side[q];
            if (lane8 == 7) reinterpret_cast<uint32_t*>(c.pos)[at * page + mv[q].w] = side[q];
          }
      }
      __syncthreads();
    }
    sync_blocks(cl, n_blocks);                                           // (others may still read this block's bits)
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

static constexpr long long run_words(long long slots, int blocks) { return ((slots + 31) / 32 + blocks - 1) / blocks; }
static constexpr size_t evict_smem(long long words, bool held, long long gather) {
  return sizeof(EvictShared) + (size_t)(words + 3) / 4 * 4 * (12 + (held ? 32 * 8 : 0)) + (size_t)gather * 12;
}
static_assert(evict_smem(run_words(OILBIRD_KV_MAX_EVICT_SLOTS, kEvMaxCluster), false, 0) <= 224 * 1024, "does not fit a block's shared memory");

cudaError_t launch_kv_evict(const KvView& c, KvEvictArgs a, int head_dim, int sms, cudaStream_t st) {
  const long long slots = (long long)c.max_pages << c.page_shift, items = (long long)c.n_seq * c.n_kv;
  // Blocks a cluster: as many as let every cluster be on the GPU at once (two blocks an SM), but
  // runs of at least 2048 slots (shorter ones do not pay for the cluster's barriers) and at
  // most what a block's shared memory takes.  8 sequences of up to 32,768 slots with
  // 8 heads took 210 us with a block for each and 112 us with clusters.
  int blocks = 1;
  while (blocks < kEvMaxCluster && ((slots > 2048LL * blocks && 2 * blocks * items <= 2 * sms) ||
                                    evict_smem(run_words(slots, blocks), false, 0) > 100 * 1024))
    blocks *= 2;
  const long long words = run_words(slots, blocks), all = (slots + 31) / 32;
  a.held = evict_smem(words, true, 0) <= 100 * 1024;     // two blocks an SM
  a.gather = blocks > 1 && evict_smem(words, a.held, all) <= 110 * 1024 ? (int)all : 0;
  a.max_words = (int)((words + 3) / 4 * 4);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(c.n_seq * c.n_kv * blocks));
  cfg.blockDim = dim3(kEvThreads);
  cfg.dynamicSmemBytes = evict_smem(words, a.held, a.gather);
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
