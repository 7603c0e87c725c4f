// Eviction from the 4-bit cache by accumulated attention weight.
//
// Each (sequence, key/value head) keeps `budget` of its slots: those whose position is below
// `sink` or among the newest `recent`, then the others by (weight descending, position
// ascending).  Attention does not depend on the order of the slots, so nothing is shifted:
// the i-th slot below the budget that was not kept takes the i-th kept slot at or above it.
// What moves is the smaller side, in steady state one row per appended token.
//
// One block handles one (sequence, head).  The weight of the last slot kept is found by radix
// selection on the weights' order-preserving integers (11 + 11 + 10 bits, a histogram in
// shared memory each), ties by the same selection on the positions; then every slot's fate is
// one bit in shared memory, and the i-th set bit is found by binary search over the words'
// prefix sums.
#include "kv.cuh"

namespace oilbird {

constexpr int kEvThreads = 1024, kEvWarps = 32, kEvBins = 2048;

// Order-preserving integer of a weight; NaN below everything, -0 as +0.
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (!(w == w)) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

struct EvictShared {
  uint32_t hist[kEvBins];
  uint32_t warp_sum[kEvWarps];
  uint32_t digit, below;
  unsigned counts[2];
};

// Finds the digit d with  sum of hist[> d] < want <= sum of hist[>= d]  (descending = true), or
// the same counted from the low end; sh.below = the sum strictly in front of d.  All threads.
__device__ __forceinline__ void find_digit(EvictShared& sh, uint32_t want, bool descending) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int i0 = 2 * tid, b0 = descending ? kEvBins - 1 - i0 : i0, b1 = descending ? b0 - 1 : b0 + 1;
  const uint32_t c0 = sh.hist[b0], c1 = sh.hist[b1];
  uint32_t x = c0 + c1;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh.warp_sum[warp] = x;
  __syncthreads();
  uint32_t base = 0;
  for (int w = 0; w < warp; ++w) base += sh.warp_sum[w];
  const uint32_t before = base + x - c0 - c1;
  if (before < want && want <= before + c0) { sh.digit = b0; sh.below = before; }
  if (before + c0 < want && want <= before + c0 + c1) { sh.digit = b1; sh.below = before + c0; }
  __syncthreads();
}

// Position of the n-th set bit (from 0) of w.
__device__ __forceinline__ int nth_bit(uint32_t w, int n) {
  for (; n; --n) w &= w - 1;
  return __ffs(w) - 1;
}

__global__ void __launch_bounds__(kEvThreads, 1)
kv_evict_kernel(const KvView c, const KvEvictArgs a, int groups) {
  extern __shared__ __align__(16) unsigned char smem[];
  EvictShared& sh = *reinterpret_cast<EvictShared*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int s = blockIdx.x / c.n_kv, head = blockIdx.x % c.n_kv;
  const int page = 1 << c.page_shift;
  pdl_enter();
  const long long room = (long long)c.max_pages << c.page_shift;
  int len = c.seq_len[s];
  len = len < 0 ? 0 : (len > room ? (int)room : len);
  const int budget = a.budget;
  if (len > budget) {
    const int words = (len + 31) / 32;
    uint32_t* keep = reinterpret_cast<uint32_t*>(smem + sizeof(EvictShared));   // a bit per slot
    uint32_t* rank = keep + a.max_words;                 // movers in front of each word
    const int newest = c.n_pos[s] - a.recent;
    // a slot's order (0 below every real one) and position; safe slots come before all others
    auto slot_at = [&](int slot, uint32_t& order, int& pos, bool& safe) {
      const int p = c.table[(size_t)s * c.max_pages + (slot >> c.page_shift)];
      order = 0;
      pos = 2147483647;
      safe = false;
      if (p >= 0 && p < c.n_pages) {
        const size_t at = ((size_t)p * c.n_kv + head) * page + (slot & (page - 1));
        order = weight_order(c.weight[at]);
        pos = c.pos[at];
        safe = pos < a.sink || pos >= newest;
      }
    };
    if (tid == 0) { sh.counts[0] = 0; sh.counts[1] = 0; }
    __syncthreads();
    // ---- radix selection ----
    uint32_t prefix = 0, mask = 0, want = 0;             // of the weights' order
    uint32_t ppre = 0, pmask = 0;                        // of the positions, among ties
    bool by_pos = false;
    for (int pass = 0; pass < 6; ++pass) {
      if (pass == 3) {
        // ties with the last kept weight: all of them, or the lowest positions
        if (sh.hist[sh.digit] == want) break;
        by_pos = true;
      }
      const int shift = pass % 3 == 0 ? 21 : pass % 3 == 1 ? 10 : 0;
      const uint32_t dmask = pass % 3 == 2 ? 1023u : 2047u;
      __syncthreads();
      for (int i = tid; i < kEvBins; i += kEvThreads) sh.hist[i] = 0;
      __syncthreads();
      unsigned n_safe = 0;
      for (int slot = tid; slot < len; slot += kEvThreads) {
        uint32_t order;
        int pos;
        bool safe;
        slot_at(slot, order, pos, safe);
        n_safe += safe;
        if (!safe && (order & mask) == prefix) {
          const uint32_t key = by_pos ? (uint32_t)pos ^ 0x80000000u : order;
          if (!by_pos || (key & pmask) == ppre) atomicAdd(&sh.hist[key >> shift & dmask], 1u);
        }
      }
      if (pass == 0) {
        n_safe = __reduce_add_sync(0xffffffffu, n_safe);
        if (lane == 0 && n_safe) atomicAdd(&sh.counts[0], n_safe);
      }
      __syncthreads();
      if (pass == 0) {
        // positions are distinct, so at most sink + recent <= budget slots are safe; should a
        // caller's be not, the first ones in slot order stay
        const unsigned safe_all = sh.counts[0];
        want = safe_all >= (unsigned)budget ? 0u : (unsigned)budget - safe_all;
        if (want == 0) break;
      }
      find_digit(sh, want, !by_pos);
      want -= sh.below;
      if (by_pos) { ppre |= sh.digit << shift; pmask |= dmask << shift; }
      else { prefix |= sh.digit << shift; mask |= dmask << shift; }
    }
    __syncthreads();
    // kept: safe, or order > prefix, or order == prefix and (position below ppre, or equal to it
    // and among the first `want`); without by_pos every tie is kept
    const bool none = mask == 0;                         // nothing but safe slots
    // ---- a bit per slot, in slot order ----
    if (tid == 0) { sh.counts[0] = 0; sh.counts[1] = 0; }
    __syncthreads();
    for (int s0 = 0; s0 < words * 32; s0 += kEvThreads) {
      const int slot = s0 + tid;
      bool safe = false, in = false, tie = false;
      if (slot < len) {
        uint32_t order;
        int pos;
        slot_at(slot, order, pos, safe);
        if (!safe && !none) {
          const uint32_t key = (uint32_t)pos ^ 0x80000000u;
          in = order > prefix || (order == prefix && (!by_pos || key < ppre));
          tie = by_pos && order == prefix && key == ppre;
        }
      }
      const uint32_t b = __ballot_sync(0xffffffffu, safe || in);
      const uint32_t t = __ballot_sync(0xffffffffu, tie);
      if (lane == 0 && slot / 32 < words) { keep[slot / 32] = b; rank[slot / 32] = t; }
    }
    __syncthreads();
    // exact ties (equal weight and position) and an excess of safe slots: the first in slot order
    if (warp == 0) {
      uint32_t left = by_pos ? want : 0u, kept = 0;
      for (int w0 = 0; w0 < words; w0 += 32) {
        const int w = w0 + lane;
        const uint32_t t = w < words && by_pos ? rank[w] : 0u;
        uint32_t n = __popc(t), x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        const uint32_t before = x - n;
        uint32_t take = before >= left ? 0u : min(n, left - before), bits = 0, r = t;
        for (; take; --take) { bits |= r & (0u - r); r &= r - 1; }
        uint32_t k = (w < words ? keep[w] : 0u) | bits;
        left -= min(left, __shfl_sync(0xffffffffu, x, 31));
        uint32_t m = __popc(k), y2 = m;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, y2, o);
          if (lane >= o) y2 += y;
        }
        const uint32_t have = kept + y2 - m;
        uint32_t room_left = have >= (uint32_t)budget ? 0u : min(m, (uint32_t)budget - have);
        uint32_t out = 0, rr = k;
        if (room_left == m) out = k;
        else for (; room_left; --room_left) { out |= rr & (0u - rr); rr &= rr - 1; }
        if (w < words) keep[w] = out;
        kept += __shfl_sync(0xffffffffu, y2, 31);
      }
      // movers (kept slots at or above the budget) in front of each word
      __syncwarp();
      uint32_t sum = 0;
      for (int w0 = budget / 32; w0 < words; w0 += 32) {
        const int w = w0 + lane;
        uint32_t k = w < words ? keep[w] : 0u;
        if (w == budget / 32) k &= ~((1u << (budget & 31)) - 1u);
        const uint32_t n = __popc(k);
        uint32_t x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        if (w < words) rank[w] = sum + x - n;
        sum += __shfl_sync(0xffffffffu, x, 31);
      }
      // holes in front of each word below the budget (the word that holds the budget has both:
      // its hole count lies in the word behind the table)
      uint32_t holes = 0;
      for (int w0 = 0; w0 * 32 < budget; w0 += 32) {
        const int w = w0 + lane;
        uint32_t h = 0;
        if (w * 32 < budget) {
          h = ~keep[w];
          if (w == budget / 32) h &= (1u << (budget & 31)) - 1u;
        }
        const uint32_t n = __popc(h);
        uint32_t x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        if (w * 32 < budget) {
          if (w == budget / 32) rank[a.max_words] = holes + x - n;
          else rank[w] = holes + x - n;
        }
        holes += __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) sh.counts[1] = holes;
    }
    __syncthreads();
    // ---- the moves: eight lanes each ----
    const int n_moves = (int)sh.counts[1];
    const int hole_words = (budget + 31) / 32, first = budget / 32;
    const size_t block = 2 * (size_t)kv_part_bytes(groups * kKvGroup, page);
    const int lane8 = tid & 7;
    for (int i = tid >> 3; i < n_moves; i += kEvThreads / 8) {
      int lo = 0, hi = hole_words - 1;                   // the word with the i-th hole
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        const uint32_t r = mid == first ? rank[a.max_words] : rank[mid];
        if (r <= (uint32_t)i) lo = mid; else hi = mid - 1;
      }
      uint32_t h = ~keep[lo];
      if (lo == first) h &= (1u << (budget & 31)) - 1u;
      const int dst = lo * 32 + nth_bit(h, i - (int)(lo == first ? rank[a.max_words] : rank[lo]));
      lo = first;
      hi = words - 1;                                    // the word with the i-th mover
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (rank[mid] <= (uint32_t)i) lo = mid; else hi = mid - 1;
      }
      uint32_t k = keep[lo];
      if (lo == first) k &= ~((1u << (budget & 31)) - 1u);
      const int src = lo * 32 + nth_bit(k, i - (int)rank[lo]);
      const int ps = c.table[(size_t)s * c.max_pages + (src >> c.page_shift)];
      const int pd = c.table[(size_t)s * c.max_pages + (dst >> c.page_shift)];
      if (ps < 0 || ps >= c.n_pages || pd < 0 || pd >= c.n_pages) continue;
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
  }
  // ---- the lengths, once nobody reads them any more ----
  __shared__ int last;
  __syncthreads();
  if (tid == 0) {
    KvWork* work = reinterpret_cast<KvWork*>(c.work);
    __threadfence();
    last = atomicAdd(&work->arrivals, 1u) == gridDim.x - 1;
    if (last) work->arrivals = 0u;
  }
  __syncthreads();
  if (last)
    for (int i = tid; i < c.n_seq; i += kEvThreads)
      if (c.seq_len[i] > budget) c.seq_len[i] = budget;
}

// Shared memory for `slots` slots per sequence.
static constexpr size_t evict_smem(long long slots) {
  return sizeof(EvictShared) + (size_t)(2 * ((slots + 31) / 32) + 1) * 4 + 16;
}
static_assert(evict_smem(OILBIRD_KV_MAX_EVICT_SLOTS) <= 224 * 1024, "does not fit a block's shared memory");

cudaError_t launch_kv_evict(const KvView& c, KvEvictArgs a, int head_dim, cudaStream_t st) {
  const long long slots = (long long)c.max_pages << c.page_shift;
  a.max_words = (int)((slots + 31) / 32);
  return launch_pdl(kv_evict_kernel, dim3(c.n_seq * c.n_kv), dim3(kEvThreads), evict_smem(slots), st, c, a,
                    head_dim / kKvGroup);
}
cudaError_t preload_kv_evict_kernels() { return preload_kernel(kv_evict_kernel, true); }

}  // namespace oilbird
