// Whole prompts: the views handed to the kernels and the list of work that attention and weights
// walk.
//
// A side (query rows, key rows) is packed - sequence s has rows first[s] .. first[s + 1) of one long
// array - or padded - count[s] of `rows` rows of its own.  Query row i of a sequence with n query
// rows and c key rows sees the keys j <= i + c - n.
#pragma once
#include <cuda.h>

#include "kv.cuh"

namespace oilbird {

constexpr int kPrMaxSeq = OILBIRD_KV_MAX_SEQ;        // their extents sit in shared memory
constexpr int kPrTile = 128;                         // keys (or rows) a tile

struct PromptSide {
  const int32_t* first;      // packed; null: padded
  const int32_t* count;      // padded; null: all rows
  int rows;                  // packed: of the array; padded: of each sequence
};

struct PromptArgs {
  PromptSide qs, ks;
  KvRows q, k, v;            // (packed: sequence stride 0)
  uint16_t* out;
  long long out_seq, out_row, out_head;
  float* lse;                // attend writes it, weigh reads it
  long long lse_seq, lse_row, lse_head;
  const float* row_weight;   // weigh: [n_seq, rows] or [rows]; null: 1
  float* weight;             // weigh: [n_seq, n_kv, key rows] or [n_kv, key rows]
  DeviceStats* stats;
  const unsigned long long* wait_limit;      // in stats
  int n_seq, n_kv, group;
  int pack, log_pack;        // query heads that lie side by side in a tile: a power of two that divides group
  float factor;              // |scale| log2 e
  bool negate;               // the scale is negative
};

// Extents of all sequences, and the numbers of items by level (see prompt_levels), in shared memory.
constexpr int kPrLevels = 256;
struct PromptList {
  int n[kPrMaxSeq], c[kPrMaxSeq];    // rows, keys
  int count[kPrLevels + 2], unit, levels;
};

// Offsets and counts are the caller's: whatever they hold, rows stay inside the arrays.
__device__ __forceinline__ int prompt_begin(const PromptSide& p, int s) {
  return p.first ? min(max(p.first[s], 0), p.rows) : 0;
}
__device__ __forceinline__ int prompt_rows(const PromptSide& p, int s) {
  if (!p.first) return p.count ? min(max(p.count[s], 0), p.rows) : p.rows;
  const int at = prompt_begin(p, s);
  return min(max(p.first[s + 1], at), p.rows) - at;
}
__device__ __forceinline__ void prompt_extents(const PromptArgs& a, PromptList& l) {
  for (int s = threadIdx.x; s < a.n_seq; s += blockDim.x) {
    l.n[s] = prompt_rows(a.qs, s);
    l.c[s] = prompt_rows(a.ks, s);
  }
}

// The list of work is not stored.  Items are numbered by falling level (tiles they have to go through, in
// units that make up to kPrLevels of them), so that the last ones are short.  How many items have a level
// or more is counted once, when the kernel begins, by all threads; a warp then finds number i by going down
// the levels from the last item's and through the sequences, while the item before it is worked on.  (A search
// that counted anew for each item took 6 us an item, which short prompts waited for.)
template <class Order>
__device__ __forceinline__ void prompt_levels(const Order& order, int n_seq, PromptList& l) {
  __shared__ int most;                                   // tiles of the longest item
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  for (int s = threadIdx.x; s < n_seq; s += blockDim.x) atomicMax(&most, order.most_tiles(s));
  __syncthreads();
  const int unit = max(1, (most + kPrLevels - 1) / kPrLevels), levels = (most + unit - 1) / unit;
  if (threadIdx.x == 0) { l.unit = unit; l.levels = levels; }
  const int lane = threadIdx.x & 31;                     // a warp a level, a lane a sequence
  for (int x = threadIdx.x >> 5; x <= levels + 1; x += blockDim.x >> 5) {
    int v = 0;
    for (int s = lane; s < n_seq; s += 32) v += order.items(s, x, unit);
    v = __reduce_add_sync(0xffffffffu, v);
    if (lane == 0) l.count[x] = v;
  }
}
// `level`: any that no item from i on passes (at first l.levels); becomes the item's.  A warp.
template <class Order>
__device__ __forceinline__ bool prompt_find(const Order& order, int n_seq, const PromptList& l, int i, int lane, int& level, int& s_out,
                                            int& t_out) {
  if (l.count[0] <= i) return false;
  while (l.count[level] <= i) --level;                   // the largest level with more than i items
  const int unit = l.unit;
  int left = i - l.count[level + 1];                     // place among the items of this level
  for (int s0 = 0; s0 < n_seq; s0 += 32) {
    const int s = s0 + lane;
    const int above = s < n_seq ? order.items(s, level + 1, unit) : 0, all = s < n_seq ? order.items(s, level, unit) : 0;
    const int here = all - above;
    int sum = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, left < sum);
    if (hit) {
      const int at = __ffs(hit) - 1;
      s_out = s0 + at;
      t_out = order.item(s_out, level, left - __shfl_sync(0xffffffffu, sum - here, at), __shfl_sync(0xffffffffu, all, at),
                         __shfl_sync(0xffffffffu, above, at));
      return true;
    }
    left -= __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}

cudaError_t launch_prompt_attend(const PromptArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st);
cudaError_t launch_prompt_weigh(const PromptArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st);
// The 4-dimensional map (channel, head, row, sequence) of one side; a box is 64 channels of `heads`
// heads of `box_rows` rows.  False: the strides are none that a map takes.
bool prompt_map(CUtensorMap* map, const KvRows& r, int head_dim, int heads, int rows, int n_seq, int box_heads, int box_rows, bool bf16);

}  // namespace oilbird
