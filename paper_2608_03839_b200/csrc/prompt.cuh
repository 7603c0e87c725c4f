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
  int n_seq, n_kv, group;
  int pack;                  // query heads that lie side by side in a tile: a power of two that divides group
  float factor;              // |scale| log2 e
  bool negate;               // the scale is negative
};

// Extents of all sequences in shared memory.
struct PromptList {
  int n[kPrMaxSeq], c[kPrMaxSeq], q0[kPrMaxSeq], k0[kPrMaxSeq];   // rows, keys, where they begin
};

// Offsets and counts are the caller's: whatever they hold, rows stay inside the arrays.
__device__ __forceinline__ void prompt_extent(const PromptSide& p, int s, int& at, int& n) {
  if (p.first) {
    at = min(max(p.first[s], 0), p.rows);
    n = min(max(p.first[s + 1], at), p.rows) - at;
  } else {
    at = 0;
    n = p.count ? min(max(p.count[s], 0), p.rows) : p.rows;
  }
}
__device__ __forceinline__ void prompt_extents(const PromptArgs& a, PromptList& l) {
  for (int s = threadIdx.x; s < a.n_seq; s += blockDim.x) {
    prompt_extent(a.qs, s, l.q0[s], l.n[s]);
    prompt_extent(a.ks, s, l.k0[s], l.c[s]);
  }
}

__device__ __forceinline__ long long warp_sum_i64(long long v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The list of work is not stored.  Items are numbered by falling level (tiles they have to go
// through), so that the last ones are short; a warp finds number i by a search over the levels, then over
// the sequences, while the item before it is worked on.  `level`: any that no item from i on passes; becomes the item's.
template <class Order>
__device__ __forceinline__ bool prompt_find(const Order& order, int n_seq, long long i, int lane, int& level, int& s_out, int& t_out) {
  auto count = [&](int x) {
    long long v = 0;
    for (int s = lane; s < n_seq; s += 32) v += order.items(s, x);
    return warp_sum_i64(v);
  };
  if (count(0) <= i) return false;
  int lo = 0, hi = level;
  while (lo < hi) {                                      // the largest level with more than i items
    const int mid = lo + (hi - lo + 1) / 2;
    if (count(mid) > i) lo = mid; else hi = mid - 1;
  }
  level = lo;
  long long left = i - count(lo + 1);                    // place among the items of this level
  for (int s0 = 0; s0 < n_seq; s0 += 32) {
    const int s = s0 + lane;
    const int above = s < n_seq ? order.items(s, lo + 1) : 0, all = s < n_seq ? order.items(s, lo) : 0;
    const long long here = all - above;
    long long sum = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, left < sum);
    if (hit) {
      const int at = __ffs(hit) - 1;
      s_out = s0 + at;
      t_out = order.item(s_out, lo, (int)(left - __shfl_sync(0xffffffffu, sum - here, at)), __shfl_sync(0xffffffffu, all, at),
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
