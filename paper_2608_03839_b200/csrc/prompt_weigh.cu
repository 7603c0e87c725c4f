// The attention weight that a prompt's keys receive, for its own queries:
//
//   w_j = sum over rows i >= j - (c - n) and the key head's query heads of r_i exp(scale q_i.k_j - lse_i)
//
// The product is taken the other way round than in attention, S = K Q^T: a row of TMEM is a key, its columns
// are query rows, so that a thread adds up one key's weight over all rows in registers and nothing is
// joined between lanes.  A block takes items of 256 keys of one key head, in two groups A and B of 128 that
// stay in shared memory, and goes through the query rows that see them in tiles of 128: 128 / pack tokens
// of `pack` query heads.  Warps:
//   0-3, 4-7, 8-11, 12-15   sums of A over the first and the last 64 columns, of B: a key a thread
//   16         loads by tensor maps: the next item's keys (two places), then this one's queries
//   17         issues the products
//   18, 19     bring what a row's exponent begins with, -lse log2 e, and its weight r to shared memory
// What counts is to have four warps an SM quarter: their chains of a load from TMEM, exponent, sum hide each other.
// (With a query row a thread and 128 sums a thread there were registers for two, and a tile took 3,400 cycles,
// where its exponentials take 2,048.)
// Rows that do not count (behind the sequence's last one, weight 0, lse -inf) have -inf there, and the exponents of
// their columns and of those that do not see the key are replaced, so that it does not matter what they hold.  Leading
// and trailing rows with weight 0 are left out of the tiles: all warps look for the first and the
// last other one of each long sequence when the kernel begins.
//
// Sums are fp32: of a tile's 64 columns as four, and over the tiles with the part that each addition
// loses carried along (a key may receive 10^5 terms).
//
// Where there are fewer items than SMs the rows of an item are shared by a cluster of blocks, whose
// totals are added in order.
//
// Measured, with 32 query heads over 8 key heads of 128: 16 prompts of up to 2,048 rows in 153 us (101 GFLOP, 660
// TFLOP/s; their exponentials at the unit's rate take 88), one of 8,192 in 358 us, the last 64 rows of 4 x 16,384 in 52 us (74
// MB; eight items a block of two tiles each, 6 us an item, of which the tiles' own time is less than half).  In
// whole items a tile of 256 keys by 128 rows takes 2,500 cycles, the exponentials 2,048 of them; shared by a cluster (one
// prompt of 4,096) the unit is busy 55 % of the time that a block runs.  A polynomial in place of an eighth of the
// exponentials gave 4 %, more of them less; not kept.
//
// Every wait is bounded, as in attention.
#include <cooperative_groups.h>

#include "prompt.cuh"
#include "tensor.cuh"

namespace cg = cooperative_groups;

namespace oilbird {

namespace {

constexpr int kPwThreads = 640, kPwSumWarps = 16, kPwLoader = 16, kPwIssuer = 17, kPwRows = 18;
// registers a thread: launched with 96; the five warpgroups' shares add up to 5 x 96
constexpr int kPwSumRegs = 104, kPwRestRegs = 64;
static_assert(4 * kPwSumRegs + kPwRestRegs <= 5 * 96, "more registers than the block was launched with");
constexpr int kPwHalf = 64;                              // a thread's columns of a tile
constexpr int kPwAhead = 4;                              // places for the rows' numbers
constexpr int kPwLong = 512;                             // rows of a sequence whose ends are looked at

struct PwItem {
  int s, head, key0;                 // first key of A
  int n, c, q0, k0;
  int from, to, tiles;               // rows that count; tiles of queries for each of the head's packs of query heads
  int skip;                          // leading tiles that nothing of B is seen in
  int begin, end;                    // of packs * tiles: this block's share
  int live;
};
struct PwShared {
  uint64_t full[8], free[8], kfull[2], kfree[2], sfull[2][2], sfree[2][2], item_full[2], item_free[2], meet;
  uint64_t rows_full[kPwAhead], rows_free[kPwAhead];
  PwItem item[2];
  alignas(16) float bias[kPwAhead][kPrTile], weight[kPwAhead][kPrTile];      // of a tile's rows, read four at a time
  int plain[kPwAhead][2];                                // all of a half count, with weight 1
  float sums[2][2][2 * kPrTile];                         // [item's parity][half of the columns][key]
  float shared[2 * kPrTile];                             // of the block, for the cluster
  int from[kPrMaxSeq], to[kPrMaxSeq];                    // rows of a sequence that count
  uint32_t tmem;
  Waits waits;
};

template <int D>
struct Pw {
  static constexpr int kBlocks = D / 64, kMat = kBlocks * kPrTile * 128;
  static constexpr int kStages = D == 128 ? 2 : 6;
  static constexpr int kBytes = 1024 + (4 + kStages) * kMat + (int)sizeof(PwShared) + 16 + (int)sizeof(PromptList);
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

// Items of 256 keys; those with more rows lie in front.
struct PwOrder {
  const PromptList* l;
  int log_span, padded;              // tokens of a tile; keys to write for every sequence (0: packed)
  static __device__ __forceinline__ int ceil(int keys) { return (int)(((unsigned)keys + 2 * kPrTile - 1) / (2 * kPrTile)); }
  __device__ __forceinline__ int most_tiles(int s) const { return (int)(((unsigned)l->n[s] + (1u << log_span) - 1) >> log_span); }
  __device__ __forceinline__ int items(int s, int level, int unit) const {
    if (level == 0) return ceil(padded ? padded : l->c[s]);
    const long long rows = ((long long)(level - 1) * unit) << log_span;  // the first key of the item is seen by more than these
    return l->n[s] <= rows || l->c[s] <= rows ? 0 : ceil((int)(l->c[s] - rows));
  }
  __device__ __forceinline__ int item(int, int, int at, int, int above) const { return above + at; }
};

// The rows [from, to) of each long sequence outside which all weights are 0; every thread calls.
__device__ __forceinline__ void live_rows(const PromptArgs& a, const PromptList& l, PwShared& sh) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto weights = [&](int s) { return a.row_weight + (a.qs.first ? 0ll : (long long)s * a.qs.rows) + prompt_begin(a.qs, s); };
  for (int s = tid; s < a.n_seq; s += kPwThreads) {
    const int n = l.n[s];
    const bool look = a.row_weight && n > kPwLong && (weights(s)[0] == 0.f || weights(s)[n - 1] == 0.f);
    sh.from[s] = look ? n : 0;
    sh.to[s] = look ? -1 : n;                            // -1: still to be looked at
  }
  __syncthreads();
  if (!a.row_weight) return;
  // pieces of 512 rows of all those sequences, a warp each, in turn
  constexpr int kPiece = 512;
  int at = warp;
  for (int s = 0; s < a.n_seq; ++s) {
    if (sh.from[s] == 0 && sh.to[s] == l.n[s]) continue;  // (no piece changes one that is looked at to this: see below)
    const int n = l.n[s], pieces = (n + kPiece - 1) / kPiece;
    const float* w = weights(s);
    for (; at < pieces; at += kPwThreads / 32) {
      int first = 0x7fffffff, last = -1;
      float x[kPiece / 32];
#pragma unroll
      for (int e = 0; e < kPiece / 32; ++e) {
        const int i = at * kPiece + e * 32 + lane;
        x[e] = i < n ? w[i] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < kPiece / 32; ++e) {
        const int i = at * kPiece + e * 32 + lane;
        if (x[e] != 0.f) { first = min(first, i); last = i; }
      }
      first = __reduce_min_sync(0xffffffffu, first);
      last = __reduce_max_sync(0xffffffffu, last);
      if (lane == 0 && last >= 0) {
        atomicMin(&sh.from[s], first);
        atomicMax(&sh.to[s], last + 1);
      }
    }
    at -= pieces;
  }
  __syncthreads();
}

}  // namespace

template <int D, bool kBf16>
__global__ void __launch_bounds__(kPwThreads, 1)
prompt_weigh_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                    const __grid_constant__ PromptArgs a, int shares) {
  using P = Pw<D>;
  extern __shared__ unsigned char raw_smem[];
  unsigned char* smem = raw_smem + ((1024 - (kv_smem(raw_smem) & 1023)) & 1023);
  unsigned char* kmat = smem;                            // two places of A, then B: [block of 64 channels][key]
  unsigned char* ring = smem + 4 * P::kMat;
  PwShared& sh = *reinterpret_cast<PwShared*>(ring + P::kStages * P::kMat);
  PromptList& list = *reinterpret_cast<PromptList*>(ring + P::kStages * P::kMat + (sizeof(PwShared) + 15) / 16 * 16);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int rank = blockIdx.x % shares;                  // in the cluster
  volatile Waits* waits = &sh.waits;

  if (tid == 0) {
    for (int i = 0; i < P::kStages; ++i) {
      bar_init(&sh.full[i], 1);
      bar_init(&sh.free[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(&sh.kfull[i], 1);
      bar_init(&sh.kfree[i], 1);
      for (int b = 0; b < 2; ++b) {
        bar_init(&sh.sfull[i][b], 1);
        bar_init(&sh.sfree[i][b], 8);
      }
      bar_init(&sh.item_full[i], 1);
      bar_init(&sh.item_free[i], kPwSumWarps + 3);
      sh.item[i].live = 0;
    }
    for (int i = 0; i < kPwAhead; ++i) {
      bar_init(&sh.rows_full[i], 2);
      bar_init(&sh.rows_free[i], kPwSumWarps);
    }
    bar_init(&sh.meet, kPwSumWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kPwIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(kv_smem(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_enter();
  if (tid == 0) waits_begin(sh.waits, a.wait_limit);
  prompt_extents(a, list);
  __syncthreads();
  const PwOrder order = {&list, 7 - a.log_pack, a.ks.first ? 0 : a.ks.rows};
  prompt_levels(order, a.n_seq, list);
  live_rows(a, list, sh);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  const int span = kPrTile >> a.log_pack, packs = a.group >> a.log_pack;

  if (warp < kPwSumWarps) {
    // ============================================================ sums ===========
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPwSumRegs));
    const int half = warp >> 2 & 1, wg = warp >> 3, row = tid & 127, col0 = half * kPwHalf;
    const uint32_t s_tm = tmem + ((uint32_t)(warp & 3) << 21) + wg * 256 + col0;
    const float2 f2 = make_float2(a.factor, a.factor);
    uint32_t u = 0, su = 0;
    for (uint32_t iu = 0;; ++iu) {
      if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, waits, a.stats)) break;
      const PwItem& now = sh.item[iu & 1];
      const int live = now.live, begin = now.begin, end = now.end, tiles = now.tiles, skip = wg ? now.skip : 0, from = now.from;
      const int s = now.s, head = now.head, c = now.c, k0 = now.k0, key = now.key0 + wg * kPrTile + row;
      const int first_row = key - (c - now.n);           // the first row that sees the key
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
      if (!live) break;
      float total = 0.f, lost = 0.f;
      bool ok = true;
      int t = tiles > 0 ? begin % tiles : 0;
      for (int i = begin; i < end; ++i, ++u, t = t + 1 == tiles ? 0 : t + 1) {
        const uint32_t rs = u % kPwAhead, b = su & 1;
        // (also where nothing is done with the tile: its place is given back once each time it is full)
        if (!warp_wait(&sh.rows_full[rs], (u / kPwAhead) & 1, waits, a.stats)) { ok = false; break; }
        if (t >= skip) {
          if (!warp_wait(&sh.sfull[wg][b], (su >> 1) & 1, waits, a.stats)) { ok = false; break; }
          fence_after();
          ++su;
          // columns whose rows do not see the key
          const int blind = min(max(first_row - (from + t * span), 0), span) * a.pack - col0;
          const float4* bias = reinterpret_cast<const float4*>(sh.bias[rs] + col0);
          const float4* weight = reinterpret_cast<const float4*>(sh.weight[rs] + col0);
          const bool plain = sh.plain[rs][half] && __all_sync(0xffffffffu, blind <= 0);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          uint32_t x[2][16];
          tmem_ask16(s_tm + b * 128, x[0]);
#pragma unroll
          for (int k = 0; k < kPwHalf / 16; ++k) {
            uint32_t (&y)[16] = x[k & 1];
            tmem_wait16(y);
            if (k + 1 < kPwHalf / 16) tmem_ask16(s_tm + b * 128 + (k + 1) * 16, x[(k + 1) & 1]);
            else {
              fence_before();
              __syncwarp();
              if (lane == 0) bar_arrive(&sh.sfree[wg][b]);
            }
            if (plain) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float4 bb = bias[4 * k + e];
                const float2 z0 = fma2(make_float2(__uint_as_float(y[4 * e]), __uint_as_float(y[4 * e + 1])), f2, make_float2(bb.x, bb.y));
                const float2 z1 = fma2(make_float2(__uint_as_float(y[4 * e + 2]), __uint_as_float(y[4 * e + 3])), f2, make_float2(bb.z, bb.w));
                sum[0] = add2(sum[0], make_float2(exp2_approx(z0.x), exp2_approx(z0.y)));
                sum[1] = add2(sum[1], make_float2(exp2_approx(z1.x), exp2_approx(z1.y)));
              }
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float4 bb = bias[4 * k + e], ww = weight[4 * k + e];
                const float2 z0 = fma2(make_float2(__uint_as_float(y[4 * e]), __uint_as_float(y[4 * e + 1])), f2, make_float2(bb.x, bb.y));
                const float2 z1 = fma2(make_float2(__uint_as_float(y[4 * e + 2]), __uint_as_float(y[4 * e + 3])), f2, make_float2(bb.z, bb.w));
                float z[4] = {z0.x, z0.y, z1.x, z1.y};
                // (the exponent is replaced, not the score: a blind row's logarithm may be NaN)
#pragma unroll
                for (int h = 0; h < 4; ++h)
                  if (16 * k + 4 * e + h < blind || (&bb.x)[h] == -INFINITY) z[h] = -INFINITY;
                sum[0] = fma2(make_float2(exp2_approx(z[0]), exp2_approx(z[1])), make_float2(ww.x, ww.y), sum[0]);
                sum[1] = fma2(make_float2(exp2_approx(z[2]), exp2_approx(z[3])), make_float2(ww.z, ww.w), sum[1]);
              }
            }
          }
          sum[0] = add2(sum[0], sum[1]);
          const float more = __fadd_rn(__fadd_rn(sum[0].x, sum[0].y), lost), next = __fadd_rn(total, more);
          // (what rounding to `next` lost; nothing once that is infinite or NaN)
          lost = fabsf(next) < INFINITY ? __fsub_rn(more, __fsub_rn(next, total)) : 0.f;
          total = next;
        }
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.rows_free[rs]);
      }
      if (!ok) break;
      // both halves of the columns
      float (&sums)[2][2 * kPrTile] = sh.sums[iu & 1];
      sums[half][wg * kPrTile + row] = total + lost;
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.meet);
      if (!warp_wait(&sh.meet, iu & 1, waits, a.stats)) break;
      if (half == 0) {
        const float sum = sums[0][wg * kPrTile + row] + sums[1][wg * kPrTile + row];
        if (shares > 1) sh.shared[wg * kPrTile + row] = sum;
        else if (key < (a.ks.first ? c : a.ks.rows))
          a.weight[((a.ks.first ? 0ll : (long long)s * a.n_kv) + head) * a.ks.rows + k0 + key] = key < c ? sum : 0.f;
      }
      if (shares > 1) break;                             // (a cluster has one item)
    }
    fence_before();
    __syncthreads();
    if (shares > 1) {
      meet_cluster();
      if (rank == 0 && tid < 2 * kPrTile) {              // a key a thread
        const PwItem& it = sh.item[0];
        if (it.live) {
          const int key = it.key0 + tid, keys = a.ks.first ? it.c : a.ks.rows;
          float sum = sh.shared[tid];
          for (int r = 1; r < shares; ++r) sum += cg::this_cluster().map_shared_rank(&sh, r)->shared[tid];
          if (key < keys)
            a.weight[((a.ks.first ? 0ll : (long long)it.s * a.n_kv) + it.head) * a.ks.rows + it.k0 + key] = key < it.c ? sum : 0.f;
        }
      }
      meet_cluster();                                    // (nobody leaves while its shared memory is read)
    }
    return;
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPwRestRegs));
    if (warp == kPwLoader) {
      // ========================================================== loads ==========
      int level = list.levels;
      const bool leader = one_lane();
      const int crew = gridDim.x / shares, me = blockIdx.x / shares;
      uint32_t u = 0, ku = 0;
      bool ok = true;
      PwItem cur, next;
      cur.live = 0;
      cur.begin = cur.end = 0;
      for (uint32_t iu = 0; ok; ++iu) {
        // ---- the next item, and its keys ----
        const long long i = (long long)iu * crew + (iu & 1 ? crew - 1 - me : me);
        int s = 0, t = 0;
        next.live = (shares == 1 || iu == 0) && prompt_find(order, a.n_seq, list, (int)(i / a.n_kv), lane, level, s, t);
        next.s = s;
        next.head = (int)(i % a.n_kv);
        next.key0 = t * 2 * kPrTile;
        next.n = list.n[s];
        next.c = list.c[s];
        next.q0 = prompt_begin(a.qs, s);
        next.k0 = prompt_begin(a.ks, s);
        const int shift = next.c - next.n;
        next.from = max(max(sh.from[s], next.key0 - shift), 0);
        next.to = sh.to[s];
        next.tiles = next.live && next.key0 < next.c && next.to > next.from ? (next.to - next.from + span - 1) / span : 0;
        next.skip = min(max((next.key0 + kPrTile - shift - next.from) / span, 0), next.tiles);
        if (next.key0 + kPrTile >= next.c) next.skip = next.tiles;           // B has no keys
        const long long all = (long long)packs * next.tiles;
        next.begin = (int)(all * rank / shares);
        next.end = (int)(all * (rank + 1) / shares);
        if (iu >= 2 && !warp_wait(&sh.item_free[iu & 1], ((iu >> 1) - 1) & 1, waits, a.stats)) break;
        if (lane == 0) {
          sh.item[iu & 1] = next;
          bar_arrive(&sh.item_full[iu & 1]);
        }
        if (next.begin < next.end) {
          const uint32_t place = ku & 1;
          if (ku >= 2 && !warp_wait(&sh.kfree[place], ((ku >> 1) - 1) & 1, waits, a.stats)) break;
          ++ku;
          if (leader) {
            bar_expect(&sh.kfull[place], 2 * P::kMat);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
              for (int b = 0; b < P::kBlocks; ++b)
                map_load4(kv_smem(kmat + (place * 2 + g) * P::kMat + b * (kPrTile * 128)), &k_map, b * 64, next.head,
                          next.k0 + next.key0 + g * kPrTile, a.ks.first ? 0 : s, &sh.kfull[place]);
          }
          __syncwarp();
        }
        // ---- this one's queries ----
        for (int j = cur.begin; j < cur.end; ++j, ++u) {
          const uint32_t st = u % P::kStages, use = u / P::kStages;
          if (use > 0 && !warp_wait(&sh.free[st], (use - 1) & 1, waits, a.stats)) { ok = false; break; }
          if (leader) {
            bar_expect(&sh.full[st], P::kMat);
#pragma unroll
            for (int b = 0; b < P::kBlocks; ++b)
              map_load4(kv_smem(ring + st * P::kMat + b * (kPrTile * 128)), &q_map, b * 64,
                        cur.head * a.group + j / cur.tiles * a.pack, cur.q0 + cur.from + j % cur.tiles * span,
                        a.qs.first ? 0 : cur.s, &sh.full[st]);
          }
          __syncwarp();
        }
        if (!next.live) break;
        cur = next;
      }
    } else if (warp >= kPwRows) {
      // ========================================================== the rows' numbers ====
      const int half = warp - kPwRows, col = half * kPwHalf + 2 * lane;
      uint32_t u = 0;
      bool ok = true;
      for (uint32_t iu = 0; ok; ++iu) {
        if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, waits, a.stats)) break;
        const PwItem& now = sh.item[iu & 1];
        const int live = now.live, begin = now.begin, end = now.end, tiles = now.tiles, from = now.from, to = now.to;
        const int s = a.qs.first ? 0 : now.s, q0 = now.q0, head0 = now.head * a.group;
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
        if (!live) break;
        const float* lse = a.lse + s * a.lse_seq + q0 * a.lse_row;
        const float* rw = a.row_weight ? a.row_weight + (long long)s * a.qs.rows + q0 : nullptr;
        // two rows a lane, asked for a tile ahead
        float l[2] = {-INFINITY, -INFINITY}, w[2] = {0.f, 0.f};
        auto ask = [&](int i) {
          const int pack = i / tiles, tok0 = from + (i - pack * tiles) * span;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int tok = tok0 + ((col + e) >> a.log_pack), hd = head0 + pack * a.pack + ((col + e) & (a.pack - 1));
            l[e] = -INFINITY;
            w[e] = 0.f;
            if (tok < to) {
              l[e] = __ldg(lse + tok * a.lse_row + hd * a.lse_head);
              w[e] = rw ? __ldg(rw + tok) : 1.f;
            }
          }
        };
        if (begin < end) ask(begin);
        for (int i = begin; i < end; ++i, ++u) {
          const uint32_t rs = u % kPwAhead, use = u / kPwAhead;
          float2 bias, weight;
          bool counts[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            counts[e] = w[e] != 0.f && l[e] != -INFINITY;
            (&bias.x)[e] = counts[e] ? -l[e] * kLog2e : -INFINITY;
            (&weight.x)[e] = counts[e] ? w[e] : 0.f;
            // A weight that is not finite goes into the exponent, which columns that do not see the key leave out (0 times
            // it would be NaN there); of a row that counts for nothing (lse +inf) it is NaN.
            if (counts[e] && !(fabsf(w[e]) < INFINITY)) {
              (&bias.x)[e] = w[e] == w[e] && l[e] < INFINITY ? INFINITY : __int_as_float(0x7fffffff);
              (&weight.x)[e] = w[e] < 0.f ? -1.f : 1.f;
            }
          }
          if (i + 1 < end) ask(i + 1);
          const bool plain = __all_sync(0xffffffffu, counts[0] && counts[1] && weight.x == 1.f && weight.y == 1.f);
          if (use > 0 && !warp_wait(&sh.rows_free[rs], (use - 1) & 1, waits, a.stats)) { ok = false; break; }
          *reinterpret_cast<float2*>(sh.bias[rs] + col) = bias;
          *reinterpret_cast<float2*>(sh.weight[rs] + col) = weight;
          if (lane == 0) sh.plain[rs][half] = plain;
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.rows_full[rs]);
        }
      }
    } else if (warp == kPwIssuer) {
      // ========================================================== products =======
      const uint32_t idesc = idesc_16(kPrTile, false, kBf16) | (a.negate ? kNegateA : 0u);
      const uint64_t k_desc = desc128(kv_smem(kmat), 16), q_desc = desc128(kv_smem(ring), 16);
      constexpr uint64_t kStage = P::kMat >> 4;
      const bool leader = one_lane();
      uint32_t u = 0, ku = 0, su[2] = {0, 0};
      bool ok = true;
      for (uint32_t iu = 0; ok; ++iu) {
        if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, waits, a.stats)) break;
        const PwItem& it = sh.item[iu & 1];
        const int live = it.live, tiles = it.tiles, skip = it.skip, begin = it.begin, end = it.end;
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
        if (!live) break;
        if (begin >= end) continue;
        const uint32_t place = ku & 1;
        if (!warp_wait(&sh.kfull[place], (ku >> 1) & 1, waits, a.stats)) break;
        ++ku;
        const uint64_t kd = k_desc + place * 2 * kStage;
        for (int i = begin; i < end && ok; ++i, ++u) {
          const uint32_t st = u % P::kStages;
          if (!warp_wait(&sh.full[st], (u / P::kStages) & 1, waits, a.stats)) { ok = false; break; }
          const uint64_t qd = q_desc + st * kStage;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (g && i % tiles < skip) continue;
            const uint32_t b = su[g] & 1, use = su[g] >> 1;
            if (use > 0 && !warp_wait(&sh.sfree[g][b], (use - 1) & 1, waits, a.stats)) { ok = false; break; }
            ++su[g];
            fence_after();
            if (leader) {
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint64_t off = (uint64_t)((k >> 2) * (kPrTile * 128 >> 4) + (k & 3) * 2);
                mma_ss(tmem + g * 256 + b * 128, kd + g * kStage + off, qd + off, idesc, k > 0);
              }
              commit(&sh.sfull[g][b]);
            }
            __syncwarp();
          }
          if (!ok) break;
          if (leader) {
            commit(&sh.free[st]);
            if (i + 1 == end) commit(&sh.kfree[place]);
          }
          __syncwarp();
        }
      }
    }
    // (as in attention: nothing follows the roles)
    fence_before();
    __syncthreads();
    if (warp == kPwIssuer) {
      fence_after();
      // (the sums waited for all products, and those for all copies, unless somebody gave up)
      if (waits->gave_up) {
        const unsigned long long t0 = now_ns();
        while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
      }
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (shares > 1) {
      meet_cluster();
      meet_cluster();
    }
    return;
  }
}

template <int D, bool kBf16>
static cudaError_t run_weigh(const PromptArgs& a, int sms, cudaStream_t st) {
  CUtensorMap qm, km;
  const int nq = a.qs.first ? 1 : a.n_seq, nk = a.ks.first ? 1 : a.n_seq;
  const bool rows = a.qs.rows > 0;                       // (without one nothing is loaded)
  if (!prompt_map(&km, a.k, D, a.n_kv, a.ks.rows, nk, 1, kPrTile, kBf16) ||
      !prompt_map(&qm, rows ? a.q : a.k, D, rows ? a.n_kv * a.group : a.n_kv, rows ? a.qs.rows : a.ks.rows, rows ? nq : nk,
                  rows ? a.pack : 1, kPrTile / a.pack, kBf16))
    return cudaErrorInvalidValue;
  constexpr long long kItem = 2 * kPrTile;
  const long long tiles = a.ks.first ? a.ks.rows / kItem + a.n_seq : (long long)a.n_seq * ((a.ks.rows + kItem - 1) / kItem);
  const long long items = tiles * a.n_kv;
  // Fewer items than SMs: the rows of each are shared by a cluster.  So they are where the longest item (of the first
  // keys of a prompt, twice the mean) would outlast the others: up to four blocks an SM one after another, while a block has
  // eight tiles in the mean (one prompt of 4,096: 135 us, by whole items 180).  With weights of the rows nothing is known of that.
  int shares = 1;
  const long long mean = (long long)a.qs.rows * a.group / kPrTile / (a.qs.first ? a.n_seq : 1) / 2;
  while (shares < 8 && (items * shares * 2 <= sms || (!a.row_weight && items <= 2 * sms && items * shares * 2 <= 4 * sms && mean >= 16 * shares)))
    shares *= 2;
  return launch_cluster(prompt_weigh_kernel<D, kBf16>, (unsigned)(shares > 1 || items < sms ? items * shares : sms), kPwThreads, Pw<D>::kBytes, shares,
                        st, qm, km, a, shares);
}
cudaError_t launch_prompt_weigh(const PromptArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st) {
  if (head_dim == 64) return bf16 ? run_weigh<64, true>(a, sms, st) : run_weigh<64, false>(a, sms, st);
  return bf16 ? run_weigh<128, true>(a, sms, st) : run_weigh<128, false>(a, sms, st);
}
cudaError_t preload_prompt_weigh_kernels() {
  cudaError_t e;
  if ((e = preload_kernel(prompt_weigh_kernel<64, true>, true)) != cudaSuccess) return e;
  if ((e = preload_kernel(prompt_weigh_kernel<64, false>, true)) != cudaSuccess) return e;
  if ((e = preload_kernel(prompt_weigh_kernel<128, true>, true)) != cudaSuccess) return e;
  return preload_kernel(prompt_weigh_kernel<128, false>, true);
}

}  // namespace oilbird
