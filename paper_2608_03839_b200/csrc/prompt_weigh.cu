// The attention weight that a prompt's keys receive, for its own queries:
//
//   w_j = sum over rows i >= j - (c - n) and the key head's query heads of r_i exp(scale q_i.k_j - lse_i)
//
// A block takes items of 256 keys of one key head, in two groups A and B of 128 that stay in shared
// memory, and goes through the query rows that see them in tiles of 128: 128 / pack tokens of `pack` query
// heads.  S = Q K^T as in attention, a row of TMEM a query row: its lse and its weight are two numbers of the
// thread's, and the thread adds its row's share to 128 sums in registers, one a key, over all tiles.
// Only every sixteenth tile, and at the item's end, are the sums added up over the lanes, to totals that
// carry along what each addition loses (a key may receive 10^5 terms).  (With a key a thread, S = K Q^T,
// nothing would have to be added up, but every exponent needs its row's two numbers from shared memory,
// and somebody to bring them there: 3,200 cycles a tile, where the exponentials take 1,024.)  Warps:
//   0-3, 4-7   sums of A and of B
//   8          loads by tensor maps: the next item's keys (two places), then this one's queries
//   9          issues the products
// Rows that do not count (behind the sequence's last one, weight 0, lse -inf) are not added, whatever
// they hold.  Leading and trailing rows with weight 0 are left out of the tiles: all warps look for the first
// and the last other one of each long sequence when the kernel begins.
//
// Where there are fewer items than SMs the rows of an item are shared by a cluster of blocks, whose
// totals are added in order.
//
// Every wait is bounded, as in attention.
#include <cooperative_groups.h>

#include "prompt.cuh"
#include "tensor.cuh"

namespace cg = cooperative_groups;

namespace oilbird {

namespace {

constexpr int kPwThreads = 384, kPwLoader = 8, kPwIssuer = 9;
constexpr int kPwSumRegs = 224, kPwRestRegs = 56;
static_assert(2 * kPwSumRegs + kPwRestRegs <= 3 * 168, "more registers than the block was launched with");
constexpr int kPwTogether = 16;                          // tiles that are added up in one go
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
  uint64_t full[8], free[8], kfull[2], kfree[2], sfull[2][2], sfree[2][2], item_full[2], item_free[2], meet[2];
  PwItem item[2];
  float sums[2][2][4][kPrTile];                          // [item's parity][group][warp]: totals
  float shared[2][kPrTile];                              // of the block, for the cluster
  int from[kPrMaxSeq], to[kPrMaxSeq];                    // rows of a sequence that count
  uint32_t tmem;
  int gave_up;
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
  int span, padded;                  // padded: keys to write for every sequence (0: packed)
  __device__ __forceinline__ int items(int s, int level) const {
    if (level == 0) return ((padded ? padded : l->c[s]) + 2 * kPrTile - 1) / (2 * kPrTile);
    const long long rows = (long long)(level - 1) * span;                // the first key of the item is seen by more than these
    if (l->n[s] <= rows) return 0;
    const long long keys = l->c[s] - rows;
    return keys > 0 ? (int)((keys + 2 * kPrTile - 1) / (2 * kPrTile)) : 0;
  }
  __device__ __forceinline__ int item(int, int, int at, int, int above) const { return above + at; }
};

// The rows [from, to) of each long sequence outside which all weights are 0; every thread calls.
__device__ __forceinline__ void live_rows(const PromptArgs& a, const PromptList& l, PwShared& sh) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto weights = [&](int s) { return a.row_weight + (a.qs.first ? 0ll : (long long)s * a.qs.rows) + l.q0[s]; };
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
  volatile int* gave_up = &sh.gave_up;

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
        bar_init(&sh.sfree[i][b], 4);
      }
      bar_init(&sh.item_full[i], 1);
      bar_init(&sh.item_free[i], 9);
      bar_init(&sh.meet[i], 4);
      sh.item[i].live = 0;
    }
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kPwIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(kv_smem(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_enter();
  prompt_extents(a, list);
  __syncthreads();
  live_rows(a, list, sh);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  const int span = kPrTile / a.pack, packs = a.group / a.pack;

  if (warp < 8) {
    // ============================================================ sums ===========
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPwSumRegs));
    const int wg = warp >> 2, row = tid & 127;
    const uint32_t s_tm = tmem + ((uint32_t)(warp & 3) << 21) + wg * 256;
    const int row_tok = row / a.pack, row_head = row % a.pack;
    uint32_t su = 0;
    bool ok = true;
    for (uint32_t iu = 0;; ++iu) {
      if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, gave_up, a.stats)) break;
      const PwItem it = sh.item[iu & 1];
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
      if (!it.live) break;
      const int shift = it.c - it.n, key0 = it.key0 + wg * kPrTile;
      const long long seq = a.qs.first ? 0 : it.s;
      const float* lse = a.lse + seq * a.lse_seq + it.q0 * a.lse_row;
      const float* rw = a.row_weight ? a.row_weight + seq * a.qs.rows + it.q0 : nullptr;
      float total[4] = {0.f, 0.f, 0.f, 0.f}, lost[4] = {0.f, 0.f, 0.f, 0.f};
      float2 acc[64];
#pragma unroll
      for (int e = 0; e < 64; ++e) acc[e] = make_float2(0.f, 0.f);
      // the lanes' sums of 128 keys: each step leaves half of the keys to either half of the lanes
      auto add_up = [&]() {
        float v[64];
        const bool h16 = lane & 16;
#pragma unroll
        for (int e = 0; e < 64; ++e) {
          const float lo = e & 1 ? acc[e >> 1].y : acc[e >> 1].x, hi = e & 1 ? acc[32 + (e >> 1)].y : acc[32 + (e >> 1)].x;
          v[e] = (h16 ? hi : lo) + __shfl_xor_sync(0xffffffffu, h16 ? lo : hi, 16);
        }
#pragma unroll
        for (int o = 8, m = 32; o; o >>= 1, m >>= 1) {
          const bool h = lane & o;
#pragma unroll
          for (int e = 0; e < m; ++e) v[e] = (h ? v[e + m] : v[e]) + __shfl_xor_sync(0xffffffffu, h ? v[e] : v[e + m], o);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {                    // keys 4 lane ..
          const float more = __fadd_rn(v[e], lost[e]), next = __fadd_rn(total[e], more);
          // (what rounding to `next` lost; nothing once that is infinite or NaN)
          lost[e] = fabsf(next) < INFINITY ? __fsub_rn(more, __fsub_rn(next, total[e])) : 0.f;
          total[e] = next;
        }
#pragma unroll
        for (int e = 0; e < 64; ++e) acc[e] = make_float2(0.f, 0.f);
      };
      // a row's numbers, asked for a tile ahead
      float l = -INFINITY, w = 0.f;
      auto ask = [&](int i) {
        l = -INFINITY;
        w = 0.f;
        const int tok = it.from + i % it.tiles * span + row_tok, head = it.head * a.group + i / it.tiles * a.pack + row_head;
        if (i < it.end && tok < it.to) {
          l = __ldg(lse + tok * a.lse_row + head * a.lse_head);
          w = rw ? __ldg(rw + tok) : 1.f;
        }
      };
      int held = 0;
      if (it.begin < it.end) ask(it.begin);
      for (int i = it.begin; i < it.end; ++i) {
        const float my_l = l, my_w = w;
        ask(i + 1);
        const int t = i % it.tiles;
        if (wg && t < it.skip) continue;
        const uint32_t b = su & 1;
        if (!warp_wait(&sh.sfull[wg][b], (su >> 1) & 1, gave_up, a.stats)) { ok = false; break; }
        fence_after();
        ++su;
        const bool counts = my_w != 0.f && my_l != -INFINITY;
        const int see = it.from + t * span + row_tok + shift - key0 + 1;     // keys of the group that the row sees
        const float2 f2 = make_float2(a.factor, a.factor), b2 = make_float2(-my_l * kLog2e, -my_l * kLog2e), w2 = make_float2(my_w, my_w);
        const bool all = __all_sync(0xffffffffu, counts && see >= kPrTile), some = __any_sync(0xffffffffu, counts && see > 0);
        uint32_t x[2][32];
        if (some) tmem_ask32(s_tm + b * 128, x[0]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (some) {
            tmem_wait32(x[k & 1]);
            if (k < 3) tmem_ask32(s_tm + b * 128 + (k + 1) * 32, x[(k + 1) & 1]);
          }
          if (k == 3) {
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.sfree[wg][b]);
          }
          if (all) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 z = fma2(make_float2(__uint_as_float(x[k & 1][2 * e]), __uint_as_float(x[k & 1][2 * e + 1])), f2, b2);
              acc[k * 16 + e] = fma2(make_float2(exp2_approx(z.x), exp2_approx(z.y)), w2, acc[k * 16 + e]);
            }
          } else if (counts && see > k * 32) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float z0 = 2 * e + k * 32 < see ? __uint_as_float(x[k & 1][2 * e]) : -INFINITY;
              const float z1 = 2 * e + 1 + k * 32 < see ? __uint_as_float(x[k & 1][2 * e + 1]) : -INFINITY;
              const float2 z = fma2(make_float2(z0, z1), f2, b2);
              acc[k * 16 + e] = fma2(make_float2(exp2_approx(z.x), exp2_approx(z.y)), w2, acc[k * 16 + e]);
            }
          }
          __syncwarp();
        }
        if (++held == kPwTogether) {
          held = 0;
          add_up();
        }
      }
      if (!ok) break;
      if (held) add_up();
      float (&sums)[4][kPrTile] = sh.sums[iu & 1][wg];
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[warp & 3][4 * lane + e] = total[e] + lost[e];
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.meet[wg]);
      if (!warp_wait(&sh.meet[wg], iu & 1, gave_up, a.stats)) break;
      const float sum = (sums[0][row] + sums[1][row]) + (sums[2][row] + sums[3][row]);
      if (shares > 1) {
        sh.shared[wg][row] = sum;
        break;                                           // (a cluster has one item)
      }
      const int key = key0 + row, keys = a.ks.first ? it.c : a.ks.rows;
      if (key < keys)
        a.weight[((a.ks.first ? 0ll : (long long)it.s * a.n_kv) + it.head) * a.ks.rows + it.k0 + key] = key < it.c ? sum : 0.f;
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPwRestRegs));
    if (warp == kPwLoader) {
      // ========================================================== loads ==========
      const PwOrder order = {&list, span, a.ks.first ? 0 : a.ks.rows};
      int level = 0;
      for (int s = lane; s < a.n_seq; s += 32) level = max(level, (list.n[s] + span - 1) / span);
      level = __reduce_max_sync(0xffffffffu, level);
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
        next.live = (shares == 1 || iu == 0) && prompt_find(order, a.n_seq, i / a.n_kv, lane, level, s, t);
        next.s = s;
        next.head = (int)(i % a.n_kv);
        next.key0 = t * 2 * kPrTile;
        next.n = list.n[s];
        next.c = list.c[s];
        next.q0 = list.q0[s];
        next.k0 = list.k0[s];
        const int shift = next.c - next.n;
        next.from = max(max(sh.from[s], next.key0 - shift), 0);
        next.to = sh.to[s];
        next.tiles = next.live && next.key0 < next.c && next.to > next.from ? (next.to - next.from + span - 1) / span : 0;
        next.skip = min(max((next.key0 + kPrTile - shift - next.from) / span, 0), next.tiles);
        if (next.key0 + kPrTile >= next.c) next.skip = next.tiles;           // B has no keys
        const long long all = (long long)packs * next.tiles;
        next.begin = (int)(all * rank / shares);
        next.end = (int)(all * (rank + 1) / shares);
        if (iu >= 2 && !warp_wait(&sh.item_free[iu & 1], ((iu >> 1) - 1) & 1, gave_up, a.stats)) break;
        if (lane == 0) {
          sh.item[iu & 1] = next;
          bar_arrive(&sh.item_full[iu & 1]);
        }
        if (next.begin < next.end) {
          const uint32_t place = ku & 1;
          if (ku >= 2 && !warp_wait(&sh.kfree[place], ((ku >> 1) - 1) & 1, gave_up, a.stats)) break;
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
          if (use > 0 && !warp_wait(&sh.free[st], (use - 1) & 1, gave_up, a.stats)) { ok = false; break; }
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
    } else if (warp == kPwIssuer) {
      // ========================================================== products =======
      const uint32_t idesc = idesc_16(kPrTile, false, kBf16) | (a.negate ? kNegateA : 0u);
      const uint64_t k_desc = desc128(kv_smem(kmat), 16), q_desc = desc128(kv_smem(ring), 16);
      constexpr uint64_t kStage = P::kMat >> 4;
      const bool leader = one_lane();
      uint32_t u = 0, ku = 0, su[2] = {0, 0};
      bool ok = true;
      for (uint32_t iu = 0; ok; ++iu) {
        if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, gave_up, a.stats)) break;
        const PwItem& it = sh.item[iu & 1];
        const int live = it.live, tiles = it.tiles, skip = it.skip, begin = it.begin, end = it.end;
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
        if (!live) break;
        if (begin >= end) continue;
        const uint32_t place = ku & 1;
        if (!warp_wait(&sh.kfull[place], (ku >> 1) & 1, gave_up, a.stats)) break;
        ++ku;
        const uint64_t kd = k_desc + place * 2 * kStage;
        for (int i = begin; i < end && ok; ++i, ++u) {
          const uint32_t st = u % P::kStages;
          if (!warp_wait(&sh.full[st], (u / P::kStages) & 1, gave_up, a.stats)) { ok = false; break; }
          const uint64_t qd = q_desc + st * kStage;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (g && i % tiles < skip) continue;
            const uint32_t b = su[g] & 1, use = su[g] >> 1;
            if (use > 0 && !warp_wait(&sh.sfree[g][b], (use - 1) & 1, gave_up, a.stats)) { ok = false; break; }
            ++su[g];
            fence_after();
            if (leader) {
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint64_t off = (uint64_t)((k >> 2) * (kPrTile * 128 >> 4) + (k & 3) * 2);
                mma_ss(tmem + g * 256 + b * 128, qd + off, kd + g * kStage + off, idesc, k > 0);
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
  }
  fence_before();
  __syncthreads();
  if (warp == kPwIssuer) {
    fence_after();
    // (as in attention: the sums waited for all products, and those for all copies, unless somebody gave up)
    if (*gave_up) {
      const unsigned long long t0 = now_ns();
      while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
  if (shares > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (rank == 0 && warp < 8) {
      const PwItem& it = sh.item[0];
      if (it.live) {
        const int wg = warp >> 2, row = tid & 127, key = it.key0 + tid, keys = a.ks.first ? it.c : a.ks.rows;
        float sum = sh.shared[wg][row];
        for (int r = 1; r < shares; ++r) sum += cluster.map_shared_rank(&sh, r)->shared[wg][row];
        if (key < keys)
          a.weight[((a.ks.first ? 0ll : (long long)it.s * a.n_kv) + it.head) * a.ks.rows + it.k0 + key] = key < it.c ? sum : 0.f;
      }
    }
    cluster.sync();                                      // (nobody leaves while its shared memory is read)
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
  // Fewer items than SMs: the rows of each are shared by a cluster.
  int shares = 1;
  while (shares < 8 && items * shares * 2 <= sms) shares *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items < sms ? items * shares : sms));
  cfg.blockDim = dim3(kPwThreads);
  cfg.dynamicSmemBytes = Pw<D>::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  if (shares > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = shares;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (!tl_pdl_off && pdl_process_ok()) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, prompt_weigh_kernel<D, kBf16>, qm, km, a, shares);
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
