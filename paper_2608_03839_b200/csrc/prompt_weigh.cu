// The attention weight that a prompt's keys receive, for its own queries:
//
//   w_j = sum over rows i >= j - (c - n) and the key head's query heads of r_i exp(scale q_i.k_j - lse_i)
//
// The product is taken the other way round than in attention, S = K Q^T: a row of TMEM is a key, its columns
// are query rows, so that a thread adds up one key's weight over all rows in registers and nothing is
// joined between threads or blocks.  A block takes items of 256 keys of one key head, in two groups
// A and B of 128 that stay in shared memory, and goes through the query rows that see them in tiles of 128:
// 128 / pack tokens of `pack` query heads.  Warps:
//   0-3, 4-7   a key a thread of A and of B: scores from TMEM (two places each), exponentials, sum
//   8          loads: the keys of an item, then tiles of queries into a ring, by tensor maps; and what a
//              row's exponent begins with, -lse log2 e, and the row's weight r
//   9          issues the products
// Rows that do not count (behind the sequence's last one, weight 0, lse -inf) have -inf there, and their
// scores are replaced, so that it does not matter what they hold.  Leading and trailing rows of a
// sequence with weight 0 are left out: the loading warp looks for the first and the last one that
// counts when it meets a sequence.
//
// Sums are fp32: of a tile's 128 columns as four, and over the tiles with the part that each addition
// loses carried along (a key may receive 10^5 terms).
//
// Every wait is bounded, as in attention.
#include "prompt.cuh"
#include "tensor.cuh"

namespace oilbird {

namespace {

constexpr int kPwThreads = 384, kPwLoader = 8, kPwIssuer = 9;
constexpr int kPwSumRegs = 208, kPwRestRegs = 88;
static_assert(2 * kPwSumRegs + kPwRestRegs <= 3 * 168, "more registers than the block was launched with");

struct PwItem {
  int s, head, key0;                 // first key of A
  int n, c, q0, k0;
  int from, tiles;                   // first token, tiles of queries for each of the head's packs of query heads
  int skip;                          // leading tiles that nothing of B is seen in
  int live;
};
struct PwShared {
  uint64_t full[8], free[8], kfull, kfree, sfull[2][2], sfree[2][2], item_full[2], item_free[2];
  PwItem item[2];
  alignas(16) float bias[8][kPrTile], weight[8][kPrTile];    // of a ring place's rows, read four at a time
  int whole[8];                                          // all of them count
  int from[kPrMaxSeq], to[kPrMaxSeq];                    // rows of a sequence that count; to < 0: not looked for yet
  uint32_t tmem;
  int gave_up;
};

template <int D>
struct Pw {
  static constexpr int kBlocks = D / 64, kMat = kBlocks * kPrTile * 128;
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr int kBytes = 1024 + (2 + kStages) * kMat + (int)sizeof(PwShared) + 16 + (int)sizeof(PromptList);
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

// The rows [from, to) of [0, n) outside which all weights are 0 (to 0: none is not); a warp.
__device__ __forceinline__ void live_rows(const float* w, int n, int lane, int& from, int& to) {
  constexpr int kAtOnce = 16;
  from = to = 0;
  for (int i0 = 0; i0 < n; i0 += 32 * kAtOnce) {
    float x[kAtOnce];
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) {
      const int i = i0 + e * 32 + lane;
      x[e] = i < n ? __ldg(w + i) : 0.f;
    }
    unsigned first = n;
#pragma unroll
    for (int e = kAtOnce - 1; e >= 0; --e) first = x[e] != 0.f ? i0 + e * 32 + lane : first;
    first = __reduce_min_sync(0xffffffffu, first);
    if ((int)first < n) { from = first; to = n; break; }
  }
  if (to == 0) return;
  for (int i0 = n; i0 > from; i0 -= 32 * kAtOnce) {
    float x[kAtOnce];
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) {
      const int i = i0 - 1 - e * 32 - lane;
      x[e] = i >= from ? __ldg(w + i) : 0.f;
    }
    int last = -1;
#pragma unroll
    for (int e = kAtOnce - 1; e >= 0; --e) last = x[e] != 0.f ? i0 - 1 - e * 32 - lane : last;
    last = __reduce_max_sync(0xffffffffu, last);
    if (last >= 0) { to = last + 1; break; }
  }
}

}  // namespace

template <int D, bool kBf16>
__global__ void __launch_bounds__(kPwThreads, 1)
prompt_weigh_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                    const __grid_constant__ PromptArgs a) {
  using P = Pw<D>;
  extern __shared__ unsigned char raw_smem[];
  unsigned char* smem = raw_smem + ((1024 - (kv_smem(raw_smem) & 1023)) & 1023);
  unsigned char* kmat = smem;                            // A, then B: [block of 64 channels][key]
  unsigned char* ring = smem + 2 * P::kMat;
  PwShared& sh = *reinterpret_cast<PwShared*>(ring + P::kStages * P::kMat);
  PromptList& list = *reinterpret_cast<PromptList*>(ring + P::kStages * P::kMat + (sizeof(PwShared) + 15) / 16 * 16);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* gave_up = &sh.gave_up;

  if (tid == 0) {
    for (int i = 0; i < P::kStages; ++i) {
      bar_init(&sh.full[i], 1);
      bar_init(&sh.free[i], 9);                          // the products and the eight warps that add up
    }
    bar_init(&sh.kfull, 1);
    bar_init(&sh.kfree, 1);
    for (int i = 0; i < 2; ++i) {
      for (int b = 0; b < 2; ++b) {
        bar_init(&sh.sfull[i][b], 1);
        bar_init(&sh.sfree[i][b], 4);
      }
      bar_init(&sh.item_full[i], 1);
      bar_init(&sh.item_free[i], 9);
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
  for (int s = tid; s < a.n_seq; s += kPwThreads) sh.to[s] = -1;
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
    const float2 f2 = make_float2(a.factor, a.factor);
    uint32_t u = 0, su = 0;
    bool ok = true;
    for (uint32_t iu = 0; ok; ++iu) {
      if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, gave_up, a.stats)) break;
      const PwItem it = sh.item[iu & 1];
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
      if (!it.live) break;
      const int key = it.key0 + wg * kPrTile + row;
      const int first_row = key - (it.c - it.n);         // the first row that sees the key
      const int skip = wg ? it.skip : 0;
      float total = 0.f, lost = 0.f;
      for (int x = 0; x < packs && ok; ++x)
        for (int t = 0; t < it.tiles; ++t, ++u) {
          const uint32_t st = u % P::kStages;
          // (also where nothing is done with the tile: its place is given back once each time it is full)
          if (!warp_wait(&sh.full[st], (u / P::kStages) & 1, gave_up, a.stats)) { ok = false; break; }
          if (t < skip) {
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.free[st]);
            continue;
          }
          const uint32_t b = su & 1;
          if (!warp_wait(&sh.sfull[wg][b], (su >> 1) & 1, gave_up, a.stats)) { ok = false; break; }
          fence_after();
          ++su;
          uint32_t y[128];
#pragma unroll
          for (int k = 0; k < 4; ++k) tmem_ask32(s_tm + b * 128 + k * 32, y + k * 32);
#pragma unroll
          for (int k = 0; k < 4; ++k) tmem_wait32(y + k * 32);
          fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.sfree[wg][b]);
          const int blind = min(max(first_row - (it.from + t * span), 0), span) * a.pack;     // columns whose rows do not see the key
          const float4* bias = reinterpret_cast<const float4*>(sh.bias[st]);
          const float4* weight = reinterpret_cast<const float4*>(sh.weight[st]);
          if (!sh.whole[st] || __any_sync(0xffffffffu, blind > 0)) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float4 bb = bias[e];
#pragma unroll
              for (int h = 0; h < 4; ++h)
                y[4 * e + h] = 4 * e + h >= blind && (&bb.x)[h] > -INFINITY ? y[4 * e + h] : 0xff800000u;
            }
          }
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float4 bb = bias[e], ww = weight[e];
            const float2 z0 = fma2(make_float2(__uint_as_float(y[4 * e]), __uint_as_float(y[4 * e + 1])), f2, make_float2(bb.x, bb.y));
            const float2 z1 = fma2(make_float2(__uint_as_float(y[4 * e + 2]), __uint_as_float(y[4 * e + 3])), f2, make_float2(bb.z, bb.w));
            sum[0] = fma2(make_float2(exp2_approx(z0.x), exp2_approx(z0.y)), make_float2(ww.x, ww.y), sum[0]);
            sum[1] = fma2(make_float2(exp2_approx(z1.x), exp2_approx(z1.y)), make_float2(ww.z, ww.w), sum[1]);
          }
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.free[st]);
          sum[0] = add2(sum[0], sum[1]);
          const float more = __fadd_rn(__fadd_rn(sum[0].x, sum[0].y), lost), next = __fadd_rn(total, more);
          // (what rounding to `next` lost; nothing once that is infinite or NaN)
          lost = fabsf(next) < INFINITY ? __fsub_rn(more, __fsub_rn(next, total)) : 0.f;
          total = next;
        }
      if (!ok) break;
      const int keys = a.ks.first ? it.c : a.ks.rows;
      if (key < keys)
        a.weight[((a.ks.first ? 0ll : (long long)it.s * a.n_kv) + it.head) * a.ks.rows + it.k0 + key] = key < it.c ? total : 0.f;
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
      uint32_t u = 0, ku = 0;
      bool ok = true;
      for (uint32_t iu = 0; ok; ++iu) {
        const long long i = (long long)iu * gridDim.x + (iu & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
        int s = 0, t = 0;
        const bool live = prompt_find(order, a.n_seq, i / a.n_kv, lane, level, s, t);
        PwItem it;
        it.live = live;
        it.s = s;
        it.head = (int)(i % a.n_kv);
        it.key0 = t * 2 * kPrTile;
        it.n = list.n[s];
        it.c = list.c[s];
        it.q0 = list.q0[s];
        it.k0 = list.k0[s];
        int from = 0, to = it.n;
        const float* rw = nullptr;
        if (a.row_weight) {
          rw = a.row_weight + (a.qs.first ? 0ll : (long long)s * a.qs.rows) + it.q0;
          if (live) {
            to = sh.to[s];
            from = sh.from[s];
            if (to < 0) {                                // (only this warp looks)
              live_rows(rw, it.n, lane, from, to);
              __syncwarp();
              if (lane == 0) { sh.from[s] = from; sh.to[s] = to; }
              __syncwarp();
            }
          }
        }
        const int shift = it.c - it.n;
        it.from = max(max(from, it.key0 - shift), 0);
        it.tiles = it.key0 < it.c && to > it.from ? (to - it.from + span - 1) / span : 0;
        it.skip = min(max((it.key0 + kPrTile - shift - it.from) / span, 0), it.tiles);
        if (it.key0 + kPrTile >= it.c) it.skip = it.tiles;                   // B has no keys
        if (iu >= 2 && !warp_wait(&sh.item_free[iu & 1], ((iu >> 1) - 1) & 1, gave_up, a.stats)) break;
        if (lane == 0) {
          sh.item[iu & 1] = it;
          bar_arrive(&sh.item_full[iu & 1]);
        }
        if (!live) break;
        if (it.tiles == 0) continue;
        const int qs = a.qs.first ? 0 : s, ks = a.ks.first ? 0 : s;
        if (ku > 0 && !warp_wait(&sh.kfree, (ku - 1) & 1, gave_up, a.stats)) break;
        ++ku;
        if (leader) {
          bar_expect(&sh.kfull, 2 * P::kMat);
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int b = 0; b < P::kBlocks; ++b)
              map_load4(kv_smem(kmat + g * P::kMat + b * (kPrTile * 128)), &k_map, b * 64, it.head,
                        it.k0 + it.key0 + g * kPrTile, ks, &sh.kfull);
        }
        __syncwarp();
        const float* lse = a.lse + qs * a.lse_seq + it.q0 * a.lse_row;
        for (int x = 0; x < packs && ok; ++x) {
          const int head0 = it.head * a.group + x * a.pack;
          for (int j = 0; j < it.tiles; ++j, ++u) {
            const uint32_t st = u % P::kStages, use = u / P::kStages;
            const int tok0 = it.from + j * span;
            float l[4], w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = e * 32 + lane, tok = tok0 + r / a.pack, hd = head0 + r % a.pack;
              l[e] = -INFINITY;
              w[e] = 0.f;
              if (tok < to) {
                l[e] = lse[tok * a.lse_row + hd * a.lse_head];
                w[e] = rw ? rw[tok] : 1.f;
              }
            }
            if (use > 0 && !warp_wait(&sh.free[st], (use - 1) & 1, gave_up, a.stats)) { ok = false; break; }
            bool counts = true;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool c = w[e] != 0.f && l[e] != -INFINITY;
              sh.bias[st][e * 32 + lane] = c ? -l[e] * kLog2e : -INFINITY;
              sh.weight[st][e * 32 + lane] = c ? w[e] : 0.f;
              counts &= c;
            }
            counts = __all_sync(0xffffffffu, counts);
            if (lane == 0) sh.whole[st] = counts;
            __syncwarp();
            if (leader) {
              bar_expect(&sh.full[st], P::kMat);
#pragma unroll
              for (int b = 0; b < P::kBlocks; ++b)
                map_load4(kv_smem(ring + st * P::kMat + b * (kPrTile * 128)), &q_map, b * 64, head0, it.q0 + tok0, qs, &sh.full[st]);
            }
            __syncwarp();
          }
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
        if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, gave_up, a.stats)) break;
        const int live = sh.item[iu & 1].live, tiles = sh.item[iu & 1].tiles, skip = sh.item[iu & 1].skip;
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
        if (!live) break;
        if (tiles == 0) continue;
        if (!warp_wait(&sh.kfull, ku++ & 1, gave_up, a.stats)) break;
        for (int x = 0; x < packs && ok; ++x)
          for (int t = 0; t < tiles && ok; ++t, ++u) {
            const uint32_t st = u % P::kStages;
            if (!warp_wait(&sh.full[st], (u / P::kStages) & 1, gave_up, a.stats)) { ok = false; break; }
            const uint64_t qd = q_desc + st * kStage;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              if (g && t < skip) continue;
              const uint32_t b = su[g] & 1, use = su[g] >> 1;
              if (use > 0 && !warp_wait(&sh.sfree[g][b], (use - 1) & 1, gave_up, a.stats)) { ok = false; break; }
              ++su[g];
              fence_after();
              if (leader) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                  const uint64_t off = (uint64_t)((k >> 2) * (kPrTile * 128 >> 4) + (k & 3) * 2);
                  mma_ss(tmem + g * 256 + b * 128, k_desc + g * kStage + off, qd + off, idesc, k > 0);
                }
                commit(&sh.sfull[g][b]);
              }
              __syncwarp();
            }
            if (!ok) break;
            if (leader) {
              commit(&sh.free[st]);
              if (x + 1 == packs && t + 1 == tiles) commit(&sh.kfree);
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
  return launch_pdl(prompt_weigh_kernel<D, kBf16>, dim3((unsigned)(items < sms ? items : sms)), dim3(kPwThreads), Pw<D>::kBytes, st,
                    qm, km, a);
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
