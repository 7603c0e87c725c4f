// Attention over whole prompts: causal, grouped query heads, sequences of different lengths, on the
// tensor cores with accumulators in TMEM.
//
//   out_i = sum_j exp(x_ij - lse_i) v_j,  lse_i = ln sum_j exp x_ij,  x_ij = scale q_i.k_j,  j <= i + c - n
//
// One pass over the keys with a running maximum.  A block takes items of 256 query rows of one key
// head, in two groups A and B of 128.  `pack` query heads that share the key head lie side by side, so a
// group is 128 / pack tokens: every tile of keys serves all of them, and fewer keys lie beyond the
// diagonal.  Warps:
//   0-7, 8-15  softmax of A and of B, 16 rows a warp, four lanes to a row: scores from TMEM, maximum,
//              exponentials, and the probabilities in 16 bits back over the scores
//   16         loads: queries, then keys and values in turn into a ring, by tensor maps
//   17         issues the products S = Q K^T and O += P V (P from TMEM)
//   18, 19     put zeros over values behind a sequence's last and, where they matter, over those that are not finite
// While A's scores go through the exponentials the tensor core works for B, and the other way round.
//
// Numbers.  Scores, maxima, sums and accumulators are fp32.  Probabilities are rounded to the inputs'
// type, as the product wants both operands alike (off by 2^-8 of each at most in bf16, 2^-11 in f16); the
// sum takes them unrounded.  m follows the row's maximum only when that has grown by 2^8 (the accumulators are
// rescaled in TMEM then), so p reaches 2^8; f16 takes them 2^7 higher, where its range ends, as
// what lies 17 below the maximum (in exp's units) would otherwise be rounded to nothing.  bf16 takes them lower, as many
// keys' large values would otherwise add up to more than fp32 holds (see room_of).
//
// Values that are not finite.  A masked key's probability is 0, and 0 times an infinity would reach every row of the
// tile.  Before the product of a tile that passes the sequence's last key two warps put zeros there (padding may hold
// anything).  And an item with a row whose accumulators are not finite is done once more: of its tiles the last ones, up
// to three, hold keys of tokens behind one of its rows, and for those keys the two warps now put zeros in place of
// infinities and NaN.  The rows that do see such a key have its value added when they are written.  (In clusters, which have one
// item, that is done at once.  For every item it took 16 prompts from 225 to 243 us.)
//
// Work.  Items by falling number of key tiles, so that the last ones are the short ones; block b takes
// b, 2G-1-b, 2G+b, ... of G blocks (see prompt_find).
//
// Where there are fewer items than SMs (few rows, over many keys perhaps) the key tiles of an item are shared
// by a cluster of blocks.  Each leaves its rows' maxima, sums and accumulators in its shared memory, and a
// part of the rows is joined by each block, in the order of the keys.
//
// Measured, with 32 query heads over 8 key heads of 128: one prompt of 32,768 tokens in 7.5 ms (8.8 TFLOP, 1,174
// TFLOP/s; 6.3 ms at cuBLAS's sustained rate), 16 of up to 2,048 in 219 us (an infinity that all their rows see, so that
// every item is done twice: 2.4 times as long), one of 37 in 10.4 us, one token over 32,768 keys in 71 us (64
// blocks, and half of each idles: an item of few rows has none for group B).  Heads of 64: 8,192 tokens in 345 us.
// What bounds long prompts is power: 990 W at 1,520 MHz, where a step of 256 rows by 128 keys takes 3,200 cycles, its
// exponentials and its products 2,048 each (tensor pipe 59 %, exponential unit 60 %).  Polynomials in place of an eighth to half of the exponentials were slower by 1 to 7 %.  A row
// a thread, with 8 warps, left the exponentials to two warps an SM quarter (7.9 ms).
// Short prompts wait for an item's chain: loads, products, a tile's exponentials, products, the rows' way out.
//
// Every wait is bounded (two seconds unless set otherwise): a wait that runs out raises `stalled`, all
// roles leave, TMEM is freed.
#include <cooperative_groups.h>

#include <atomic>

#include "prompt.cuh"
#include "tensor.cuh"

namespace cg = cooperative_groups;

namespace oilbird {

namespace {

constexpr int kPaThreads = 640, kPaSoftWarps = 16, kPaLoader = 16, kPaIssuer = 17, kPaCleaner = 18, kPaCleaners = 2;
// registers a thread: launched with 96; the five warpgroups' shares add up to 5 x 96
constexpr int kPaSoftRegs = 112, kPaRestRegs = 32;
static_assert(4 * kPaSoftRegs + kPaRestRegs <= 5 * 96, "more registers than the block was launched with");
constexpr float kPaLn2 = 0.6931471805599453f;
constexpr int kPaSlack = 8;

struct PaItem {
  int s, tok, head, q_head;          // sequence, first token, key head, first query head
  int n, c, q0, k0;
  int tiles[2];                      // of A and of B: all that their rows see
  int seen, part;                    // keys that every row sees; the tile in which they end
  int clean;                         // from this tile on values are cleaned: part, or none
  int begin;                         // this block's: from here on,
  int end[2];                        // up to here
  float room;                        // probabilities are 2^room times as large
  int live;                          // 0: no item is left
};
// f16 probabilities use the type's whole range (see above).  In bf16, which ends where fp32 does, they are so small
// that neither their sum over `tiles` of keys, each up to 2^kPaSlack, reaches 1, nor the sum of the values that they weigh
// fp32's end: as far down as values of 2^-117 over 2,048 keys that costs no bit.
template <bool kBf16>
__device__ __forceinline__ float room_of(int tiles) {
  return kBf16 ? -(float)(1 + kPaSlack + 7 + (tiles > 1 ? 32 - __clz(tiles - 1) : 0)) : 7.f;
}
// A row's exponents are x f - m f + room with f = scale log2 e and m the running maximum of its scores x.  One fused
// multiply-add does that while m f is small: what rounding m f loses is the same in every exponent.  Beyond 2^20
// that would be worth something, beyond 2^24 whole powers of two, and m f may be infinite: there the difference x - m
// comes first.
constexpr float kPaFar = 1048576.f;
__device__ __forceinline__ bool row_far(float m, float f) { return fabsf(m * f) > kPaFar && m != -INFINITY; }
__device__ __forceinline__ float row_shift(float m, float f, float room) {
  return fabsf(m * f) <= kPaFar ? fmaf(-m, f, room) : room;      // (no maximum yet: room)
}
// log2 of what sums and accumulators under the maximum `from` are multiplied with to be under `to`
__device__ __forceinline__ float row_fall(float from, float to, float f, float room) {
  const float far = (from - to) * f, near = row_shift(to, f, room) - row_shift(from, f, room);
  return fabsf(from * f) <= kPaFar && fabsf(to * f) <= kPaFar ? near : far;      // (branches here took a microsecond an item)
}
// (the room is taken out of the sum, which is exact: as part of the logarithm it would cost its last bits)
__device__ __forceinline__ float row_lse(float m, float l, float f, float room) {
  const float ls = __log2f(l * __int_as_float((127 - (int)room) << 23));
  return row_far(m, f) ? fmaf(m, f * kPaLn2, ls * kPaLn2) : (ls - (row_shift(m, f, room) - room)) * kPaLn2;
}
struct PaShared {
  uint64_t full[16], free[16], qfull, qfree, sfull[2], pfull[2][2], ofull[2], item_full[2], item_free[2], meet;
  uint64_t ask, clean, found, written[2];
  PaItem item[2];
  int again[2];                                          // the item has to be done again, with clean values
  uint32_t asked;                                        // the use of the ring whose values are to be cleaned
  struct Odd { int from, to; } odd[kPaCleaners];         // keys among which values were taken out
  float2 ml[2][256];                                     // maxima and sums of A's rows and B's, of items that are cleaned
  uint32_t tmem;
  Waits waits;
};

template <int D>
struct Pa {
  static constexpr int kBlocks = D / 64, kMat = kBlocks * kPrTile * 128;      // one tile of 128 rows
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr int kBytes = 1024 + (2 + kStages) * kMat + (int)sizeof(PaShared) + 16 + (int)sizeof(PromptList);
  static_assert(kBytes <= 227 * 1024, "shared memory");
  // accumulators of a block of a cluster, over the tiles; rows spread over the banks
  static constexpr int kRow = D + 8;
  static_assert(256 * kRow * 4 <= (2 + kStages) * kMat, "accumulators in the tiles' place");
};

// Items of 2 `span` tokens.  Those with more keys lie behind those with fewer; in the padded form what
// lies behind a sequence's rows is written too.
struct PaOrder {
  const PromptList* l;
  int log_span, padded;              // tokens of an item; rows to write for every sequence (0: packed)
  __device__ __forceinline__ int ceil(int rows) const { return (int)(((unsigned)rows + (1u << log_span) - 1) >> log_span); }
  __device__ __forceinline__ int there(int s) const { return ceil(l->n[s]); }
  __device__ __forceinline__ int most_tiles(int s) const { return (l->c[s] + kPrTile - 1) / kPrTile; }
  // items of sequence s with `level` units of key tiles or more
  __device__ __forceinline__ int items(int s, int level, int unit) const {
    if (level == 0) return padded ? ceil(padded) : there(s);
    const int c = l->c[s], n = l->n[s];
    const long long keys = (long long)(level - 1) * unit * kPrTile;      // the last row of the item sees more than these
    if (c <= keys) return 0;
    const long long d = (keys - c + n) >> log_span;
    return d > 0 ? (int)max(there(s) - d, 0ll) : there(s);
  }
  // the `at`-th item of sequence s among those of one level; `all` items have that level or more, `above` more
  __device__ __forceinline__ int item(int s, int level, int at, int all, int above) const {
    if (level > 0) return there(s) - all + at;
    return at < there(s) - above ? at : at + above;      // rows in front that see nothing, then padding
  }
};

// Two results in the type: of finite accumulators o the largest number of the type where u, rounded, lies behind it (the
// probabilities are rounded, the sum that divides them is not, so that a result may pass the largest value that it is
// made of).
template <bool kBf16>
__device__ __forceinline__ uint32_t pack_finite(float lo, float hi) {
  uint32_t r;
  if (kBf16) asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack_result(float o0, float o1, float u0, float u1) {
  const uint32_t a = pack_finite<kBf16>(u0, u1), b = pack16<kBf16>(u0, u1);
  return ((fabsf(o0) < INFINITY ? a : b) & 0xffffu) | ((fabsf(o1) < INFINITY ? a : b) & 0xffff0000u);
}

// The sign bits of those halves of a word that are not finite.
template <bool kBf16>
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) {
  return ((w & (kBf16 ? 0x7f807f80u : 0x7c007c00u)) + (kBf16 ? 0x00800080u : 0x04000400u)) & 0x80008000u;
}
// Adds a lane's channels (pairs, 64 apart) of values [from, to) that are not finite.
template <int D, bool kBf16>
__device__ __forceinline__ void add_odd(const PromptArgs& a, const PaItem& it, int from, int to, int lane, float2 (&sum)[D / 64]) {
#pragma unroll 2
  for (int j = from; j < to; ++j)
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(a.v.at(a.ks.first ? 0 : it.s, it.k0 + j, it.head) + e * 64 + 2 * lane);
      const uint32_t odd = odd_halves<kBf16>(w);
      if (odd & 0xffffu) sum[e].x += half_lo<kBf16>(w);
      if (odd >> 16) sum[e].y += half_hi<kBf16>(w);
    }
}
// The values among keys [from, to) that were taken out, added to those of an item's rows [row0, row0 + 128) that see them; a
// warp.  The rows' tokens rise, and so does what they see.
template <int D, bool kBf16>
__device__ __forceinline__ void odd_rows(const PromptArgs& a, const PaItem& it, const float2* ml, int row0, int from, int to,
                                         int lane) {
  float2 sum[D / 64];
#pragma unroll
  for (int e = 0; e < D / 64; ++e) sum[e] = make_float2(0.f, 0.f);
  int at = from;
#pragma unroll 1
  for (int row = row0; row < row0 + 128; ++row) {
    const int tok = it.tok + (row >> a.log_pack), stop = min(min(it.c, it.c - it.n + tok + 1), to);
    if (tok >= it.n) break;
    if (stop <= from) continue;                          // it sees none of them
    add_odd<D, kBf16>(a, it, at, stop, lane, sum);
    at = max(at, stop);
    if (ml[row].y == 0.f) continue;                      // it sees nothing
    uint16_t* op = a.out + (a.qs.first ? 0 : it.s) * a.out_seq + (long long)(it.q0 + tok) * a.out_row +
                   (it.q_head + (row & (a.pack - 1))) * a.out_head + 2 * lane;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
      const bool x = !(fabsf(sum[e].x) < INFINITY), y = !(fabsf(sum[e].y) < INFINITY);
      if (!x && !y) continue;
      uint32_t* at_e = reinterpret_cast<uint32_t*>(op + e * 64);
      const uint32_t was = *at_e, w = pack16<kBf16>(half_lo<kBf16>(was) + sum[e].x, half_hi<kBf16>(was) + sum[e].y);
      *at_e = ((x ? w : was) & 0xffffu) | ((y ? w : was) & 0xffff0000u);
    }
  }
}

// The item of a cluster.  First every block leaves its accumulators in its shared memory (a softmax warp its 16 rows) ..
template <int D>
__device__ __forceinline__ void leave_rows(float* acc, uint32_t o_tm, int row0) {
  const int quad = threadIdx.x & 3;
#pragma unroll 1
  for (int k = 0; k < D; k += 32) {
    uint32_t o[16];
    tmem_ask_rows(o_tm + k, o);
    tmem_wait_rows(o);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r)
        *reinterpret_cast<float2*>(acc + (row0 + 8 * r) * Pa<D>::kRow + k + 8 * i + 2 * quad) =
            make_float2(__uint_as_float(o[4 * i + 2 * r]), __uint_as_float(o[4 * i + 2 * r + 1]));
  }
}
// .. then it joins its part of the 256 rows, a row a softmax warp.
template <int D, bool kBf16>
__device__ __noinline__ void join_rows(const PromptArgs& a, PaShared& sh, float* acc, int shares, int rank) {
  const PaItem& it = sh.item[0];
  float2* ml = sh.ml[0];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  cg::cluster_group cluster = cg::this_cluster();
  constexpr int E = D / 64;                            // pairs of channels a lane
  const int rows = 256 / shares;
  PaShared::Odd odd = {0x7fffffff, 0};
  static_assert(16 * kPaCleaners <= 32, "a lane for each of a cluster's");
  if (lane < shares * kPaCleaners) odd = cluster.map_shared_rank(&sh, lane / kPaCleaners)->odd[lane % kPaCleaners];
  odd.from = __reduce_min_sync(0xffffffffu, odd.from);
  odd.to = __reduce_max_sync(0xffffffffu, odd.to);
  for (int i = warp; i < rows; i += kPaSoftWarps) {    // a row a warp
    const int row = rank * rows + i, tok = it.tok + (row >> a.log_pack), head = it.q_head + (row & (a.pack - 1));
    if (tok >= (a.qs.first ? it.n : a.qs.rows)) continue;
    float big = -INFINITY, sum = 0.f;
    for (int s = 0; s < shares; ++s) big = fmaxf(big, cluster.map_shared_rank(ml, s)[row].x);
    float2 o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = make_float2(0.f, 0.f);
    for (int s = 0; s < shares; ++s) {
      const float2 y = cluster.map_shared_rank(ml, s)[row];
      if (y.x == -INFINITY && y.y == 0.f) continue;    // it saw nothing there
      const float f = y.x == big ? 1.f : exp2_approx(row_fall(y.x, big, a.factor, it.room));
      const float* from = cluster.map_shared_rank(acc, s) + row * Pa<D>::kRow + 2 * lane;
      sum = fmaf(f, y.y, sum);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 x = *reinterpret_cast<const float2*>(from + 64 * e);
        o[e].x = fmaf(f, x.x, o[e].x);
        o[e].y = fmaf(f, x.y, o[e].y);
      }
    }
    if (odd.from < odd.to) add_odd<D, kBf16>(a, it, odd.from, min(odd.to, min(it.c, it.c - it.n + tok + 1)), lane, o);
    const float inv = sum == 0.f ? 0.f : __frcp_rn(sum);
    const long long seq = a.qs.first ? 0 : it.s, at = (long long)it.q0 + tok;
    uint16_t* op = a.out + seq * a.out_seq + at * a.out_row + head * a.out_head + 2 * lane;
#pragma unroll
    for (int e = 0; e < E; ++e)
      *reinterpret_cast<uint32_t*>(op + 64 * e) = sum == 0.f ? 0u : pack_result<kBf16>(o[e].x, o[e].y, o[e].x * inv, o[e].y * inv);
    if (lane == 0 && a.lse)
      a.lse[seq * a.lse_seq + at * a.lse_row + head * a.lse_head] = sum == 0.f ? -INFINITY : row_lse(big, sum, a.factor, it.room);
  }
}

}  // namespace

template <int D, bool kBf16, bool kSplit>
__global__ void __launch_bounds__(kPaThreads, 1)
prompt_attend_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                     const __grid_constant__ CUtensorMap v_map, const __grid_constant__ PromptArgs a, int blocks) {
  using P = Pa<D>;
  const int shares = kSplit ? blocks : 1;                // of an item, one a block of a cluster
  extern __shared__ unsigned char raw_smem[];
  unsigned char* smem = raw_smem + ((1024 - (kv_smem(raw_smem) & 1023)) & 1023);
  unsigned char* qmat = smem;                            // A, then B: [block of 64 channels][row]
  unsigned char* ring = smem + 2 * P::kMat;
  PaShared& sh = *reinterpret_cast<PaShared*>(ring + P::kStages * P::kMat);
  PromptList& list = *reinterpret_cast<PromptList*>(ring + P::kStages * P::kMat + (sizeof(PaShared) + 15) / 16 * 16);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile Waits* waits = &sh.waits;

  if (tid == 0) {
    for (int i = 0; i < P::kStages; ++i) {
      bar_init(&sh.full[i], 1);
      bar_init(&sh.free[i], 1);
    }
    bar_init(&sh.qfull, 1);
    bar_init(&sh.qfree, 1);
    bar_init(&sh.meet, kPaSoftWarps);
    for (int i = 0; i < 2; ++i) {
      bar_init(&sh.sfull[i], 1);
      for (int h = 0; h < 2; ++h) bar_init(&sh.pfull[i][h], kPaSoftWarps / 2);
      bar_init(&sh.ofull[i], 1);
      bar_init(&sh.item_full[i], 1);
      bar_init(&sh.item_free[i], kPaSoftWarps + 1 + kPaCleaners);
      bar_init(&sh.written[i], kPaSoftWarps);
      sh.again[i] = 0;
    }
    bar_init(&sh.ask, 1);
    bar_init(&sh.clean, kPaCleaners);
    bar_init(&sh.found, kPaCleaners);
    for (int x = 0; x < kPaCleaners; ++x) sh.odd[x] = {0x7fffffff, 0};
    sh.item[0].live = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kPaIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(kv_smem(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_enter();
  if (tid == 0) waits_begin(sh.waits, &a.stats->wait_limit_ns);
  prompt_extents(a, list);
  const PaOrder order = {&list, 8 - a.log_pack, a.qs.first ? 0 : a.qs.rows};
  __syncthreads();
  prompt_levels(order, a.n_seq, list);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  const int span = kPrTile >> a.log_pack;                // tokens of a group
  const int rank = kSplit ? blockIdx.x % shares : 0;     // in the cluster

  // The roles leave when no item is left.  They meet then, and go on if the last one has to be done again, with the number
  // behind that of the item that was none.  (Only behind the barrier is it known for good whether somebody gave up.)
  auto over = [&](uint32_t iu) {
    if (kSplit) return true;
    fence_before();
    __syncthreads();
    return waits->gave_up || !*const_cast<volatile int*>(&sh.again[(iu + 1) & 1]);
  };

  if (warp < kPaSoftWarps) {
    // ============================================================ softmax ========
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPaSoftRegs));
    const int wg = warp >> 3, quad = lane & 3;
    const int row0 = (warp & 3) * 32 + (warp >> 2 & 1) * 16 + (lane >> 2);       // the lane's rows: this one and 8 on
    const uint32_t s_tm = tmem + ((uint32_t)((warp & 3) * 32 + (warp >> 2 & 1) * 16) << 16) + wg * 128, o_tm = s_tm + 256;
    const float2 g2 = make_float2(a.factor, a.factor);
    uint32_t su = 0, ou = 0;
    bool ok = true;
    uint32_t iu = 0;
    do {
      for (; ok; ++iu) {
        if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, waits, a.stats)) break;
        // (read again where the rows are written: there are no registers to keep it in)
        volatile const PaItem& now = sh.item[iu & 1];
        if (!now.live) break;
        int vis[2];                                        // keys the row sees (0 or less: none)
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int tok = now.tok + wg * span + ((row0 + 8 * r) >> a.log_pack), n = now.n, c = now.c;
          vis[r] = tok < n ? min(c, c - n + tok + 1) : 0;
        }
        for (int j = now.begin; j < now.end[wg]; ++j, ++su) {
          if (!warp_wait(&sh.sfull[wg], su & 1, waits, a.stats)) { ok = false; break; }
          fence_after();
          uint32_t x[64];
          tmem_ask_rows(s_tm, x);
          tmem_wait_rows(x);
          if (__any_sync(0xffffffffu, min(vis[0], vis[1]) < (j + 1) * kPrTile)) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int see = vis[r] - j * kPrTile - 2 * quad;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                if (8 * i >= see) x[4 * i + 2 * r] = 0xff800000u;
                if (8 * i + 1 >= see) x[4 * i + 2 * r + 1] = 0xff800000u;
              }
            }
          }
          float mx[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float y[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 16; ++i)
              y[i & 1] = max3(y[i & 1], __uint_as_float(x[4 * i + 2 * r]), __uint_as_float(x[4 * i + 2 * r + 1]));
            mx[r] = fmaxf(y[0], y[1]);
          }
#pragma unroll
          for (int o = 1; o < 4; o <<= 1) {
            mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], o));
            mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], o));
          }
          const float room = kBf16 ? now.room : 7.f;
          // (differences of scores: as products with the factor both may be infinite)
          if (__any_sync(0xffffffffu, (mx[0] - m[0]) * a.factor > kPaSlack || (mx[1] - m[1]) * a.factor > kPaSlack)) {
            // (each row for itself; the products so far are done, or there were no scores)
            float down[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float mn = (mx[r] - m[r]) * a.factor > kPaSlack ? mx[r] : m[r];
              down[r] = mn == m[r] ? 1.f : exp2_approx(row_fall(m[r], mn, a.factor, room));
              m[r] = mn;
              l[r] *= down[r];
            }
            if (j > now.begin) {
#pragma unroll 1
              for (int k = 0; k < D; k += 32) {
                uint32_t r[16];
                tmem_ask_rows(o_tm + k, r);
                tmem_wait_rows(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * down[e >> 1 & 1]);
                tmem_st_rows(o_tm + k, r);
              }
            }
          }
          if (__any_sync(0xffffffffu, row_far(m[0], a.factor) || row_far(m[1], a.factor))) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float less = row_far(m[r], a.factor) ? m[r] : 0.f;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                x[4 * i + 2 * r] = __float_as_uint(__uint_as_float(x[4 * i + 2 * r]) - less);
                x[4 * i + 2 * r + 1] = __float_as_uint(__uint_as_float(x[4 * i + 2 * r + 1]) - less);
              }
            }
          }
          float2 shift2[2], sum[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float shift = row_shift(m[r], a.factor, room);
            shift2[r] = make_float2(shift, shift);
            sum[r] = make_float2(0.f, 0.f);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const int e = 16 * k + 4 * i + 2 * r;
                const float2 z = fma2(make_float2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), g2, shift2[r]);
                const float2 pr = make_float2(exp2_approx(z.x), exp2_approx(z.y));
                sum[r] = add2(sum[r], pr);
                w[2 * i + r] = pack16<kBf16>(pr.x, pr.y);
              }
            tmem_st_pairs(s_tm + k * 16, w);               // over the scores
            if (k & 1) {                                   // a half of the keys: their product can begin
              tmem_wait_st();
              fence_before();
              __syncwarp();
              if (lane == 0) bar_arrive(&sh.pfull[wg][k >> 1]);
            }
          }
          l[0] += sum[0].x + sum[0].y;
          l[1] += sum[1].x + sum[1].y;
        }
        if (!ok) break;
        const bool any = now.end[wg] > now.begin;
        if (any) {
          if (!warp_wait(&sh.ofull[wg], ou++ & 1, waits, a.stats)) break;
          fence_after();
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
          l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        }
        if (kSplit) {                                      // (a cluster has one item, joined below)
          if (quad == 0) {
            sh.ml[0][wg * 128 + row0] = make_float2(m[0], l[0]);
            sh.ml[0][wg * 128 + row0 + 8] = make_float2(m[1], l[1]);
          }
          break;
        }
        // ---- out ----
        // (Once a tile of short prompts: every instruction counts.  A row's four lanes swap their words in two steps, so
        // that each has eight columns that lie together.)
        const PaItem& it = sh.item[iu & 1];
        const long long seq = a.qs.first ? 0 : it.s;
        const float zero = 0.f;
        float2 inv[2], odd2[2];
        uint16_t* op[2];
        int tok[2], head[2];
        bool write[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float i = l[r] == 0.f ? 0.f : __frcp_rn(l[r]);
          inv[r] = make_float2(i, i);
          odd2[r] = make_float2(0.f, 0.f);
          tok[r] = it.tok + wg * span + ((row0 + 8 * r) >> a.log_pack);
          head[r] = it.q_head + ((row0 + 8 * r) & (a.pack - 1));
          write[r] = tok[r] < (a.qs.first ? it.n : a.qs.rows);
          const long long row = (long long)it.q0 + tok[r];
          op[r] = a.out + seq * a.out_seq + row * a.out_row + head[r] * a.out_head + 8 * quad;
          if (write[r] && a.lse && quad == 0)
            a.lse[seq * a.lse_seq + row * a.lse_row + head[r] * a.lse_head] =
                l[r] == 0.f ? -INFINITY : row_lse(m[r], l[r], a.factor, it.room);
        }
        // (a second time where a row has accumulators that are not finite: those results are infinite or NaN too)
        for (bool exact = false;; exact = true) {
#pragma unroll 1
          for (int k = 0; k < D; k += 32) {
            uint32_t o[16];
            if (any) {
              tmem_ask_rows(o_tm + k, o);
              tmem_wait_rows(o);
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              uint32_t w[4];                               // columns 8i + 2 quad, .. of the 32
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float2 x = make_float2(__uint_as_float(o[4 * i + 2 * r]), __uint_as_float(o[4 * i + 2 * r + 1]));
                const float2 u = mul2(x, inv[r]);
                odd2[r] = fma2(x, make_float2(zero, zero), odd2[r]);           // (NaN once one is not finite)
                w[i] = l[r] == 0.f ? 0u : exact ? pack_result<kBf16>(x.x, x.y, u.x, u.y) : pack_finite<kBf16>(u.x, u.y);
              }
#pragma unroll
              for (int x = 2; x; x >>= 1) {
                const bool up = quad & x;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (!(i & x)) {
                    const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[i] : w[i + x], x);
                    w[i] = up ? got : w[i];
                    w[i + x] = up ? w[i + x] : got;
                  }
              }
              if (write[r]) *reinterpret_cast<uint4*>(op[r] + k) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
          const bool odd = (l[0] != 0.f && !(odd2[0].x + odd2[0].y == 0.f)) || (l[1] != 0.f && !(odd2[1].x + odd2[1].y == 0.f));
          if (exact || !__any_sync(0xffffffffu, any && odd)) break;
          if (it.clean != it.part && it.part < max(it.tiles[0], it.tiles[1])) {
            if (lane == 0) sh.again[iu & 1] = 1;
            break;
          }
        }
        // Warps 18 and 19 add what they have taken out.  (A group without tiles may be here while they are still at the item
        // before: each place has sums and a barrier of its own, and they give it back when they are through.)
        if (it.clean == it.part) {
          if (quad == 0) {
            sh.ml[iu & 1][wg * 128 + row0] = make_float2(m[0], l[0]);
            sh.ml[iu & 1][wg * 128 + row0 + 8] = make_float2(m[1], l[1]);
          }
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.written[iu & 1]);
        }
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
      }
    } while (!over(iu++));
    if (kSplit) {
      // (the tiles' place is free when both groups have their last products)
      float* acc = reinterpret_cast<float*>(smem);
      const PaItem& it = sh.item[0];
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.meet);
      if (warp_wait(&sh.meet, 0, waits, a.stats) && it.live && it.end[wg] > it.begin) leave_rows<D>(acc, o_tm, wg * 128 + row0);
      fence_before();
      meet_cluster();
      if (it.live) join_rows<D, kBf16>(a, sh, acc, shares, rank);
      meet_cluster();                                    // (nobody leaves while its shared memory is read)
      fence_before();
      __syncthreads();
    }
    return;                                              // (see below)
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPaRestRegs));
    if (warp == kPaLoader) {
      // ========================================================== loads ==========
      int level = list.levels;                           // of the last item found: the next one has no more
      const int heads = a.n_kv * (a.group / a.pack);
      const bool leader = one_lane();
      const int crew = gridDim.x / shares, me = blockIdx.x / shares;
      uint32_t u = 0, qu = 0, no = 0;
      int s = 0, t = 0, hd = 0;
      bool ok = true, live = false, used = true;         // the item found last: there is one; it has been posted
      uint32_t iu = 0;
      bool ended = false;
      do {
        for (; ok; ++iu) {
          if (used) {
            const long long i = (long long)no * crew + (no & 1 ? crew - 1 - me : me);
            hd = (int)(i % heads);
            live = (!kSplit || no == 0) && prompt_find(order, a.n_seq, list, (int)(i / heads), lane, level, s, t);
            ++no;
          }
          // An item that has to be done again goes first, in the place that it had.  (Once the roles have met all are free.)
          if (iu >= 2 && !ended && !warp_wait(&sh.item_free[iu & 1], ((iu >> 1) - 1) & 1, waits, a.stats)) break;
          used = kSplit || !*const_cast<volatile int*>(&sh.again[iu & 1]);
          PaItem& it = sh.item[iu & 1];
          if (used) {
            const int head = hd / (a.group / a.pack), tok = t * 2 * span, n = list.n[s], c = list.c[s];
            int tiles[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const int last = min(n, tok + (g + 1) * span) - 1;           // the group's last row that is there
              const int vis = last >= tok + g * span ? min(c, c - n + last + 1) : 0;
              tiles[g] = vis > 0 ? (vis + kPrTile - 1) / kPrTile : 0;
            }
            const int all = max(tiles[0], tiles[1]), seen = max(min(c, c - n + tok + 1), 0), part = seen / kPrTile;
            const int begin = (int)((long long)all * rank / shares), end = (int)((long long)all * (rank + 1) / shares);
            if (lane == 0) {
              it.live = live;
              it.s = s;
              it.tok = tok;
              it.head = head;
              it.q_head = hd * a.pack;
              it.n = n;
              it.c = c;
              it.q0 = prompt_begin(a.qs, s);
              it.k0 = prompt_begin(a.ks, s);
              it.room = room_of<kBf16>(all);
              it.seen = seen;
              it.part = part;
              it.clean = kSplit ? part : 0x7fffffff;
              it.begin = begin;
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                it.tiles[g] = tiles[g];
                it.end[g] = max(min(end, tiles[g]), begin);
              }
            }
          } else if (lane == 0) {
            it.clean = it.part;
          }
          if (lane == 0) {
            sh.again[iu & 1] = 0;
            bar_arrive(&sh.item_full[iu & 1]);
          }
          __syncwarp();
          if (!it.live) { ended = true; break; }
          const int end = max(it.end[0], it.end[1]);
          const int n_tiles = end - it.begin;
          if (n_tiles == 0) continue;
          const int qs = a.qs.first ? 0 : it.s, ks = a.ks.first ? 0 : it.s;
          for (int j = 0; j < 2 * n_tiles && ok; ++j, ++u) {               // K0 (then Q), V0, K1, V1, ..
            const uint32_t st = u % P::kStages, use = u / P::kStages;
            if (use > 0 && !warp_wait(&sh.free[st], (use - 1) & 1, waits, a.stats)) { ok = false; break; }
            if (leader) {
              bar_expect(&sh.full[st], P::kMat);
#pragma unroll
              for (int b = 0; b < P::kBlocks; ++b)
                map_load4(kv_smem(ring + st * P::kMat + b * (kPrTile * 128)), j & 1 ? &v_map : &k_map, b * 64, it.head,
                          it.k0 + (it.begin + (j >> 1)) * kPrTile, ks, &sh.full[st]);
            }
            __syncwarp();
            if (j == 0) {
              if (qu > 0 && !warp_wait(&sh.qfree, (qu - 1) & 1, waits, a.stats)) { ok = false; break; }
              ++qu;
              if (leader) {
                bar_expect(&sh.qfull, 2 * P::kMat);
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                  for (int b = 0; b < P::kBlocks; ++b)
                    map_load4(kv_smem(qmat + g * P::kMat + b * (kPrTile * 128)), &q_map, b * 64, it.q_head,
                              it.q0 + it.tok + g * span, qs, &sh.qfull);
              }
              __syncwarp();
            }
          }
        }
      } while (!over(iu++));
    } else if (warp == kPaIssuer) {
      // ========================================================== products =======
      const uint32_t s_idesc = idesc_16(kPrTile, false, kBf16) | (a.negate ? kNegateA : 0u);
      constexpr uint32_t o_idesc = idesc_16(D, true, kBf16);
      const uint64_t q_desc = desc128(kv_smem(qmat), 16), k_desc = desc128(kv_smem(ring), 16),
                     v_desc = desc128(kv_smem(ring), kPrTile * 128);
      constexpr uint64_t kStage = P::kMat >> 4;
      const bool leader = one_lane();
      uint32_t u = 0, qu = 0, cu = 0, pu[2] = {0, 0};
      bool ok = true;
      uint32_t iu = 0;
      do {
        for (; ok; ++iu) {
          if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, waits, a.stats)) break;
          const int live = sh.item[iu & 1].live, begin = sh.item[iu & 1].begin, tiles0 = sh.item[iu & 1].end[0] - begin,
                    tiles1 = sh.item[iu & 1].end[1] - begin, clean = min(sh.item[iu & 1].clean, sh.item[iu & 1].c / kPrTile) - begin;
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
          if (!live) break;
          const int n_tiles = max(tiles0, tiles1);
          if (n_tiles == 0) continue;
          auto landed = [&](uint32_t v) { ok = ok && warp_wait(&sh.full[v % P::kStages], (v / P::kStages) & 1, waits, a.stats); };
          auto scores = [&](int g, uint32_t kv) {          // of group g, keys in ring place kv
            const uint64_t kd = k_desc + (kv % P::kStages) * kStage;
            if (leader) {
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint64_t off = (uint64_t)((k >> 2) * (kPrTile * 128 >> 4) + (k & 3) * 2);
                mma_ss(tmem + g * 128, q_desc + g * kStage + off, kd + off, s_idesc, k > 0);
              }
              commit(&sh.sfull[g]);
            }
            __syncwarp();
          };
          landed(u);
          ok = ok && warp_wait(&sh.qfull, qu++ & 1, waits, a.stats);
          if (!ok) break;
          fence_after();
          if (tiles0 > 0) scores(0, u);
          if (tiles1 > 0) scores(1, u);
          if (leader) {
            commit(&sh.free[u % P::kStages]);
            if (n_tiles == 1) commit(&sh.qfree);
          }
          __syncwarp();
          for (int j = 0; j < n_tiles && ok; ++j) {
            const uint32_t vu = u + 2 * j + 1, ku = vu + 1;
            landed(vu);
            if (ok && j >= clean) {                        // (while the softmax warps are at work on the scores)
              if (lane == 0) {
                sh.asked = vu;
                bar_arrive(&sh.ask);
              }
              __syncwarp();
            }
            if (j + 1 < n_tiles) landed(ku);
            if (ok && j >= clean) ok = warp_wait(&sh.clean, cu++ & 1, waits, a.stats);
            if (!ok) break;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const int mine = g ? tiles1 : tiles0;
              if (j < mine) {
                const uint64_t vd = v_desc + (vu % P::kStages) * kStage;
#pragma unroll
                for (int h = 0; h < 2 && ok; ++h) {        // half of the keys at a time, as the probabilities come
                  if (!warp_wait(&sh.pfull[g][h], pu[g] & 1, waits, a.stats)) { ok = false; break; }
                  fence_after();
                  if (leader) {
#pragma unroll
                    for (int k = h * kPrTile / 32; k < (h + 1) * kPrTile / 32; ++k)
                      mma_ts(tmem + 256 + g * 128, tmem + g * 128 + k * 8, vd + (uint64_t)(k * 2048 >> 4), o_idesc, j > 0 || k > 0);
                    if (h == 1 && j + 1 == mine) commit(&sh.ofull[g]);
                  }
                  __syncwarp();
                }
                ++pu[g];
                if (!ok) break;
                if (j + 1 < mine) scores(g, ku);
              }
            }
            if (!ok) break;
            if (leader) {
              commit(&sh.free[vu % P::kStages]);
              if (j + 1 < n_tiles) commit(&sh.free[ku % P::kStages]);
              if (j + 2 == n_tiles) commit(&sh.qfree);
            }
            __syncwarp();
          }
          u += 2 * n_tiles;
        }
      } while (!over(iu++));
    } else {
      // ========================================================== values =========
      const int who = warp - kPaCleaner;
      uint32_t au = 0, cu = 0, places = 0;               // places: parities of the items cleaned in either so far
      bool ok = true;
      uint32_t iu = 0;
      do {
        for (; ok; ++iu) {
          if (!warp_wait(&sh.item_full[iu & 1], (iu >> 1) & 1, waits, a.stats)) break;
          const PaItem& now = sh.item[iu & 1];
          if (!now.live) break;
          const int c = now.c, end = max(now.end[0], now.end[1]);
          int from = 0x7fffffff, to = 0;
          for (int j = max(now.begin, min(now.clean, c / kPrTile)); j < end; ++j, ++au) {
            if (!warp_wait(&sh.ask, au & 1, waits, a.stats)) { ok = false; break; }
            const uint32_t vu = *const_cast<volatile uint32_t*>(&sh.asked);
            // (it has landed, and stays until these warps are through with it)
            if (!warp_wait(&sh.full[vu % P::kStages], (vu / P::kStages) & 1, waits, a.stats)) { ok = false; break; }
            uint4* tile = reinterpret_cast<uint4*>(ring + vu % P::kStages * P::kMat);
            // (a block of 64 channels: rows of 128 bytes, whatever their swizzle)
            const bool zero = j < now.clean;               // behind the last key; the other values as they are
            const int first = max((zero ? c : now.seen) - j * kPrTile, 0) * 8 + who * 32 + lane;
            for (int b = 0; b < P::kBlocks; ++b, tile += kPrTile * 8) {
              if (zero) {
                for (int i = first; i < kPrTile * 8; i += 32 * kPaCleaners) tile[i] = make_uint4(0u, 0u, 0u, 0u);
                continue;
              }
#pragma unroll 2
              for (int i = first; i < kPrTile * 8; i += 32 * kPaCleaners) {
                uint4 w = tile[i];
                const uint32_t x = odd_halves<kBf16>(w.x), y = odd_halves<kBf16>(w.y);
                const uint32_t z = odd_halves<kBf16>(w.z), q = odd_halves<kBf16>(w.w);
                if (x | y | z | q) {
                  w.x &= ~((x >> 15) * 0xffffu);
                  w.y &= ~((y >> 15) * 0xffffu);
                  w.z &= ~((z >> 15) * 0xffffu);
                  w.w &= ~((q >> 15) * 0xffffu);
                  tile[i] = w;
                  const int key = j * kPrTile + (i >> 3);
                  if (key < c) {
                    from = min(from, key);
                    to = max(to, key + 1);
                  }
                }
              }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.clean);
          }
          if (!ok) break;
          if (now.clean == now.part) {
            from = __reduce_min_sync(0xffffffffu, from);
            to = __reduce_max_sync(0xffffffffu, to);
            if (lane == 0) {
              sh.odd[who] = {from, to};
              bar_arrive(&sh.found);
            }
            if (!kSplit) {                                 // (a cluster's rows are joined with them)
              if (!warp_wait(&sh.found, cu++ & 1, waits, a.stats)) break;
              if (!warp_wait(&sh.written[iu & 1], places >> (iu & 1) & 1, waits, a.stats)) break;
              places ^= 1u << (iu & 1);
              from = min(sh.odd[0].from, sh.odd[1].from);
              to = max(sh.odd[0].to, sh.odd[1].to);
              if (from < to) odd_rows<D, kBf16>(a, now, sh.ml[iu & 1], who * 128, from, to, lane);
            }
          }
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.item_free[iu & 1]);
        }
      } while (!over(iu++));
    }
    // Nothing follows the roles: code that all warps share may use any register that the block was launched with, and
    // these warps have given most of theirs away.
    if (kSplit) {
      meet_cluster();
      meet_cluster();
      fence_before();
      __syncthreads();
    }
    if (warp == kPaIssuer) {
      fence_after();
      // The softmax warps waited for the last products, and the products for the last copies, unless
      // somebody gave up: then what is in flight gets time to end.  (Read behind the barrier, when nobody
      // can any more.)
      if (waits->gave_up) {
        const unsigned long long t0 = now_ns();
        while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
      }
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    return;
  }
}

// ------------------------------------------------------------------ host side ---
bool prompt_map(CUtensorMap* map, const KvRows& r, int head_dim, int heads, int rows, int n_seq, int box_heads, int box_rows, bool bf16) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult res;
    const bool there = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &res) == cudaSuccess &&
                       res == cudaDriverEntryPointSuccess;
    return there ? (Encode)p : (Encode)nullptr;
  }();
  if (!encode) return false;
  // (the stride of an extent of one is never used: any that the map takes)
  const cuuint64_t dims[4] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)rows, (cuuint64_t)n_seq};
  const cuuint64_t strides[3] = {(cuuint64_t)(heads > 1 ? r.head * 2 : 16), (cuuint64_t)(rows > 1 ? r.row * 2 : 16),
                                 (cuuint64_t)(n_seq > 1 ? r.seq * 2 : 16)};
  const cuuint32_t box[4] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows, 1}, step[4] = {1, 1, 1, 1};
  return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, (void*)r.p, dims, strides,
                box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How many clusters of 16 blocks run at once (0 until it has been asked for, when the kernels are loaded).
template <int D, bool kBf16>
static std::atomic<int>& most_clusters() {
  static std::atomic<int> n(0);
  return n;
}
template <int D, bool kBf16>
static cudaError_t run_attend(const PromptArgs& a, int sms, cudaStream_t st) {
  CUtensorMap qm, km, vm;
  const int nq = a.qs.first ? 1 : a.n_seq, nk = a.ks.first ? 1 : a.n_seq;
  // (without a key row nothing is loaded by the maps, but they have to be over something)
  const bool keys = a.ks.rows > 0;
  if (!prompt_map(&qm, a.q, D, a.n_kv * a.group, a.qs.rows, nq, a.pack, kPrTile / a.pack, kBf16) ||
      !prompt_map(&km, keys ? a.k : a.q, D, a.n_kv, keys ? a.ks.rows : 1, keys ? nk : 1, 1, kPrTile, kBf16) ||
      !prompt_map(&vm, keys ? a.v : a.q, D, a.n_kv, keys ? a.ks.rows : 1, keys ? nk : 1, 1, kPrTile, kBf16))
    return cudaErrorInvalidValue;
  // the most items there can be: a sequence's last one may be short
  const long long span = 2 * kPrTile / a.pack;
  const long long tiles = a.qs.first ? a.qs.rows / span + a.n_seq : (long long)a.n_seq * ((a.qs.rows + span - 1) / span);
  const long long items = tiles * a.n_kv * (a.group / a.pack);
  // Fewer items than SMs: the keys of each are shared by a cluster (of tiles, as far as there can be some), of 16
  // blocks where the device takes that many clusters of that size at once.
  int shares = 1;
  while (shares < 16 && items * shares * 2 <= sms && (long long)a.ks.rows > kPrTile * shares) shares *= 2;
  if (shares == 16 && items > most_clusters<D, kBf16>()) shares = 8;
  const unsigned grid = (unsigned)(items < sms ? items * shares : sms);
  return launch_cluster(shares > 1 ? prompt_attend_kernel<D, kBf16, true> : prompt_attend_kernel<D, kBf16, false>, grid, kPaThreads,
                        Pa<D>::kBytes, shares, st, qm, km, vm, a, shares);
}
cudaError_t launch_prompt_attend(const PromptArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st) {
  if (head_dim == 64) return bf16 ? run_attend<64, true>(a, sms, st) : run_attend<64, false>(a, sms, st);
  return bf16 ? run_attend<128, true>(a, sms, st) : run_attend<128, false>(a, sms, st);
}
template <int D, bool kBf16>
static cudaError_t preload_both() {
  auto split = prompt_attend_kernel<D, kBf16, true>;
  cudaError_t e = preload_kernel(prompt_attend_kernel<D, kBf16, false>, true);
  if (e == cudaSuccess) e = preload_kernel(split, true);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(split, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 16;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3(16);
  cfg.blockDim = dim3(kPaThreads);
  cfg.dynamicSmemBytes = Pa<D>::kBytes;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, split, &cfg) != cudaSuccess) { n = 0; (void)cudaGetLastError(); }
  most_clusters<D, kBf16>().store(n);
  return cudaSuccess;
}
cudaError_t preload_prompt_attend_kernels() {
  cudaError_t e;
  if ((e = preload_both<64, true>()) != cudaSuccess) return e;
  if ((e = preload_both<64, false>()) != cudaSuccess) return e;
  if ((e = preload_both<128, true>()) != cudaSuccess) return e;
  return preload_both<128, false>();
}

}  // namespace oilbird
