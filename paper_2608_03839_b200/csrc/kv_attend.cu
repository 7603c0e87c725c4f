// Attention over the 4-bit cache for few query rows per key/value head (single-token decode and
// small draft trees): one pass over the codes.
//
// For a row (node i, query head h) of a sequence and its key/value head:
//   s_j = c q.k_j over the cached slots and the new nodes the row sees,
//   out = sum_j exp(s_j - M) v_j / sum_j exp(s_j - M),   lse = M + log sum_j exp(s_j - M).
// A group's key is scale * code + lo, so  q.k = sum_groups scale (q.code) + lo (sum q):  the
// products run on the codes alone, as f16 numbers that are exact, and one fp32 multiply-add
// per (slot, row, group) brings in scale and offset; the scores carry no rounding but fp32's.
// For the values the scale joins the probability before it becomes an f16 operand (one
// rounding, at most 2^-11 of each term, in units that use f16's whole range: slots 17.5 nats below
// another one still bring in their values, not their groups' middles alone).  All codes are positive, so over a long sequence their
// sums would outgrow the result by far, and with them what the tensor cores cut off: half of the
// slots therefore go in with 15 - code and a negative operand, and the groups' middles
// (lo + 7.5 scale, in fp32) in place of the offsets make up the difference, with 7.5 times the
// operands' own sums.  On 131,085 slots that took the error from 8e-4 of the result to 2.8e-4
// (the result's own rounding to f16: 2.1e-4) for 3 to 5 % of the time.
//
// Layout.  The products are taken transposed, S^T = K Q^T with 16 slots x 8 rows and
// O^T = V^T P^T with 16 channels x 8 rows, so that 8 rows (the query heads of one key head)
// fill a matrix instruction; P^T goes from accumulator to operand layout by an 8 x 8
// transpose.  Rows of a 16-slot chunk are dealt out so that logical row 2t is slot t and
// 2t+1 is slot t+4: then both the K loads (8 bytes a lane) and the V loads (4 bytes a lane)
// take 256 and 128 contiguous bytes of shared memory.
//
// Work.  The tiles (64 slots) of all (sequence, head) items are one list, cut into equal runs, one
// per block, two blocks an SM; a block's warps take the run's tiles in turn, each through a
// buffer of its own (asynchronous 16-byte copies, no block-wide waits), which runs on across
// items.  At the end of an item's share the warps' results are joined in shared memory; items cut
// between blocks go through the workspace, and the block that finishes last joins the pieces, in
// their order, whichever block that is.
//
// Measured, with 8 key/value heads of 128: 64 sequences of 4,096 to 8,192 slots, 444 MB of cache
// under 32 query heads, in 107 us (4.2 TB/s; 68 us at the copy rate); 131,085 slots under 64
// query heads in 44 us (23 us at the copy rate); 517 slots in 10 us.  The long ones fill half the
// issue slots (taking codes apart, 32 lanes' worth of exponentials and scales for each slot and
// row) with twelve warps an SM that wait for their own results in between, unevenly between the two
// blocks of an SM; the short one is bound by the latency of one tile, one join and one launch.
#include "kv.cuh"

namespace oilbird {

// A block takes all rows of a key head, 8 NT at most (16, so 16 new nodes at most).  A warp holds its tile's keys and values in buffers of their own: the
// next tile's keys are asked for as soon as the scores are taken, its values after the products
// with them, so that a single buffer of each keeps half a tile per warp in flight.
// Eight rows leave registers (168 a thread) for twelve warps an SM, sixteen rows for eight.
//
// More rows go to kv_tree.cu, whose tensor core products cost the same for 17 rows as for 128.
// With 16 rows or fewer one reading of the cache is enough here.  Measured beyond that, there
// against as many calls of 16 rows here as it takes, 8 heads of 128 channels, f16 (bf16 within 2 %):
//   slots          17..32 rows          33..48 rows          49..64 rows
//   8 x 4,096      66 us against 58     66 against 87        67 against 116
//   65,536         87 against 86        87 against 129       87 against 172
//   32 x 8,192     366 against 209      367 against 313      367 against 417
// and 21 rows of 64 channels over 777 slots 17.2 us against 18.6.  So up to 32 rows over long
// sequences, where the GPU is full, two readings here would be faster; the change stands at 16.
constexpr int kFewRows = 16;
// Probability times value scale is an f16 operand, in units in which the largest scale lies below
// 2^7: with probabilities up to 2^8 f16 just holds it, and small probabilities keep their bits.
constexpr int kRoom = 7;
template <int D, int NT>
struct Attend {
  static constexpr int kWarps = NT == 1 ? 6 : 4, kThreads = 32 * kWarps, kCtas = 2;
  static constexpr int kPart = kKvTile * (D / kKvGroup) * 36;        // codes, meta of K or of V
  static constexpr int kRing = kWarps * 2 * kPart;
  static constexpr int kObuf = kWarps * 8 * (D + 4) * 4;
  static constexpr int kMl = kWarps * 8 * 8;
  static constexpr int kCum = (kKvMaxSeq + 1) * 8;
  static constexpr int kBytes = kRing + kObuf + kMl + kCum + kWarps * 8 + kKvMaxSeq * 5 + 64;
};
struct OpenItem { int b0, b1, s, head, n_rows; };  // an item whose pieces are all there

template <int N> __device__ __forceinline__ void load_floats(const float* p, float (&v)[N]) {
  if (N == 4) { const float4 x = *reinterpret_cast<const float4*>(p); v[0] = x.x; v[1] = x.y; v[N - 2] = x.z; v[N - 1] = x.w; }
  else { const float2 x = *reinterpret_cast<const float2*>(p); v[0] = x.x; v[1] = x.y; }
}
template <int N> __device__ __forceinline__ void load_floats_cg(const float* p, float (&v)[N]) {
  if (N == 4) { const float4 x = __ldcg(reinterpret_cast<const float4*>(p)); v[0] = x.x; v[1] = x.y; v[N - 2] = x.z; v[N - 1] = x.w; }
  else { const float2 x = __ldcg(reinterpret_cast<const float2*>(p)); v[0] = x.x; v[1] = x.y; }
}
template <int N> __device__ __forceinline__ void store_floats(float* p, const float (&v)[N]) {
  if (N == 4) __stcg(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[N - 2], v[N - 1]));
  else __stcg(reinterpret_cast<float2*>(p), make_float2(v[0], v[1]));
}

template <int D, int NT, bool kBf16>
__global__ void __launch_bounds__(Attend<D, NT>::kThreads, Attend<D, NT>::kCtas)
kv_attend_kernel(const KvView c, const KvAttendArgs a) {
  using Sh = Attend<D, NT>;
  constexpr int kAtThreads = Sh::kThreads, kAtWarps = Sh::kWarps;
  constexpr int G = D / kKvGroup, kRows = NT * 8, kSteps = D / 16;
  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* ring = smem;
  float* obuf = reinterpret_cast<float*>(smem + Sh::kRing);
  float2* ml = reinterpret_cast<float2*>(smem + Sh::kRing + Sh::kObuf);
  long long* cum = reinterpret_cast<long long*>(smem + Sh::kRing + Sh::kObuf + Sh::kMl);
  long long* scratch = cum + kKvMaxSeq + 1;
  int* len_s = reinterpret_cast<int*>(scratch + kAtWarps);
  unsigned char* nodes_s = reinterpret_cast<unsigned char*>(len_s + kKvMaxSeq);
  int* n_open = reinterpret_cast<int*>(nodes_s + kKvMaxSeq);
  OpenItem* open = reinterpret_cast<OpenItem*>(n_open + 1);

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  if (tid == 0) *n_open = 0;                             // (barriers follow)
  pdl_enter();

  TileList list;
  list.cum = cum;
  list.len = len_s;
  list.nodes = nodes_s;
  list.items = c.n_kv;
  list.group = a.group;
  list.rows = kRows;
  list.build<kAtThreads>(c, a.n_new, a.m, scratch);
  const long long total = list.total;
  // blocks share the list evenly; no block gets less than a tile for each of its warps
  const int n_cta = (int)min((long long)gridDim.x, (total + kAtWarps - 1) / kAtWarps);
  if (blockIdx.x >= n_cta) return;
  TileCursor bc, pc;                                     // the block's item; the warp's next tile to copy
  const long long u1_all = list.cut(pc, blockIdx.x + 1, n_cta), u0 = list.cut(bc, blockIdx.x, n_cta);
  const int u1 = (int)(u1_all - u0);                     // positions from here on count from u0
  if (u1 <= 0) return;

  // ---- the warp's ring of tiles ----
  unsigned char* st = ring + warp * (2 * Sh::kPart);
  int pu = warp, ahead = -1;                             // the next tile to copy; its pages
  unsigned long long valid_next = 0;
  pc = bc;
  if (pu < u1) { list.advance(pc, warp); ahead = tile_pages(c, pc, lane); }
  auto issue_keys = [&]() {
    if (pu < u1 && pc.cached()) {
      copy_tile<D, 0>(c, pc, ahead, st, lane);
      valid_next = tile_valid(pc, ahead);
    }
    cp_async_commit();
  };
  auto issue_values = [&]() {                            // and on to the next tile
    if (pu < u1) {
      if (pc.cached()) copy_tile<D, 1>(c, pc, ahead, st + Sh::kPart, lane);
      pu += kAtWarps;
      if (pu < u1) { list.advance(pc, kAtWarps); ahead = tile_pages(c, pc, lane); }
    }
    cp_async_commit();
  };
  issue_keys();
  issue_values();

  constexpr int kOs = D + 4, kPer = D / 32;              // floats a lane handles of a row in a join
  constexpr size_t kPartFloats = (size_t)kRows * (D + 2);
  float* parts = reinterpret_cast<float*>(c.work + kKvPartOff);
  // row `row` of (s, head) is complete: v relative to 2^big, with the sum of its weights
  auto finish = [&](int s, int head, int row, int n_rows, float big, float sum, const float (&v)[kPer]) {
    if (row >= a.m * a.group) return;
    const int node = row / a.group, hq = head * a.group + row % a.group;
    if (row >= n_rows) sum = 0.f;                        // behind the sequence's nodes
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t* op = a.out + s * a.out_seq + node * a.out_row + hq * a.out_head + lane * kPer;
    uint32_t w[kPer / 2];
#pragma unroll
    for (int e = 0; e < kPer / 2; ++e) w[e] = sum == 0.f ? 0u : pack16<kBf16>(v[2 * e] * inv, v[2 * e + 1] * inv);
    if (kPer == 4) *reinterpret_cast<uint2*>(op) = make_uint2(w[0], w[kPer / 2 - 1]);
    else *reinterpret_cast<uint32_t*>(op) = w[0];
    if (a.lse && lane == 0)
      a.lse[s * a.lse_seq + node * a.lse_row + hq * a.lse_head] =
          sum == 0.f ? -INFINITY : (big + log2f(sum)) * 0.6931471805599453f;
  };

  // ---- item by item ----
  int mu = warp;                                         // the warp's next tile to compute
  for (int at = 0; at < u1;) {
    const int item = bc.item, tile0 = bc.tile;
    const int n_tiles = item < bc.live ? bc.tiles : 1;
    const int piece = min(n_tiles - tile0, u1 - at), item_u0 = at - tile0;
    const int head = bc.head;
    const int n_rows = bc.nodes * a.group;               // rows of the sequence that exist
    const int s = bc.s;

    float o[NT][4 * G][4];                               // channel tiles x rows, in units of 2^(eref + 24)
    float olo[NT][G][2], l[NT][2], m[NT][2];
    int eref = -120;
    bool fresh = true, had = false;                      // eref is free to fall; the warp took a tile
#pragma unroll
    for (int r = 0; r < NT; ++r) {
#pragma unroll
      for (int i = 0; i < 4 * G; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[r][i][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[r][e] = 0.f;
        m[r][e] = -INFINITY;
#pragma unroll
        for (int i = 0; i < G; ++i) olo[r][i][e] = 0.f;
      }
    }

    if (item < bc.live && mu < at + piece && mu == item_u0) {
      // ---- the item's first tile: new nodes, 16-bit keys and values, with the tree's mask ----
      if (a.k.p) {
        had = true;
        float sc[NT][4];
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[r][e] = 0.f;
        uint4 qw[NT][G][2], kw[2][G][2];
#pragma unroll
        for (int r = 0; r < NT; ++r) {
          const int row = r * 8 + g;
          const int node = row < n_rows ? row / a.group : 0, sub = row < n_rows ? row % a.group : 0;
          const uint16_t* qp = a.q.at(s, node, head * a.group + sub) + t4 * 16;
#pragma unroll
          for (int i = 0; i < G; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              qw[r][i][half] = make_uint4(0, 0, 0, 0);
              if (row < n_rows) qw[r][i][half] = *reinterpret_cast<const uint4*>(qp + i * kKvGroup + half * 8);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int node = g + 8 * k;
          const uint16_t* kp = a.k.at(s, node < bc.nodes ? node : 0, head) + t4 * 16;
#pragma unroll
          for (int i = 0; i < G; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              kw[k][i][half] = make_uint4(0, 0, 0, 0);
              if (node < bc.nodes) kw[k][i][half] = *reinterpret_cast<const uint4*>(kp + i * kKvGroup + half * 8);
            }
        }
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < NT; ++r) {
              const uint4 &x = kw[0][i][half], &y = kw[1][i][half], &z = qw[r][i][half];
              mma16816<kBf16>(sc[r], x.x, y.x, x.y, y.y, z.x, z.y);
              mma16816<kBf16>(sc[r], x.z, y.z, x.w, y.w, z.z, z.w);
            }
        const float fs = a.scale * kLog2e;
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int row = r * 8 + 2 * t4 + e;
            unsigned long long sees = 0;
            if (row < n_rows) {
              const int node = row / a.group;
              sees = a.mask ? a.mask[s * a.mask_stride + node] : (2ull << node) - 1ull;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int node = g + 8 * k;
              const bool ok = node < bc.nodes && (sees >> node & 1ull);
              float& x = sc[r][e + 2 * k];
              x = ok ? x * fs : -INFINITY;
              mx = fmaxf(mx, x);
            }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
            m[r][e] = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          }
        // these products need no units: eref = 0 after them, where no finite value overflows;
        // the first cached tile chooses anew
        eref = 0;
        bool odd = false;
        // p as the sum of two 16-bit numbers: with bf16 one alone would be as coarse as the
        // result's own rounding
        uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float p[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              p[e] = exp2_approx(sc[r][e + 2 * k] - (m[r][e] == -INFINITY ? 0.f : m[r][e]));
              l[r][e] += p[e];
            }
            const uint32_t h = pack16<kBf16>(p[0], p[1]);
            hi[r][k] = transpose8x8(h);
            lo[r][k] = transpose8x8(pack16<kBf16>(p[0] - half_lo<kBf16>(h), p[1] - half_hi<kBf16>(h)));
          }
        uint4 w[G][4];                                   // nodes 2t, 2t+1, 2t+8, 2t+9; 8 channels
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int node = 2 * t4 + (k & 1) + 8 * (k >> 1);
          const uint16_t* vp = a.v.at(s, node < bc.nodes ? node : 0, head) + g * 8;
#pragma unroll
          for (int i = 0; i < G; ++i) {
            w[i][k] = make_uint4(0, 0, 0, 0);
            if (node < bc.nodes) w[i][k] = *reinterpret_cast<const uint4*>(vp + i * kKvGroup);
#pragma unroll
            for (int x = 0; x < 4; ++x) {                // infinities and NaN: see below
              uint32_t& v = (&w[i][k].x)[x];
              constexpr uint32_t kInf = kBf16 ? 0x7f80u : 0x7c00u;
              if ((v & kInf) == kInf) { odd = true; v &= 0xffff0000u; }
              if ((v >> 16 & kInf) == kInf) { odd = true; v &= 0x0000ffffu; }
            }
          }
        }
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const uint32_t x0 = (&w[i][0].x)[n], x1 = (&w[i][1].x)[n], x2 = (&w[i][2].x)[n], x3 = (&w[i][3].x)[n];
            const uint32_t ea = __byte_perm(x0, x1, 0x5410), oa = __byte_perm(x0, x1, 0x7632);
            const uint32_t eb = __byte_perm(x2, x3, 0x5410), ob = __byte_perm(x2, x3, 0x7632);
#pragma unroll
            for (int r = 0; r < NT; ++r) {
              mma16816<kBf16>(o[r][i * 4 + n], ea, oa, eb, ob, hi[r][0], hi[r][1]);
              mma16816<kBf16>(o[r][i * 4 + n], ea, oa, eb, ob, lo[r][0], lo[r][1]);
            }
          }
        if (__any_sync(0xffffffffu, odd)) {
          // values that are not finite stayed out of the products (0 times a hidden node's
          // would have reached every row): they are added to the rows that see them
#pragma unroll
          for (int r = 0; r < NT; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int row = r * 8 + 2 * t4 + e;
              if (row >= n_rows) continue;
              const int node = row / a.group;
              const unsigned long long sees = a.mask ? a.mask[s * a.mask_stride + node] : (2ull << node) - 1ull;
              for (int j = 0; j < bc.nodes; ++j)
                if (sees >> j & 1ull) {
                  const uint16_t* vp = a.v.at(s, j, head) + g * 8;
#pragma unroll
                  for (int i = 0; i < G; ++i)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                      const uint32_t w = *reinterpret_cast<const uint32_t*>(vp + i * kKvGroup + 2 * n);
                      const float v0 = half_lo<kBf16>(w), v1 = half_hi<kBf16>(w);
                      if (!(fabsf(v0) < INFINITY)) o[r][i * 4 + n][e] += v0;
                      if (!(fabsf(v1) < INFINITY)) o[r][i * 4 + n][e + 2] += v1;
                    }
                }
            }
        }
        // (the cached codes of odd pairs carry 16 times their value)
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int i = 0; i < 4 * G; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][i][e] *= i & 1 ? 0x1p-20f : 0x1p-24f;
      }
    }

    // ---- cached tiles ----
    uint32_t qf[NT][kSteps][2];
    float f[NT][2], qsum[NT][G][2];
    bool loaded = false;
    for (; mu < at + piece; mu += kAtWarps) {
      const int tile = mu - item_u0;
      if (item < bc.live && tile >= kKvFront) {
        if (!loaded) {                                   // query rows as operands
          loaded = had = true;
#pragma unroll
          for (int r = 0; r < NT; ++r) {
            const int row = r * 8 + g;
            const bool have = row < n_rows;
            const int node = have ? row / a.group : 0;
            float sum[G];
            const int e0 = row_operands<D, kBf16>(a.q.at(s, node, head * a.group + (have ? row % a.group : 0)), have, t4,
                                                  a.scale < 0.f, qf[r], sum);
#pragma unroll
            for (int i = 0; i < G; ++i) {                // accumulators hold rows 2t and 2t+1
              qsum[r][i][0] = __shfl_sync(0xffffffffu, sum[i], 8 * t4) * 0x1p-24f;
              qsum[r][i][1] = __shfl_sync(0xffffffffu, sum[i], 8 * t4 + 4) * 0x1p-24f;
            }
            const float ff = row_factor(a.scale, e0);
            f[r][0] = __shfl_sync(0xffffffffu, ff, 8 * t4);
            f[r][1] = __shfl_sync(0xffffffffu, ff, 8 * t4 + 4);
          }
        }
        cp_async_wait<1>();
        __syncwarp();
        unsigned char* kmeta = st + G * kKvTile * 32;
        const unsigned long long valid = valid_next;
        const bool partial = valid != ~0ull;             // the sequence's end, or a page that is none
        if (partial) {
          clear_meta<G>(kmeta, valid, lane);
          __syncwarp();
        }
        const int slot_g = (g >> 1) + 4 * (g & 1);       // logical row g of a chunk
        // ---- scores ----
        float sc[NT][4][4];
#pragma unroll
        for (int c0 = 0; c0 < 4; c0 += 4) {       // independent sums side by side
          uint2 w[4][2][G];
          float acc[4][G][NT][4];
#pragma unroll
          for (int ch = 0; ch < 4; ++ch)
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const int sl = (c0 + ch) * 16 + slot_g;
              w[ch][0][i] = *reinterpret_cast<const uint2*>(st + (i * kKvTile + sl) * 32 + t4 * 8);
              w[ch][1][i] = *reinterpret_cast<const uint2*>(st + (i * kKvTile + sl + 8) * 32 + t4 * 8);
#pragma unroll
              for (int r = 0; r < NT; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[ch][i][r][e] = 0.f;
            }
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int ch = 0; ch < 4; ++ch)
#pragma unroll
              for (int i = 0; i < G; ++i) {
                const uint32_t x0 = (j & 2 ? w[ch][0][i].y : w[ch][0][i].x) >> (8 * (j & 1));
                const uint32_t x1 = (j & 2 ? w[ch][1][i].y : w[ch][1][i].x) >> (8 * (j & 1));
#pragma unroll
                for (int r = 0; r < NT; ++r)
                  mma16816<false>(acc[ch][i][r], x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u,
                                  x1 & 0x00f000f0u, qf[r][i * 4 + j][0], qf[r][i * 4 + j][1]);
              }
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            const int sl = (c0 + ch) * 16 + slot_g;
            uint32_t km[2][G];
            load_meta<G>(kmeta + sl * 4 * G, km[0]);
            load_meta<G>(kmeta + (sl + 8) * 4 * G, km[1]);
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const float s0 = half_lo<kBf16>(km[0][i]), l0 = half_hi<kBf16>(km[0][i]);
              const float s1 = half_lo<kBf16>(km[1][i]), l1 = half_hi<kBf16>(km[1][i]);
#pragma unroll
              for (int r = 0; r < NT; ++r) {
                float (&x)[4] = sc[r][c0 + ch];
                const float (&y)[4] = acc[ch][i][r];
                x[0] = fmaf(s0, y[0], i ? fmaf(l0, qsum[r][i][0], x[0]) : l0 * qsum[r][i][0]);
                x[1] = fmaf(s0, y[1], i ? fmaf(l0, qsum[r][i][1], x[1]) : l0 * qsum[r][i][1]);
                x[2] = fmaf(s1, y[2], i ? fmaf(l1, qsum[r][i][0], x[2]) : l1 * qsum[r][i][0]);
                x[3] = fmaf(s1, y[3], i ? fmaf(l1, qsum[r][i][1], x[3]) : l1 * qsum[r][i][1]);
              }
            }
          }
        }
        if (partial) {
#pragma unroll
          for (int ch = 0; ch < 4; ++ch)
#pragma unroll
            for (int k = 0; k < 2; ++k)
              if (!(valid >> (ch * 16 + slot_g + 8 * k) & 1)) {
#pragma unroll
                for (int r = 0; r < NT; ++r) sc[r][ch][2 * k] = sc[r][ch][2 * k + 1] = -INFINITY;
              }
        }
        __syncwarp();
        issue_keys();
        // ---- running maximum; the value scales' power of two ----
        const unsigned char* vst = st + Sh::kPart;
        unsigned char* vmeta = st + Sh::kPart + G * kKvTile * 32;
        cp_async_wait<1>();
        __syncwarp();
        if (partial) {
          clear_meta<G>(vmeta, valid, lane);
          __syncwarp();
        }
        constexpr uint32_t kInf = kBf16 ? 0x7f80u : 0x7c00u;
        uint32_t vtop;
        {
          const uint2 x = *reinterpret_cast<const uint2*>(vmeta + lane * 8);
          vtop = __vmaxu2(x.x, x.y);
          uint2 y = make_uint2(0, 0);
          if (G == 2) {
            y = *reinterpret_cast<const uint2*>(vmeta + 256 + lane * 8);
            vtop = __vmaxu2(vtop, __vmaxu2(y.x, y.y));
          }
          vtop = __reduce_max_sync(0xffffffffu, vtop & 0xffffu);
          if (vtop >= kInf) {                            // a group that reads as NaN says nothing
            vtop = 0;
            for (const uint32_t w : {x.x, x.y, y.x, y.y}) vtop = max(vtop, (w & 0xffffu) < kInf ? w & 0xffffu : 0u);
            vtop = __reduce_max_sync(0xffffffffu, vtop);
          }
        }
        const int etile = kBf16 ? max((int)(vtop >> 7) - 126 - kRoom, -120) : (int)(vtop >> 10) - 14 - kRoom;
        float mx[NT][2];
        bool grow = etile > eref || fresh;
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = fmaxf(sc[r][0][e], sc[r][0][e + 2]);
#pragma unroll
            for (int ch = 1; ch < 4; ++ch) x = fmaxf(x, fmaxf(sc[r][ch][e], sc[r][ch][e + 2]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            mx[r][e] = x * f[r][e];
            // p may grow to 2^8 before the accumulators are brought to a new maximum
            grow |= mx[r][e] > m[r][e] + 8.f;
          }
        if (__any_sync(0xffffffffu, grow)) {
          // (behind new nodes, which leave eref at 0, it falls no further than their sums allow)
          const int enew = fresh ? (eref == 0 ? max(etile, -60) : etile) : max(eref, etile);
          const float ve = pow2(min(max(eref - enew, -126), 126));
          eref = enew;
          fresh = false;
#pragma unroll
          for (int r = 0; r < NT; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // (each row for itself: what its warp's other rows look at changes nothing)
              const float mn = mx[r][e] > m[r][e] + 8.f ? mx[r][e] : m[r][e];
              const float down = mn == -INFINITY ? 1.f : exp2_approx(m[r][e] - mn);
              m[r][e] = mn;
              l[r][e] *= down;
#pragma unroll
              for (int i = 0; i < G; ++i) olo[r][i][e] *= down;
#pragma unroll
              for (int i = 0; i < 4 * G; ++i) { o[r][i][e] *= down * ve; o[r][i][e + 2] *= down * ve; }
            }
        }
        const float up = pow2(eref), vdown = g & 1 ? -pow2(-eref) : pow2(-eref);
        float neg[NT][2];
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) neg[r][e] = m[r][e] == -INFINITY ? 0.f : -m[r][e];
        // ---- probabilities, and the products with the values ----
        float side[NT][G][4];                            // 15/16 of the operands' sums
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int i = 0; i < G; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) side[r][i][e] = 0.f;
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          const int sl = ch * 16 + slot_g;
          uint32_t vm[2][G], pb[NT][G][2];
          load_meta<G>(vmeta + sl * 4 * G, vm[0]);
          load_meta<G>(vmeta + (sl + 8) * 4 * G, vm[1]);
          float v0[G], l0[G], v1[G], l1[G];              // scales, the groups' middles
#pragma unroll
          for (int i = 0; i < G; ++i) {
            v0[i] = half_lo<kBf16>(vm[0][i]);
            v1[i] = half_lo<kBf16>(vm[1][i]);
            l0[i] = fmaf(7.5f, v0[i], half_hi<kBf16>(vm[0][i]));
            l1[i] = fmaf(7.5f, v1[i], half_hi<kBf16>(vm[1][i]));
            v0[i] *= vdown;
            v1[i] *= vdown;
          }
#pragma unroll
          for (int r = 0; r < NT; ++r) {
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = exp2_approx(fmaf(sc[r][ch][e], f[r][e & 1], neg[r][e & 1]));
            l[r][0] += p[0] + p[2];
            l[r][1] += p[1] + p[3];
#pragma unroll
            for (int i = 0; i < G; ++i) {
              olo[r][i][0] = fmaf(p[0], l0[i], fmaf(p[2], l1[i], olo[r][i][0]));
              olo[r][i][1] = fmaf(p[1], l0[i], fmaf(p[3], l1[i], olo[r][i][1]));
              pb[r][i][0] = transpose8x8(pack16<false>(p[0] * v0[i], p[1] * v0[i]));
              pb[r][i][1] = transpose8x8(pack16<false>(p[2] * v1[i], p[3] * v1[i]));
              mma16816<false>(side[r][i], 0x3b803b80u, 0x3b803b80u, 0x3b803b80u, 0x3b803b80u, pb[r][i][0], pb[r][i][1]);
            }
          }
          // operand column 2t is slot t, 2t+1 slot t+4 (and +8): as the scores' rows
#pragma unroll
          for (int i = 0; i < G; ++i) {
            const unsigned char* vp = vst + (i * kKvTile + ch * 16 + t4) * 32 + g * 4;
            const uint32_t w0 = *reinterpret_cast<const uint32_t*>(vp);
            const uint32_t w1 = ~*reinterpret_cast<const uint32_t*>(vp + 4 * 32);
            const uint32_t w2 = *reinterpret_cast<const uint32_t*>(vp + 8 * 32);
            const uint32_t w3 = ~*reinterpret_cast<const uint32_t*>(vp + 12 * 32);
            // even channels of both slots, odd channels of both slots
            const uint32_t ea = __byte_perm(w0, w1, 0x5410), oa = __byte_perm(w0, w1, 0x7632);
            const uint32_t eb = __byte_perm(w2, w3, 0x5410), ob = __byte_perm(w2, w3, 0x7632);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              const uint32_t mask = n & 1 ? 0x00f000f0u : 0x000f000fu;
              const int sh = n & 2 ? 8 : 0;
#pragma unroll
              for (int r = 0; r < NT; ++r)
                mma16816<false>(o[r][i * 4 + n], (ea >> sh) & mask, (oa >> sh) & mask, (eb >> sh) & mask,
                                (ob >> sh) & mask, pb[r][i][0], pb[r][i][1]);
            }
          }
        }
        // (in all eight lanes of a row, which are added up at the end: 7.5 times)
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int i = 0; i < G; ++i) {
            olo[r][i][0] = fmaf(-up, side[r][i][0], olo[r][i][0]);
            olo[r][i][1] = fmaf(-up, side[r][i][1], olo[r][i][1]);
          }
      } else {
        cp_async_wait<1>();              // an empty tile: nothing was copied
        __syncwarp();
        issue_keys();
      }
      __syncwarp();
      issue_values();
    }

    // ---- the warps' results joined; the item's share written ----
    int b0, b1;
    list.owners(u0 + item_u0, n_tiles, n_cta, b0, b1);
    const bool whole = b0 == b1;
    float* my_part = parts + (size_t)(2 * blockIdx.x + (blockIdx.x == b0 ? 1 : 0)) * kPartFloats;
    const float unit = pow2(eref);

#pragma unroll
    for (int r = 0; r < NT; ++r) {
      if (r) __syncthreads();
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) {
          l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], x);
#pragma unroll
          for (int i = 0; i < G; ++i) olo[r][i][e] += __shfl_xor_sync(0xffffffffu, olo[r][i][e], x);
        }
        float* dst = obuf + (warp * 8 + 2 * t4 + e) * kOs + g * 8;
        if (had)
#pragma unroll
        for (int i = 0; i < G; ++i) {
          // channels 8g + 2n (accumulator e) and 8g + 2n + 1 (e + 2); odd n carry 16 times
          float v[8];
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const float u = n & 1 ? 0x1p20f : 0x1p24f;   // (with the unit it could pass fp32's range)
            v[2 * n] = fmaf(o[r][i * 4 + n][e] * u, unit, olo[r][i][e]);
            v[2 * n + 1] = fmaf(o[r][i * 4 + n][e + 2] * u, unit, olo[r][i][e]);
          }
          *reinterpret_cast<float4*>(dst + i * kKvGroup) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4*>(dst + i * kKvGroup + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
        if (g == 0) ml[warp * 8 + 2 * t4 + e] = make_float2(m[r][e], l[r][e]);
      }
      __syncthreads();
      for (int rr = warp; rr < 8; rr += kAtWarps) {
        float2 x[kAtWarps];
        float big = -INFINITY, sum = 0.f, v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kAtWarps; ++w) { x[w] = ml[w * 8 + rr]; big = fmaxf(big, x[w].x); }
#pragma unroll
        for (int w = 0; w < kAtWarps; ++w) {
          const float k = x[w].x == -INFINITY ? (x[w].y == 0.f ? 0.f : 1.f) : exp2_approx(x[w].x - big);
          sum = fmaf(k, x[w].y, sum);
          if (k != 0.f) {                                // (a warp without tiles left nothing)
            float y[kPer];
            load_floats<kPer>(obuf + (w * 8 + rr) * kOs + lane * kPer, y);
#pragma unroll
            for (int e = 0; e < kPer; ++e) v[e] = fmaf(k, y[e], v[e]);
          }
        }
        if (whole) {
          finish(s, head, r * 8 + rr, n_rows, big, sum, v);
        } else {
          store_floats<kPer>(my_part + (size_t)(r * 8 + rr) * D + lane * kPer, v);
          if (lane == 0)
            __stcg(reinterpret_cast<float2*>(my_part + (size_t)kRows * D) + r * 8 + rr, make_float2(big, sum));
        }
      }
    }
    __syncthreads();
    if (!whole && tid == 0) {                            // the block that brings the last piece joins them
      unsigned* ticket = reinterpret_cast<unsigned*>(c.work + kKvTicketOff) + b0;
      __threadfence();                                   // (after the barrier: for all that the block wrote)
      const unsigned n = atomicAdd(ticket, 1u);
      __threadfence();
      if (n == (unsigned)(b1 - b0)) {
        *ticket = 0u;                                    // for the next call
        open[*n_open] = OpenItem{b0, b1, s, head, n_rows};
        ++*n_open;                                       // its first and its last item, at most
      }
    }
    at += piece;
    if (at < u1) list.advance(bc, piece);
  }

  // ---- items whose last piece came from here: the pieces joined, in their order ----
  __syncthreads();
  for (int q = 0; q < *n_open; ++q) {
    const OpenItem it = open[q];
    auto part_of = [&](int b) { return parts + (size_t)(2 * b + (b == it.b0 ? 1 : 0)) * kPartFloats; };
    for (int r = warp; r < kRows; r += kAtWarps) {
      float big = -INFINITY, sum = 0.f, v[kPer];
#pragma unroll
      for (int e = 0; e < kPer; ++e) v[e] = 0.f;
      constexpr int kBatch = 20;                         // pieces asked for at once
      for (int p0 = it.b0; p0 <= it.b1; p0 += kBatch) {
        const int n = min(kBatch, it.b1 - p0 + 1);
        float2 x = make_float2(-INFINITY, 0.f);
        if (lane < n) x = __ldcg(reinterpret_cast<const float2*>(part_of(p0 + lane) + (size_t)kRows * D) + r);
        float y[kBatch][kPer];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (i < n) load_floats_cg<kPer>(part_of(p0 + i) + (size_t)r * D + lane * kPer, y[i]);
        float top = x.x;
#pragma unroll
        for (int sft = 16; sft; sft >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, sft));
        const float nb = fmaxf(big, top);
        const float down = big == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : exp2_approx(big - nb);
        sum *= down;
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] *= down;
        big = nb;
        const float k = x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : exp2_approx(x.x - nb);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const float ki = __shfl_sync(0xffffffffu, k, i), li = __shfl_sync(0xffffffffu, x.y, i);
          if (i < n) {
            sum = fmaf(ki, li, sum);
#pragma unroll
            for (int e = 0; e < kPer; ++e) v[e] = ki != 0.f ? fmaf(ki, y[i][e], v[e]) : v[e];
          }
        }
      }
      finish(it.s, it.head, r, it.n_rows, big, sum, v);
    }
  }
}

template <int D, int NT, bool kBf16>
static cudaError_t attend_launch(const KvView& c, const KvAttendArgs& a, int sms, cudaStream_t st) {
  return launch_pdl(kv_attend_kernel<D, NT, kBf16>, dim3(Attend<D, NT>::kCtas * sms), dim3(Attend<D, NT>::kThreads), Attend<D, NT>::kBytes,
                    st, c, a);
}
template <int D, bool kBf16>
static cudaError_t attend_rows(const KvView& c, const KvAttendArgs& a, int sms, cudaStream_t st) {
  if (a.m * a.group <= 8) return attend_launch<D, 1, kBf16>(c, a, sms, st);
  if (a.m * a.group <= kFewRows) return attend_launch<D, 2, kBf16>(c, a, sms, st);
  return launch_kv_tree(c, a, D, kBf16, sms, st);
}

cudaError_t launch_kv_attend(const KvView& c, const KvAttendArgs& a, int head_dim, bool bf16, int sms,
                             cudaStream_t st) {
  if (2 * sms > kKvMaxCtas) sms = kKvMaxCtas / 2;
  if (head_dim == 64) return bf16 ? attend_rows<64, true>(c, a, sms, st) : attend_rows<64, false>(c, a, sms, st);
  return bf16 ? attend_rows<128, true>(c, a, sms, st) : attend_rows<128, false>(c, a, sms, st);
}

template <int D, bool kBf16>
static cudaError_t preload_rows() {
  const cudaError_t e = preload_kernel(kv_attend_kernel<D, 1, kBf16>, true);
  return e != cudaSuccess ? e : preload_kernel(kv_attend_kernel<D, 2, kBf16>, true);
}
cudaError_t preload_kv_attend_kernels() {
  cudaError_t e;
  if ((e = preload_rows<64, true>()) != cudaSuccess) return e;
  if ((e = preload_rows<64, false>()) != cudaSuccess) return e;
  if ((e = preload_rows<128, true>()) != cudaSuccess) return e;
  return preload_rows<128, false>();
}

}  // namespace oilbird
