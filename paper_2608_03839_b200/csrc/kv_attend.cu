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
// rounding, at most 2^-11 of each term), and the offsets are summed in fp32.
//
// Layout.  The products are taken transposed, S^T = K Q^T with 16 slots x 8 rows and
// O^T = V^T P^T with 16 channels x 8 rows, so that 8 rows (the query heads of one key head)
// fill a matrix instruction; P^T goes from accumulator to operand layout by an 8 x 8
// transpose.  Rows of a 16-slot chunk are dealt out so that logical row 2t is slot t and
// 2t+1 is slot t+4: then both the K loads (8 bytes a lane) and the V loads (4 bytes a lane)
// take 256 and 128 contiguous bytes of shared memory.
//
// Work.  The tiles (32 slots) of all (sequence, head, row block) items are one list, cut into
// equal runs, one per block; a block's eight warps take the run's tiles in turn, each
// through a ring of its own (asynchronous 16-byte copies, no block-wide waits), which runs on
// across items.  At the end of an item's share the warps' results are joined in
// shared memory; items cut between blocks go through the workspace, and the block that
// finishes last joins the pieces, in their order, whichever block that is.
#include "kv.cuh"

namespace oilbird {

constexpr int kAtThreads = 256, kAtWarps = 8, kAtTile = kKvTile, kAtStages = 4;

template <int D>
struct AttendShared {
  static constexpr int kStage = kAtTile * (D / kKvGroup) * 72;       // K codes, K meta, V codes, V meta
  static constexpr int kRing = kAtWarps * kAtStages * kStage;
  static constexpr int kObuf = kAtWarps * 8 * (D + 4) * 4;
  static constexpr int kMl = kAtWarps * 8 * 8;
  static constexpr int kValid = kAtWarps * kAtStages * 4;
  static constexpr int kCum = (kKvMaxSeq + 1) * 8;
  static constexpr int kBytes = kRing + kObuf + kMl + kValid + kCum + kKvMaxSeq * 5 + kAtWarps * 8 + 16;
};

template <int D, int NT, bool kBf16>
__global__ void __launch_bounds__(kAtThreads, 1)
kv_attend_kernel(const KvView c, const KvAttendArgs a) {
  using Sh = AttendShared<D>;
  constexpr int G = D / kKvGroup, kRows = NT * 8, kSteps = D / 16;
  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* ring = smem;
  float* obuf = reinterpret_cast<float*>(smem + Sh::kRing);
  float2* ml = reinterpret_cast<float2*>(smem + Sh::kRing + Sh::kObuf);
  uint32_t* valid_s = reinterpret_cast<uint32_t*>(smem + Sh::kRing + Sh::kObuf + Sh::kMl);
  long long* cum = reinterpret_cast<long long*>(smem + Sh::kRing + Sh::kObuf + Sh::kMl + Sh::kValid);
  long long* scratch = cum + kKvMaxSeq + 1;
  int* len_s = reinterpret_cast<int*>(scratch + kAtWarps);
  unsigned char* nodes_s = reinterpret_cast<unsigned char*>(len_s + kKvMaxSeq);
  int* flag = reinterpret_cast<int*>(nodes_s + kKvMaxSeq);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const int rblocks = (a.m * a.group + kRows - 1) / kRows;
  pdl_enter();

  TileList list;
  list.cum = cum;
  list.len = len_s;
  list.nodes = nodes_s;
  list.items = c.n_kv * rblocks;
  list.group = a.group;
  list.rows = kRows;
  list.node_tiles = a.k.p ? -1 : 0;
  list.build<kAtThreads>(c, a.n_new, a.m, scratch);
  const long long total = list.total;
  // blocks share the list evenly; no block gets less than a tile for each of its warps
  const long long n_cta = min((long long)gridDim.x, (total + kAtWarps - 1) / kAtWarps);
  if (blockIdx.x >= n_cta) return;
  auto share_at = [&](long long b) { return total * b / n_cta; };
  auto owner = [&](long long u) { return (int)(((u + 1) * n_cta - 1) / total); };
  const long long u0 = share_at(blockIdx.x), u1 = share_at(blockIdx.x + 1);

  // ---- the warp's ring of tiles ----
  unsigned char* my_ring = ring + warp * (kAtStages * Sh::kStage);
  uint32_t* my_valid = valid_s + warp * kAtStages;
  TileCursor pc;
  long long pu = u0 + warp;                              // the next tile to copy, its pages
  int ahead = -1;
  if (pu < u1) { list.seek(pc, pu); ahead = tile_pages(c, pc, lane); }
  auto issue = [&](int stage) {
    if (pu < u1) {
      const int slot0 = pc.tile * kAtTile;
      if (pc.item < pc.live && slot0 < pc.len) {
        const int p0 = __shfl_sync(0xffffffffu, ahead, 0), p1 = __shfl_sync(0xffffffffu, ahead, 1);
        copy_tile<D, true>(c, pc.item % c.n_kv, slot0, p0, p1, my_ring + stage * Sh::kStage, lane);
        if (lane == 0) my_valid[stage] = tile_valid(pc.len - slot0, p0, p1);
      }
      pu += kAtWarps;
      if (pu < u1) { list.advance(pc, kAtWarps); ahead = tile_pages(c, pc, lane); }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kAtStages - 1; ++i) issue(i);
  int stage = 0;

  // ---- item by item ----
  TileCursor bc;
  list.seek(bc, u0);
  long long mu = u0 + warp;                              // the warp's next tile to compute
  for (long long at = u0; at < u1;) {
    const int item = bc.item, tile0 = bc.tile;
    const int n_tiles = item < bc.live ? bc.tiles : 1;
    const int piece = (int)min((long long)(n_tiles - tile0), u1 - at);
    const long long item_u0 = at - tile0;
    // live items: head fastest, then row block; the others follow in the same order
    const int head = item % c.n_kv;
    const int rb = item / c.n_kv, row0 = rb * kRows;
    const int n_rows = bc.nodes * a.group;               // rows of the sequence that exist
    const int s = bc.s;

    float o[NT][4 * G][4];                               // channel tiles x rows, in units of 2^(eref + 24)
    float olo[NT][G][2], l[NT][2], m[NT][2];
    int eref = -120;
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

    if (mu < at + piece && item < bc.live) {
      // ---- query rows as operands ----
      uint32_t qf[NT][kSteps][2];
      float f[NT][2], qsum[NT][G][2];
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        const int row = row0 + r * 8 + g;
        const bool have = row < n_rows;
        const int node = have ? row / a.group : 0;
        float sum[G];
        const int e0 = row_operands<D, kBf16>(a.q.at(s, node, head * a.group + (have ? row % a.group : 0)), have, t4,
                                              qf[r], sum);
#pragma unroll
        for (int i = 0; i < G; ++i) {                    // accumulators hold rows 2t and 2t+1
          qsum[r][i][0] = __shfl_sync(0xffffffffu, sum[i], 8 * t4) * 0x1p-24f;
          qsum[r][i][1] = __shfl_sync(0xffffffffu, sum[i], 8 * t4 + 4) * 0x1p-24f;
        }
        const float ff = row_factor(a.scale, e0);
        f[r][0] = __shfl_sync(0xffffffffu, ff, 8 * t4);
        f[r][1] = __shfl_sync(0xffffffffu, ff, 8 * t4 + 4);
      }

      for (; mu < at + piece; mu += kAtWarps) {
        const int tile = (int)(mu - item_u0);
        cp_async_wait<kAtStages - 2>();
        __syncwarp();
        const unsigned char* st = my_ring + stage * Sh::kStage;
        const int slot0 = tile * kAtTile;
        if (slot0 < bc.len) {
          const uint32_t valid = my_valid[stage];
          const uint32_t* kmeta = reinterpret_cast<const uint32_t*>(st + G * kAtTile * 32);
          const unsigned char* vst = st + G * kAtTile * 36;
          const uint32_t* vmeta = reinterpret_cast<const uint32_t*>(vst + G * kAtTile * 32);
          float sc[NT][2][4];
          const int slot_g = (g >> 1) + 4 * (g & 1);     // logical row g of a chunk
          // ---- scores ----
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            const int sl = ch * 16 + slot_g;
            const bool ok0 = valid >> sl & 1, ok1 = valid >> (sl + 8) & 1;
#pragma unroll
            for (int r = 0; r < NT; ++r)
#pragma unroll
              for (int e = 0; e < 4; ++e) sc[r][ch][e] = 0.f;
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const uint2 w0 = *reinterpret_cast<const uint2*>(st + (i * kAtTile + sl) * 32 + t4 * 8);
              const uint2 w1 = *reinterpret_cast<const uint2*>(st + (i * kAtTile + sl + 8) * 32 + t4 * 8);
              uint32_t meta0 = kmeta[sl * G + i], meta1 = kmeta[(sl + 8) * G + i];
              meta0 = ok0 ? meta0 : 0u;
              meta1 = ok1 ? meta1 : 0u;
              float acc[NT][4];
#pragma unroll
              for (int r = 0; r < NT; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[r][e] = 0.f;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t x0 = (j & 2 ? w0.y : w0.x) >> (8 * (j & 1));
                const uint32_t x1 = (j & 2 ? w1.y : w1.x) >> (8 * (j & 1));
#pragma unroll
                for (int r = 0; r < NT; ++r)
                  mma16816<false>(acc[r], x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u,
                                  x1 & 0x00f000f0u, qf[r][i * 4 + j][0], qf[r][i * 4 + j][1]);
              }
              const float s0 = half_lo<kBf16>(meta0), l0 = half_hi<kBf16>(meta0);
              const float s1 = half_lo<kBf16>(meta1), l1 = half_hi<kBf16>(meta1);
#pragma unroll
              for (int r = 0; r < NT; ++r) {
                sc[r][ch][0] = fmaf(s0, acc[r][0], fmaf(l0, qsum[r][i][0], sc[r][ch][0]));
                sc[r][ch][1] = fmaf(s0, acc[r][1], fmaf(l0, qsum[r][i][1], sc[r][ch][1]));
                sc[r][ch][2] = fmaf(s1, acc[r][2], fmaf(l1, qsum[r][i][0], sc[r][ch][2]));
                sc[r][ch][3] = fmaf(s1, acc[r][3], fmaf(l1, qsum[r][i][1], sc[r][ch][3]));
              }
            }
#pragma unroll
            for (int r = 0; r < NT; ++r) {
              sc[r][ch][0] = ok0 ? sc[r][ch][0] * f[r][0] : -INFINITY;
              sc[r][ch][1] = ok0 ? sc[r][ch][1] * f[r][1] : -INFINITY;
              sc[r][ch][2] = ok1 ? sc[r][ch][2] * f[r][0] : -INFINITY;
              sc[r][ch][3] = ok1 ? sc[r][ch][3] * f[r][1] : -INFINITY;
            }
          }
          // ---- running maximum; the value scales' power of two ----
          uint32_t vm[2][2][G];
          uint32_t vtop = 0;
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            const int sl = ch * 16 + slot_g;
#pragma unroll
            for (int i = 0; i < G; ++i) {
              vm[ch][0][i] = (valid >> sl & 1) ? vmeta[sl * G + i] : 0u;
              vm[ch][1][i] = (valid >> (sl + 8) & 1) ? vmeta[(sl + 8) * G + i] : 0u;
              const uint32_t b0 = vm[ch][0][i] & 0xffffu, b1 = vm[ch][1][i] & 0xffffu;
              const uint32_t inf = kBf16 ? 0x7f80u : 0x7c00u;
              vtop = max(vtop, b0 < inf ? b0 : 0u);
              vtop = max(vtop, b1 < inf ? b1 : 0u);
            }
          }
          vtop = __reduce_max_sync(0xffffffffu, vtop);
          const int etile = kBf16 ? min(max((int)(vtop >> 7) - 126, -120), 100) : (int)(vtop >> 10) - 14;
          float mx[NT][2];
          bool grow = etile > eref;
#pragma unroll
          for (int r = 0; r < NT; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x = fmaxf(fmaxf(sc[r][0][e], sc[r][0][e + 2]), fmaxf(sc[r][1][e], sc[r][1][e + 2]));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
              mx[r][e] = x;
              // p may grow to 2^8 before the accumulators are brought to a new maximum
              grow |= x > m[r][e] + 8.f;
            }
          if (__any_sync(0xffffffffu, grow)) {
            const int enew = max(eref, etile);
            const float ve = pow2(max(eref - enew, -126));
            eref = enew;
#pragma unroll
            for (int r = 0; r < NT; ++r)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float mn = fmaxf(m[r][e], mx[r][e]);
                const float down = mn == -INFINITY ? 1.f : exp2_approx(m[r][e] - mn);
                m[r][e] = mn;
                l[r][e] *= down;
#pragma unroll
                for (int i = 0; i < G; ++i) olo[r][i][e] *= down;
#pragma unroll
                for (int i = 0; i < 4 * G; ++i) { o[r][i][e] *= down * ve; o[r][i][e + 2] *= down * ve; }
              }
          }
          const float vdown = pow2(-eref);
          // ---- probabilities, and the products with the values ----
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            float vs[2][G], vl[2][G];
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                vs[k][i] = half_lo<kBf16>(vm[ch][k][i]) * vdown;
                vl[k][i] = half_hi<kBf16>(vm[ch][k][i]);
              }
            uint32_t pb[NT][G][2];
#pragma unroll
            for (int r = 0; r < NT; ++r) {
              float p[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float mm = m[r][e & 1] == -INFINITY ? 0.f : m[r][e & 1];
                p[e] = exp2_approx(sc[r][ch][e] - mm);
              }
              l[r][0] += p[0] + p[2];
              l[r][1] += p[1] + p[3];
#pragma unroll
              for (int i = 0; i < G; ++i) {
                olo[r][i][0] = fmaf(p[0], vl[0][i], fmaf(p[2], vl[1][i], olo[r][i][0]));
                olo[r][i][1] = fmaf(p[1], vl[0][i], fmaf(p[3], vl[1][i], olo[r][i][1]));
                pb[r][i][0] = transpose8x8(pack16<false>(p[0] * vs[0][i], p[1] * vs[0][i]));
                pb[r][i][1] = transpose8x8(pack16<false>(p[2] * vs[1][i], p[3] * vs[1][i]));
              }
            }
            // operand column 2t is slot t, 2t+1 slot t+4 (and +8): as the scores' rows
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const unsigned char* vp = vst + (i * kAtTile + ch * 16 + t4) * 32 + g * 4;
              const uint32_t w0 = *reinterpret_cast<const uint32_t*>(vp);
              const uint32_t w1 = *reinterpret_cast<const uint32_t*>(vp + 4 * 32);
              const uint32_t w2 = *reinterpret_cast<const uint32_t*>(vp + 8 * 32);
              const uint32_t w3 = *reinterpret_cast<const uint32_t*>(vp + 12 * 32);
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
        } else {
          // ---- new nodes: 16-bit keys and values, with the tree's mask ----
          const int cached_tiles = (bc.len + kAtTile - 1) / kAtTile;
          const int node0 = (tile - cached_tiles) * kAtTile;
          if (a.k.p && node0 < bc.nodes) {
            float sc[NT][2][4];
#pragma unroll
            for (int r = 0; r < NT; ++r)
#pragma unroll
              for (int ch = 0; ch < 2; ++ch)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[r][ch][e] = 0.f;
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
              for (int half = 0; half < 2; ++half) {     // 8 channels at a time
                uint4 kw[2][2];
#pragma unroll
                for (int ch = 0; ch < 2; ++ch)
#pragma unroll
                  for (int k = 0; k < 2; ++k) {
                    const int node = node0 + ch * 16 + g + 8 * k;
                    kw[ch][k] = make_uint4(0, 0, 0, 0);
                    if (node < bc.nodes)
                      kw[ch][k] = *reinterpret_cast<const uint4*>(a.k.at(s, node, head) + i * kKvGroup + t4 * 16 + half * 8);
                  }
#pragma unroll
                for (int r = 0; r < NT; ++r) {
                  const int row = row0 + r * 8 + g;
                  uint4 qw = make_uint4(0, 0, 0, 0);
                  if (row < n_rows)
                    qw = *reinterpret_cast<const uint4*>(a.q.at(s, row / a.group, head * a.group + row % a.group) +
                                                         i * kKvGroup + t4 * 16 + half * 8);
#pragma unroll
                  for (int ch = 0; ch < 2; ++ch) {
                    mma16816<kBf16>(sc[r][ch], kw[ch][0].x, kw[ch][1].x, kw[ch][0].y, kw[ch][1].y, qw.x, qw.y);
                    mma16816<kBf16>(sc[r][ch], kw[ch][0].z, kw[ch][1].z, kw[ch][0].w, kw[ch][1].w, qw.z, qw.w);
                  }
                }
              }
            const float fs = a.scale * kLog2e;
            float mx[NT][2];
#pragma unroll
            for (int r = 0; r < NT; ++r)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int row = row0 + r * 8 + 2 * t4 + e;
                unsigned long long sees = 0;
                if (row < n_rows) {
                  const int node = row / a.group;
                  sees = a.mask ? a.mask[s * a.mask_stride + node] : (2ull << node) - 1ull;
                }
                mx[r][e] = -INFINITY;
#pragma unroll
                for (int ch = 0; ch < 2; ++ch)
#pragma unroll
                  for (int k = 0; k < 2; ++k) {
                    const int node = node0 + ch * 16 + g + 8 * k;
                    const bool ok = node < bc.nodes && (sees >> node & 1ull);
                    float& x = sc[r][ch][e + 2 * k];
                    x = ok ? x * fs : -INFINITY;
                    mx[r][e] = fmaxf(mx[r][e], x);
                  }
                mx[r][e] = fmaxf(mx[r][e], __shfl_xor_sync(0xffffffffu, mx[r][e], 4));
                mx[r][e] = fmaxf(mx[r][e], __shfl_xor_sync(0xffffffffu, mx[r][e], 8));
                mx[r][e] = fmaxf(mx[r][e], __shfl_xor_sync(0xffffffffu, mx[r][e], 16));
              }
            // These products need no units: the accumulators are brought to 1 and, as the last
            // tiles of the item, left at eref >= 0, where no finite value overflows.
            const float there = pow2(min(eref + 24, 127));
            eref = max(eref, 0);
            const float back = pow2(-(eref + 24));
#pragma unroll
            for (int r = 0; r < NT; ++r)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float mn = fmaxf(m[r][e], mx[r][e]);
                const float down = mn == -INFINITY ? 1.f : exp2_approx(m[r][e] - mn);
                m[r][e] = mn;
                l[r][e] *= down;
#pragma unroll
                for (int i = 0; i < G; ++i) olo[r][i][e] *= down;
#pragma unroll
                for (int i = 0; i < 4 * G; ++i) { o[r][i][e] *= down * there; o[r][i][e + 2] *= down * there; }
              }
#pragma unroll
            for (int ch = 0; ch < 2; ++ch) {
              // p as the sum of two 16-bit numbers: with bf16 one alone would be as coarse as
              // the result's own rounding
              uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
              for (int r = 0; r < NT; ++r)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  float p[2], q[2];
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const float mm = m[r][e] == -INFINITY ? 0.f : m[r][e];
                    p[e] = exp2_approx(sc[r][ch][e + 2 * k] - mm);
                    l[r][e] += p[e];
                  }
                  const uint32_t h = pack16<kBf16>(p[0], p[1]);
                  q[0] = p[0] - half_lo<kBf16>(h);
                  q[1] = p[1] - half_hi<kBf16>(h);
                  hi[r][k] = transpose8x8(h);
                  lo[r][k] = transpose8x8(pack16<kBf16>(q[0], q[1]));
                }
#pragma unroll
              for (int i = 0; i < G; ++i) {
                uint4 w[4];                              // nodes 2t, 2t+1, 2t+8, 2t+9; 8 channels
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const int node = node0 + ch * 16 + 2 * t4 + (k & 1) + 8 * (k >> 1);
                  w[k] = make_uint4(0, 0, 0, 0);
                  if (node < bc.nodes)
                    w[k] = *reinterpret_cast<const uint4*>(a.v.at(s, node, head) + i * kKvGroup + g * 8);
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                  const uint32_t x0 = (&w[0].x)[n], x1 = (&w[1].x)[n], x2 = (&w[2].x)[n], x3 = (&w[3].x)[n];
                  const uint32_t ea = __byte_perm(x0, x1, 0x5410), oa = __byte_perm(x0, x1, 0x7632);
                  const uint32_t eb = __byte_perm(x2, x3, 0x5410), ob = __byte_perm(x2, x3, 0x7632);
#pragma unroll
                  for (int r = 0; r < NT; ++r) {
                    // channel pair 2n: the cached codes of odd n carry 16 times their value
                    float (&d)[4] = o[r][i * 4 + n];
                    if (n & 1) {
#pragma unroll
                      for (int e = 0; e < 4; ++e) d[e] *= 0.0625f;
                    }
                    mma16816<kBf16>(d, ea, oa, eb, ob, hi[r][0], hi[r][1]);
                    mma16816<kBf16>(d, ea, oa, eb, ob, lo[r][0], lo[r][1]);
                    if (n & 1) {
#pragma unroll
                      for (int e = 0; e < 4; ++e) d[e] *= 16.f;
                    }
                  }
                }
              }
            }
#pragma unroll
            for (int r = 0; r < NT; ++r)
#pragma unroll
              for (int i = 0; i < 4 * G; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][i][e] *= back;
          }
        }
        __syncwarp();
        issue(stage == 0 ? kAtStages - 1 : stage - 1);
        stage = stage == kAtStages - 1 ? 0 : stage + 1;
      }
    } else {
      for (; mu < at + piece; mu += kAtWarps) {          // items without rows: nothing was copied
        cp_async_wait<kAtStages - 2>();
        issue(stage == 0 ? kAtStages - 1 : stage - 1);
        stage = stage == kAtStages - 1 ? 0 : stage + 1;
      }
    }

    // ---- the warps' results joined; the item's share written ----
    const int b0 = owner(item_u0), b1 = owner(item_u0 + n_tiles - 1);
    const bool whole = b0 == b1;
    float* parts = reinterpret_cast<float*>(c.work + kKvPartOff);
    const size_t part_floats = (size_t)kRows * (D + 2);
    float* my_part = parts + (size_t)(2 * blockIdx.x + (blockIdx.x == b0 ? 1 : 0)) * part_floats;
    const float unit = pow2(min(eref + 24, 127));
    constexpr int kOs = D + 4, kPer = D / 32;            // floats a thread handles of its row
    const int row_w = warp;                              // joining: warp w takes row w

    auto finish = [&](int r, float big, float sum, const float (&v)[kPer]) {
      const int row = row0 + r * 8 + row_w;
      if (row < a.m * a.group) {
        const int node = row / a.group, hq = head * a.group + row % a.group;
        if (row >= n_rows) sum = 0.f;                    // behind the sequence's nodes
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint16_t* op = a.out + s * a.out_seq + node * a.out_row + hq * a.out_head + lane * kPer;
        uint32_t w[kPer / 2];
#pragma unroll
        for (int e = 0; e < kPer / 2; ++e)
          w[e] = sum == 0.f ? 0u : pack16<kBf16>(v[2 * e] * inv, v[2 * e + 1] * inv);
        if (kPer == 4) *reinterpret_cast<uint2*>(op) = make_uint2(w[0], w[kPer / 2 - 1]);
        else *reinterpret_cast<uint32_t*>(op) = w[0];
        if (a.lse && lane == 0)
          a.lse[s * a.lse_seq + node * a.lse_row + hq * a.lse_head] =
              sum == 0.f ? -INFINITY : (big + log2f(sum)) * 0.6931471805599453f;
      }
    };

#pragma unroll
    for (int r = 0; r < NT; ++r) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) {
          l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], x);
#pragma unroll
          for (int i = 0; i < G; ++i) olo[r][i][e] += __shfl_xor_sync(0xffffffffu, olo[r][i][e], x);
        }
        float* dst = obuf + (warp * 8 + 2 * t4 + e) * kOs + g * 8;
#pragma unroll
        for (int i = 0; i < G; ++i) {
          // channels 8g + 2n (accumulator e) and 8g + 2n + 1 (e + 2); odd n carry 16 times
          float v[8];
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const float u = n & 1 ? unit * 0.0625f : unit;
            v[2 * n] = fmaf(o[r][i * 4 + n][e], u, olo[r][i][e]);
            v[2 * n + 1] = fmaf(o[r][i * 4 + n][e + 2], u, olo[r][i][e]);
          }
          *reinterpret_cast<float4*>(dst + i * kKvGroup) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4*>(dst + i * kKvGroup + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
        if (g == 0) ml[warp * 8 + 2 * t4 + e] = make_float2(m[r][e], l[r][e]);
      }
      __syncthreads();
      {
        float big = -INFINITY, sum = 0.f, v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kAtWarps; ++w) big = fmaxf(big, ml[w * 8 + row_w].x);
#pragma unroll
        for (int w = 0; w < kAtWarps; ++w) {
          const float2 x = ml[w * 8 + row_w];
          const float k = x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : exp2_approx(x.x - big);
          sum = fmaf(k, x.y, sum);
          if (k != 0.f) {
            const float* src = obuf + (w * 8 + row_w) * kOs + lane * kPer;
#pragma unroll
            for (int e = 0; e < kPer; ++e) v[e] = fmaf(k, src[e], v[e]);
          }
        }
        if (whole) {
          finish(r, big, sum, v);
        } else {
          float* dst = my_part + (size_t)(r * 8 + row_w) * D + lane * kPer;
#pragma unroll
          for (int e = 0; e < kPer; ++e) __stcg(dst + e, v[e]);
          if (lane == 0)
            __stcg(reinterpret_cast<float2*>(my_part + (size_t)kRows * D) + r * 8 + row_w, make_float2(big, sum));
        }
      }
      __syncthreads();
    }
    if (!whole) {
      unsigned* ticket = reinterpret_cast<unsigned*>(c.work + kKvTicketOff) + b0;
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const unsigned n = atomicAdd(ticket, 1u);
        *flag = n == (unsigned)(b1 - b0);
        if (*flag) *ticket = 0u;                         // for the next call
      }
      __syncthreads();
      if (*flag) {
        __threadfence();
#pragma unroll 1
        for (int r = 0; r < NT; ++r) {
          float big = -INFINITY, sum = 0.f, v[kPer];
#pragma unroll
          for (int e = 0; e < kPer; ++e) v[e] = 0.f;
          auto part_of = [&](int b) { return parts + (size_t)(2 * b + (b == b0 ? 1 : 0)) * part_floats; };
          for (int p0 = b0; p0 <= b1; p0 += 32) {
            float2 x = make_float2(-INFINITY, 0.f);
            if (p0 + lane <= b1)
              x = __ldcg(reinterpret_cast<const float2*>(part_of(p0 + lane) + (size_t)kRows * D) + r * 8 + row_w);
            float top = fmaxf(x.x, __shfl_xor_sync(0xffffffffu, x.x, 16));
#pragma unroll
            for (int sft = 8; sft; sft >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, sft));
            const float nb = fmaxf(big, top);
            const float down = big == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : exp2_approx(big - nb);
            sum *= down;
#pragma unroll
            for (int e = 0; e < kPer; ++e) v[e] *= down;
            big = nb;
            const float k = x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : exp2_approx(x.x - nb);
            const int n = min(32, b1 - p0 + 1);
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
              const float ki = __shfl_sync(0xffffffffu, k, i);
              const float li = __shfl_sync(0xffffffffu, x.y, i);
              sum = fmaf(ki, li, sum);
              const float* src = part_of(p0 + i) + (size_t)(r * 8 + row_w) * D + lane * kPer;
#pragma unroll
              for (int e = 0; e < kPer; ++e) {
                const float y = __ldcg(src + e);
                v[e] = ki != 0.f ? fmaf(ki, y, v[e]) : v[e];
              }
            }
          }
          finish(r, big, sum, v);
        }
      }
      __syncthreads();
    }
    at += piece;
    if (at < u1) list.advance(bc, piece);
  }
}

template <int D, int NT, bool kBf16>
static cudaError_t attend_launch(const KvView& c, const KvAttendArgs& a, int sms, cudaStream_t st) {
  return launch_pdl(kv_attend_kernel<D, NT, kBf16>, dim3(sms), dim3(kAtThreads), AttendShared<D>::kBytes, st, c, a);
}
template <int D, bool kBf16>
static cudaError_t attend_rows(const KvView& c, const KvAttendArgs& a, int sms, cudaStream_t st) {
  const int rows = a.m * a.group;
  if (rows <= 8) return attend_launch<D, 1, kBf16>(c, a, sms, st);
  if (rows <= 16) return attend_launch<D, 2, kBf16>(c, a, sms, st);
  return attend_launch<D, 4, kBf16>(c, a, sms, st);
}

cudaError_t launch_kv_attend(const KvView& c, const KvAttendArgs& a, int head_dim, bool bf16, int sms,
                             cudaStream_t st) {
  if (sms > kKvMaxCtas) sms = kKvMaxCtas;
  if (head_dim == 64) return bf16 ? attend_rows<64, true>(c, a, sms, st) : attend_rows<64, false>(c, a, sms, st);
  return bf16 ? attend_rows<128, true>(c, a, sms, st) : attend_rows<128, false>(c, a, sms, st);
}

template <int D, bool kBf16>
static cudaError_t preload_rows() {
  cudaError_t e;
  if ((e = preload_kernel(kv_attend_kernel<D, 1, kBf16>, true)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_attend_kernel<D, 2, kBf16>, true)) != cudaSuccess) return e;
  return preload_kernel(kv_attend_kernel<D, 4, kBf16>, true);
}
cudaError_t preload_kv_attend_kernels() {
  cudaError_t e;
  if ((e = preload_rows<64, true>()) != cudaSuccess) return e;
  if ((e = preload_rows<64, false>()) != cudaSuccess) return e;
  if ((e = preload_rows<128, true>()) != cudaSuccess) return e;
  return preload_rows<128, false>();
}

}  // namespace oilbird
