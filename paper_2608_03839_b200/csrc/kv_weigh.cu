// Attention weight that cached slots receive: for every slot j and key/value head
//   weight[j] += sum_i r_i sum_{h of the head's group} exp(c q_ih.k_j - lse_ih),
// and the same sums for the new nodes.  Rows with r_i = 0 (the draft tree's rejected nodes) and
// rows that see nothing take no part.
//
// The keys' half of the cache is read once, with the products and the layout of the attention
// kernel (exact codes as f16 operands, scale and offset in fp32); what follows the scores is
// one exponential each and a sum over the rows.  A slot's sum is formed by one warp in a fixed
// order and added once, so the result does not depend on which block ran when (where every page is one
// sequence's).  The rows that
// take part are gathered per item, so a tree of sixty nodes of which five were accepted costs
// five; their operands lie in shared memory and every tile is multiplied with all of them.
//
// Measured, with 8 key/value heads of 128: one row of 32 query heads over 64 sequences of 4,096
// to 8,192 slots in 76 us (250 MB of codes, scales and weights read and written: 3.3 TB/s; 38 us
// at the copy rate), accepted paths of up to seven nodes over 8 sequences of 2,048 to 4,096 slots
// in 26 us.  Bound by instructions: a slot's share of taking codes apart is the attention
// kernel's, while it brings half of the bytes; on short sequences by the launch, the gathering of
// the rows and the first tile.
#include "kv.cuh"

namespace oilbird {

constexpr int kWgThreads = 256, kWgWarps = 8, kWgStages = 2;
constexpr int kWgMaxRows = 256;                          // rows of one launch

template <int D>
struct WeighShared {
  static constexpr int kStage = kKvTile * (D / kKvGroup) * 36;       // K codes, K meta
  static constexpr int kRing = kWgWarps * kWgStages * kStage;
  static constexpr int kRowTile = 32 * (D / 16) * 8;                 // operands of 8 rows
  // behind the ring: cum, scratch, len, per row: sum per group, factor, lse, weight, index
  static constexpr int kFixed = kRing + (kKvMaxSeq + 1) * 8 + kWgWarps * 8 + kKvMaxSeq * 5 +
                                kWgWarps * kWgStages * 8 + 64;
  static int bytes(int row_tiles) { return kFixed + row_tiles * (kRowTile + 8 * 4 * (D / kKvGroup + 4)); }
};

template <int D, bool kBf16>
__global__ void __launch_bounds__(kWgThreads, 2)
kv_weigh_kernel(const KvView c, const KvWeighArgs a, int row_tiles) {
  using Sh = WeighShared<D>;
  constexpr int G = D / kKvGroup, kSteps = D / 16;
  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* ring = smem;
  uint2* qs = reinterpret_cast<uint2*>(smem + Sh::kRing);            // [row tile][step][lane]
  float* row_sum = reinterpret_cast<float*>(smem + Sh::kRing + row_tiles * Sh::kRowTile);   // [G][row]
  float* row_f = row_sum + row_tiles * 8 * G;
  float* row_lse = row_f + row_tiles * 8;                            // in exponents of two
  float* row_w = row_lse + row_tiles * 8;
  int* row_id = reinterpret_cast<int*>(row_w + row_tiles * 8);
  long long* cum = reinterpret_cast<long long*>(row_id + row_tiles * 8);
  long long* scratch = cum + kKvMaxSeq + 1;
  unsigned long long* valid_s = reinterpret_cast<unsigned long long*>(scratch + kWgWarps);
  int* len_s = reinterpret_cast<int*>(valid_s + kWgWarps * kWgStages);
  int* count_s = len_s + kKvMaxSeq;                                  // [kWgWarps + 1]
  unsigned char* nodes_s = reinterpret_cast<unsigned char*>(count_s + kWgWarps + 1);

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  pdl_enter();

  TileList list;
  list.cum = cum;
  list.len = len_s;
  list.nodes = nodes_s;
  list.items = c.n_kv;
  list.group = a.group;
  list.rows = 0;
  list.build<kWgThreads>(c, a.n_new, a.m, scratch);
  const long long total = list.total;
  const int n_cta = (int)min((long long)gridDim.x, (total + kWgWarps - 1) / kWgWarps);
  if (blockIdx.x >= n_cta) return;
  TileCursor bc, pc;                                     // the block's item; the warp's next tile to copy
  const long long u1_all = list.cut(pc, blockIdx.x + 1, n_cta), u0 = list.cut(bc, blockIdx.x, n_cta);
  const int u1 = (int)(u1_all - u0);                     // positions from here on count from u0
  if (u1 <= 0) return;

  unsigned char* my_ring = ring + warp * (kWgStages * Sh::kStage);
  unsigned long long* my_valid = valid_s + warp * kWgStages;
  int pu = warp, ahead = -1;
  pc = bc;
  if (pu < u1) { list.advance(pc, warp); ahead = tile_pages(c, pc, lane); }
  auto issue = [&](int stage) {
    if (pu < u1) {
      if (pc.cached()) {
        copy_tile<D, 0>(c, pc, ahead, my_ring + stage * Sh::kStage, lane);
        const unsigned long long v = tile_valid(pc, ahead);
        if (lane == 0) my_valid[stage] = v;
      }
      pu += kWgWarps;
      if (pu < u1) { list.advance(pc, kWgWarps); ahead = tile_pages(c, pc, lane); }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kWgStages; ++i) issue(i);
  int stage = 0;

  int mu = warp;
  for (int at = 0; at < u1;) {
    const int head = bc.item, s = bc.s;
    const int piece = min(bc.tiles - bc.tile, u1 - at), item_u0 = at - bc.tile;

    // ---- the rows that take part, in order ----
    const int first = a.node0 * a.group, last = min(a.node1, bc.nodes) * a.group;
    float rw = 0.f, rl = -INFINITY;
    const int row = first + tid;                         // at most kWgMaxRows of them
    if (row < last) {
      const int node = row / a.group;
      rw = a.row_weight ? a.row_weight[(size_t)s * a.m + node] : 1.f;
      rl = a.lse[s * a.lse_seq + node * a.lse_row + (head * a.group + row % a.group) * a.lse_head];
    }
    const bool part = rw != 0.f && rl != -INFINITY;      // (a NaN takes part)
    const uint32_t votes = __ballot_sync(0xffffffffu, part);
    if (lane == 0) count_s[warp] = __popc(votes);
    for (int i = tid; i < row_tiles * 8; i += kWgThreads) { row_w[i] = 0.f; row_lse[i] = 0.f; row_id[i] = -1; }
    __syncthreads();
    int before = 0, n_part = 0;
#pragma unroll
    for (int w = 0; w < kWgWarps; ++w) {
      if (w < warp) before += count_s[w];
      n_part += count_s[w];
    }
    if (part) {
      const int i = before + __popc(votes & ((1u << lane) - 1u));
      row_w[i] = rw;
      row_lse[i] = rl * kLog2e;
      row_id[i] = row;
    }
    __syncthreads();
    const int n_tiles = (n_part + 7) / 8;
    for (int r = warp; r < n_tiles; r += kWgWarps) {
      const int id = row_id[r * 8 + g];
      const bool have = id >= 0;
      uint32_t b[kSteps][2];
      float sum[G];
      const int e0 = row_operands<D, kBf16>(a.q.at(s, have ? id / a.group : 0, head * a.group + (have ? id % a.group : 0)),
                                            have, t4, a.scale < 0.f, b, sum);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) qs[(r * kSteps + j) * 32 + lane] = make_uint2(b[j][0], b[j][1]);
      if (t4 == 0) {
        row_f[r * 8 + g] = have ? row_factor(a.scale, e0) : 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i) row_sum[i * row_tiles * 8 + r * 8 + g] = sum[i] * 0x1p-24f;
      }
    }
    __syncthreads();

    for (; mu < at + piece; mu += kWgWarps) {
      const int tile = mu - item_u0, slot0 = (tile - kKvFront) * kKvTile;
      cp_async_wait<kWgStages - 1>();
      __syncwarp();
      if (tile >= kKvFront) {
        unsigned char* st = my_ring + stage * Sh::kStage;
        unsigned char* kmeta = st + G * kKvTile * 32;
        const unsigned long long valid = my_valid[stage];
        if (__any_sync(0xffffffffu, valid != ~0ull)) {
          clear_meta<G>(kmeta, valid, lane);
          __syncwarp();
        }
        const int slot_g = (g >> 1) + 4 * (g & 1);
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {           // 32 slots: two chunks
          float got[2][2] = {{0.f, 0.f}, {0.f, 0.f}};    // chunk, logical rows g and g + 8
          uint2 w[2][2][G];
          float sc[2][2][G], lo[2][2][G];
#pragma unroll
          for (int ch = 0; ch < 2; ++ch)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int sl = pair * 32 + ch * 16 + slot_g + 8 * k;
              uint32_t meta[G];
              load_meta<G>(kmeta + sl * 4 * G, meta);
#pragma unroll
              for (int i = 0; i < G; ++i) {
                w[ch][k][i] = *reinterpret_cast<const uint2*>(st + (i * kKvTile + sl) * 32 + t4 * 8);
                sc[ch][k][i] = half_lo<kBf16>(meta[i]);
                lo[ch][k][i] = half_hi<kBf16>(meta[i]);
              }
            }
          for (int r = 0; r < n_tiles; ++r) {
            float f[2], ls[2], rwt[2], qsum[G][2];
            const int i2 = r * 8 + 2 * t4;               // the lane's two rows
            *reinterpret_cast<float2*>(f) = *reinterpret_cast<const float2*>(row_f + i2);
            *reinterpret_cast<float2*>(ls) = *reinterpret_cast<const float2*>(row_lse + i2);
            *reinterpret_cast<float2*>(rwt) = *reinterpret_cast<const float2*>(row_w + i2);
#pragma unroll
            for (int k = 0; k < G; ++k)
              *reinterpret_cast<float2*>(qsum[k]) = *reinterpret_cast<const float2*>(row_sum + k * row_tiles * 8 + i2);
            float x[2][4];
#pragma unroll
            for (int i = 0; i < G; ++i) {
              float acc[2][4];
#pragma unroll
              for (int ch = 0; ch < 2; ++ch)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[ch][e] = 0.f;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint2 b = qs[(r * kSteps + i * 4 + j) * 32 + lane];
#pragma unroll
                for (int ch = 0; ch < 2; ++ch) {
                  const uint32_t x0 = (j & 2 ? w[ch][0][i].y : w[ch][0][i].x) >> (8 * (j & 1));
                  const uint32_t x1 = (j & 2 ? w[ch][1][i].y : w[ch][1][i].x) >> (8 * (j & 1));
                  mma16816<false>(acc[ch], x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u,
                                  b.x, b.y);
                }
              }
#pragma unroll
              for (int ch = 0; ch < 2; ++ch)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float y = lo[ch][e >> 1][i] * qsum[i][e & 1];
                  x[ch][e] = fmaf(sc[ch][e >> 1][i], acc[ch][e], i ? x[ch][e] + y : y);
                }
            }
#pragma unroll
            for (int ch = 0; ch < 2; ++ch)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                got[ch][e >> 1] = fmaf(rwt[e & 1], exp2_approx(fmaf(x[ch][e], f[e & 1], -ls[e & 1])), got[ch][e >> 1]);
          }
          // the four lanes of a slot hold two rows each; then lane t4 adds slot (t4 & 1) * 8 of
          // chunk t4 / 2
          float mine = 0.f;
#pragma unroll
          for (int ch = 0; ch < 2; ++ch)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float v = got[ch][k];
              v += __shfl_xor_sync(0xffffffffu, v, 1);
              v += __shfl_xor_sync(0xffffffffu, v, 2);
              if (t4 == ch * 2 + k) mine = v;
            }
          const int sl = pair * 32 + (t4 >> 1) * 16 + (t4 & 1) * 8 + slot_g;
          if (n_tiles && (valid >> sl & 1)) {
            const int slot = slot0 + sl, page = 1 << c.page_shift;
            const int p = c.table[(size_t)s * c.max_pages + (slot >> c.page_shift)];
            // nobody else adds to this slot in this launch (unless sequences share the page): the
            // result has no order to depend on
            atomicAdd(c.weight + ((size_t)p * c.n_kv + head) * page + (slot & (page - 1)), mine);
          }
        }
      } else if (a.node_weight && tile * kKvNodeTile < a.m) {
        // ---- new nodes ----
        const int node0 = tile * kKvNodeTile;
        float got[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
        for (int r = 0; r < n_tiles; ++r) {
          const int id = row_id[r * 8 + g];
          float x[2][4];
#pragma unroll
          for (int ch = 0; ch < 2; ++ch)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[ch][e] = 0.f;
#pragma unroll
          for (int i = 0; i < G; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int at_ch = i * kKvGroup + t4 * 16 + half * 8;
              uint4 qw = make_uint4(0, 0, 0, 0);
              if (id >= 0) qw = *reinterpret_cast<const uint4*>(a.q.at(s, id / a.group, head * a.group + id % a.group) + at_ch);
#pragma unroll
              for (int ch = 0; ch < 2; ++ch) {
                uint4 kw[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const int node = node0 + ch * 16 + g + 8 * k;
                  kw[k] = make_uint4(0, 0, 0, 0);
                  if (node < bc.nodes) kw[k] = *reinterpret_cast<const uint4*>(a.k.at(s, node, head) + at_ch);
                }
                mma16816<kBf16>(x[ch], kw[0].x, kw[1].x, kw[0].y, kw[1].y, qw.x, qw.y);
                mma16816<kBf16>(x[ch], kw[0].z, kw[1].z, kw[0].w, kw[1].w, qw.z, qw.w);
              }
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int i = r * 8 + 2 * t4 + e, rid = row_id[i];
            const int node_r = rid < 0 ? 0 : rid / a.group;
            const unsigned long long sees = rid < 0 ? 0ull : a.mask ? a.mask[s * a.mask_stride + node_r] : (2ull << node_r) - 1ull;
            const float w = row_w[i], ls = row_lse[i];
#pragma unroll
            for (int ch = 0; ch < 2; ++ch)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int node = node0 + ch * 16 + g + 8 * k;
                if (node < bc.nodes && (sees >> node & 1ull))
                  got[ch][k] = fmaf(w, exp2_approx(fmaf(x[ch][e + 2 * k], a.scale * kLog2e, -ls)), got[ch][k]);
              }
          }
        }
#pragma unroll
        for (int ch = 0; ch < 2; ++ch)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float v = got[ch][k];
            v += __shfl_xor_sync(0xffffffffu, v, 1);
            v += __shfl_xor_sync(0xffffffffu, v, 2);
            const int node = node0 + ch * 16 + g + 8 * k;
            if (t4 == ch * 2 + k && node < a.m) {
              float* p = a.node_weight + ((size_t)s * c.n_kv + head) * a.m + node;
              *p = a.node0 == 0 ? v : *p + v;            // a later launch of the same call adds
            }
          }
      }
      __syncwarp();
      issue(stage);
      stage = stage == kWgStages - 1 ? 0 : stage + 1;
    }
    __syncthreads();
    at += piece;
    if (at < u1) list.advance(bc, piece);
  }
}

template <int D, bool kBf16>
static cudaError_t weigh_launch(const KvView& c, KvWeighArgs a, int sms, cudaStream_t st) {
  // a launch takes kWgMaxRows rows; more nodes follow in launches of their own, on the same
  // stream, so that a slot's sums are added one after the other
  const int per = a.group >= kWgMaxRows ? 1 : kWgMaxRows / a.group;
  for (int n = 0; n < a.m; n += per) {
    a.node0 = n;
    a.node1 = n + per < a.m ? n + per : a.m;
    const int row_tiles = ((a.node1 - a.node0) * a.group + 7) / 8;
    const cudaError_t e = launch_pdl(kv_weigh_kernel<D, kBf16>, dim3(2 * sms),
                                     dim3(kWgThreads), WeighShared<D>::bytes(row_tiles), st, c, a, row_tiles);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_kv_weigh(const KvView& c, const KvWeighArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st) {
  if (head_dim == 64) return bf16 ? weigh_launch<64, true>(c, a, sms, st) : weigh_launch<64, false>(c, a, sms, st);
  return bf16 ? weigh_launch<128, true>(c, a, sms, st) : weigh_launch<128, false>(c, a, sms, st);
}

cudaError_t preload_kv_weigh_kernels() {
  cudaError_t e;
  if ((e = preload_kernel(kv_weigh_kernel<64, true>, true)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_weigh_kernel<64, false>, true)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_weigh_kernel<128, true>, true)) != cudaSuccess) return e;
  return preload_kernel(kv_weigh_kernel<128, false>, true);
}

}  // namespace oilbird
