// Storing into the 4-bit cache and reading it back.
//
// append: a warp takes one row's four key/value heads of a block (or fewer), 16 bytes a lane: eight lanes
// share the 64 channels of a group, agree on its minimum and maximum (as packed 16-bit
// numbers, three shuffles for both), and write one word of codes each and one word of scale and
// offset; a token's group costs 128 bytes in and 36 out.  read: the same lanes, the other way,
// four slots at a time.  All loads of a warp are on their way before the first is used.
//
// Measured, with 8 heads of 128: 4 prompts of 2,048 to 4,096 rows (12,800 in all) are stored in
// 32 us (68 MB, 2.1 TB/s; bound by the instructions of minima, quotients and packing) and read
// in 16 us (with the zeros behind the shorter ones 85 MB, 5.3 TB/s: memory); 16 paths of four to
// seven rows in 7 and 4.6 us: latency of a launch and three dependent loads.
//
// The quotient (x - lo) / scale is IEEE division's, by Markstein's correction of a product with
// the reciprocal (one division a group): q = x r, q += (x - q scale) r.
//
// The lengths are device memory that every block reads and the call must advance: the block
// that finishes last does it, when nobody reads them any more.
#include "kv.cuh"

namespace oilbird {

constexpr int kStThreads = 256;

// The cache position of a slot: page number or -1.
__device__ __forceinline__ int page_of(const KvView& c, int s, long long slot) {
  if (slot >= (long long)c.max_pages << c.page_shift) return -1;
  const int p = c.table[(size_t)s * c.max_pages + (slot >> c.page_shift)];
  return (p >= 0 && p < c.n_pages) ? p : -1;
}

// True in the block that arrives last (every thread calls; all of the block's reads are done).
__device__ __forceinline__ bool last_block(unsigned* arrivals, unsigned blocks) {
  __shared__ int last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(arrivals, 1u) == blocks - 1;
    if (last) *arrivals = 0u;
  }
  __syncthreads();
  return last;
}

// packed 16-bit minimum and maximum; a NaN wins
template <bool kBf16> __device__ __forceinline__ uint32_t min16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  if (kBf16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <bool kBf16> __device__ __forceinline__ uint32_t max16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  if (kBf16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight lanes' 64 elements (eight each) -> the lane's word of codes, the group's meta.  Two
// elements an instruction wherever there is one for pairs: this is what bounds long appends.
template <bool kBf16>
__device__ __forceinline__ uint32_t quantise64(const uint4& v, uint32_t& meta) {
  const uint32_t lo2 = min16x2<kBf16>(min16x2<kBf16>(v.x, v.y), min16x2<kBf16>(v.z, v.w));
  const uint32_t hi2 = max16x2<kBf16>(max16x2<kBf16>(v.x, v.y), max16x2<kBf16>(v.z, v.w));
  // both halves' minimum in the low half, maximum in the high half
  uint32_t mm = __byte_perm(min16x2<kBf16>(lo2, lo2 >> 16), max16x2<kBf16>(hi2, hi2 << 16), 0x7610);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    const uint32_t y = __shfl_xor_sync(0xffffffffu, mm, o);
    mm = __byte_perm(min16x2<kBf16>(mm, y), max16x2<kBf16>(mm, y), 0x7610);
  }
  const float lo = half_lo<kBf16>(mm), hi = half_hi<kBf16>(mm);
  // halves: the difference of two finite elements cannot overflow
  const float spread = hi * 0.5f - lo * 0.5f;
  constexpr float kInv = 1.f / 7.5f;
  float step = spread * kInv;
  step = fmaf(fmaf(-step, 7.5f, spread), kInv, step);
  meta = pack16<kBf16>(step, lo);
  const float half = half_lo<kBf16>(meta) * 0.5f, base = lo * -0.5f, r = 1.f / half;
  const float2 r2 = make_float2(r, r), h2 = make_float2(-half, -half), b2 = make_float2(base, base),
               two = make_float2(0.5f, 0.5f), one = make_float2(1.f, 1.f), magic = make_float2(12582912.f, 12582912.f);
  uint32_t codes = 0;
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const uint32_t w = (&v.x)[n];
    const float2 x = fma2(make_float2(half_lo<kBf16>(w), half_hi<kBf16>(w)), two, b2);
    float2 q = mul2(x, r2);
    q = fma2(fma2(q, h2, x), r2, q);
    // + 1.5 * 2^23: the sum's low bits are the integer, rounded to nearest, ties to even
    q = fma2(q, one, magic);
    const uint32_t t = __vminu2(__byte_perm(__float_as_uint(q.x), __float_as_uint(q.y), 0x5410), 0x000f000fu);
    codes |= t << (4 * n);
  }
  if (!(half >= 0x1p-120f)) {                            // no scale, or one whose reciprocal is none
    codes = 0;
    if (half > 0.f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = (&v.x)[e >> 1];
        const float x = fmaf(e & 1 ? half_hi<kBf16>(w) : half_lo<kBf16>(w), 0.5f, base);
        codes |= (uint32_t)(int)fminf(rintf(x / half), 15.f) << (4 * (e >> 1) + 16 * (e & 1));
      }
    }
  }
  if (!(fabsf(lo) < INFINITY) || !(fabsf(hi) < INFINITY)) { codes = 0; meta = kBf16 ? 0x7fc07fc0u : 0x7e007e00u; }
  return codes;
}

// grid.y: sequences; a warp: one row's kHeads heads after another, the next one's elements asked
// for before this one's are worked on
constexpr int kStTurns = 4;
template <int D, bool kBf16>
__global__ void __launch_bounds__(kStThreads, 3)
kv_append_kernel(const KvView c, const KvAppendArgs a) {
  constexpr int G = D / kKvGroup, kUnits = 2 * G;        // units of eight lanes per (token, head)
  constexpr int kHeadsATurn = 4 / kUnits, kHeads = kStTurns * kHeadsATurn;
  pdl_enter();
  KvWork* work = reinterpret_cast<KvWork*>(c.work);
  const int lane = threadIdx.x & 31, lane8 = lane & 7, unit = lane >> 3;
  const int kv = unit % kUnits / G, grp = unit % G;
  const int page = 1 << c.page_shift;
  const size_t block = 2 * (size_t)kv_part_bytes(D, page);
  const int s = blockIdx.y;
  int n = a.n_new ? a.n_new[s] : a.rows;
  n = min(n, a.rows);
  const int before = max(c.seq_len[s], 0), pos0 = c.n_pos[s];
  const int head_groups = (c.n_kv + kHeads - 1) / kHeads, stride = gridDim.x * (kStThreads / 32);
  const KvRows& rows = kv ? a.v : a.k;
  struct Row {
    uint4 v[kStTurns];
    float w;
    int j, head0, p;                                     // p: the page; -1: none; -2 - page: no such row
  };
  auto ask = [&](Row& r, int task) {
    r.j = task / head_groups;
    r.head0 = (task - r.j * head_groups) * kHeads;
    r.p = -1;
    if (r.j < n) {
      int src = a.select ? a.select[(size_t)s * a.rows + r.j] : r.j;
      r.p = page_of(c, s, (long long)before + r.j);
      if (src < 0 || src >= a.m) {
        if (r.p >= 0) r.p = -2 - r.p;
        src = 0;
      }
#pragma unroll
      for (int t = 0; t < kStTurns; ++t) {
        const int head = r.head0 + t * kHeadsATurn + unit / kUnits;
        r.v[t] = make_uint4(0, 0, 0, 0);
        if (head < c.n_kv) r.v[t] = *reinterpret_cast<const uint4*>(rows.at(s, src, head) + grp * kKvGroup + lane8 * 8);
      }
      r.w = a.weight && lane < kHeads && r.head0 + lane < c.n_kv
                ? a.weight[((size_t)s * c.n_kv + r.head0 + lane) * a.m + src] : 0.f;
    }
  };
  int task = blockIdx.x * (kStThreads / 32) + (threadIdx.x >> 5);
  Row cur, next;
  ask(cur, task);
  while (cur.j < n) {
    ask(next, task += stride);
    if (cur.p < 0) {
      if (cur.head0 == 0 && lane == 0) atomicAdd(&work->dropped, 1ull);
      if (cur.p < -1) {                                  // its slot counts: NaN, not what lay there before
        cur.p = -2 - cur.p;
#pragma unroll
        for (int t = 0; t < kStTurns; ++t) cur.v[t] = make_uint4(~0u, ~0u, ~0u, ~0u);
        cur.w = 0.f;
      }
    }
    if (cur.p >= 0) {
      const int in = (before + cur.j) & (page - 1);
#pragma unroll
      for (int t = 0; t < kStTurns; ++t) {
        const int head = cur.head0 + t * kHeadsATurn + unit / kUnits;
        uint32_t meta;
        const uint32_t codes = quantise64<kBf16>(cur.v[t], meta);
        if (head < c.n_kv) {
          unsigned char* b = c.pages + ((size_t)cur.p * c.n_kv + head) * block + kv * (block / 2);
          *reinterpret_cast<uint32_t*>(b + (grp * page + in) * 32 + lane8 * 4) = codes;
          if (lane8 == 0) *reinterpret_cast<uint32_t*>(b + (G * page * 8 + in * G + grp) * 4) = meta;
        }
      }
      if (lane < kHeads && cur.head0 + lane < c.n_kv) {
        const size_t at = ((size_t)cur.p * c.n_kv + cur.head0 + lane) * page + in;
        c.weight[at] = cur.w;
        c.pos[at] = pos0 + cur.j;
      }
    }
    cur = next;
  }
  if (last_block(&work->arrivals, gridDim.x * gridDim.y)) {
    const long long room = (long long)c.max_pages << c.page_shift;
    for (int i = threadIdx.x; i < c.n_seq; i += kStThreads) {
      int m = a.n_new ? a.n_new[i] : a.rows;
      m = m < 0 ? 0 : (m > a.rows ? a.rows : m);
      const long long after = (long long)max(c.seq_len[i], 0) + m;
      c.seq_len[i] = (int)(after > room ? room : after);
      c.n_pos[i] += m;
    }
  }
}

// grid.y: sequences; a warp: four slots of one head, K and V, every group
template <int D, bool kBf16>
__global__ void __launch_bounds__(kStThreads)
kv_read_kernel(const KvView c, const KvReadArgs a) {
  constexpr int G = D / kKvGroup;
  pdl_enter();
  const int lane = threadIdx.x & 31, lane8 = lane & 7;
  const int page = 1 << c.page_shift;
  const size_t block = 2 * (size_t)kv_part_bytes(D, page);
  const int s = blockIdx.y, task = blockIdx.x * (kStThreads / 32) + (threadIdx.x >> 5);
  const int j4 = task / c.n_kv, head = task - j4 * c.n_kv, j = j4 * 4 + (lane >> 3);
  if (j >= a.n) return;
  const long long slot = (a.start ? (long long)a.start[s] : 0) + j;
  const int p = slot >= 0 && slot < c.seq_len[s] ? page_of(c, s, slot) : -1;
  uint32_t w[2][G], meta[2][G];
  const int in = (int)(slot & (page - 1));
  const unsigned char* b = c.pages + ((size_t)max(p, 0) * c.n_kv + head) * block;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      w[kv][g] = meta[kv][g] = 0;
      if (p >= 0) w[kv][g] = *reinterpret_cast<const uint32_t*>(b + kv * (block / 2) + (g * page + in) * 32 + lane8 * 4);
    }
    if (p >= 0) load_meta<G>(b + kv * (block / 2) + (G * page * 8 + in * G) * 4, meta[kv]);
  }
  const size_t at = (((size_t)s * a.n + j) * c.n_kv + head) * D + lane8 * 8;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv)
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float sc = half_lo<kBf16>(meta[kv][g]), lo = half_hi<kBf16>(meta[kv][g]);
      uint32_t out[4];
#pragma unroll
      for (int n = 0; n < 4; ++n)
        out[n] = pack16<kBf16>(fmaf((float)(w[kv][g] >> (4 * n) & 15u), sc, lo), fmaf((float)(w[kv][g] >> (16 + 4 * n) & 15u), sc, lo));
      // The scale was rounded, up perhaps, so the largest code may stand for more than the type
      // holds: its largest number then, as the group's elements were finite.
      if (half_hi<kBf16>(pack16<kBf16>(0.f, fmaf(15.f, sc, lo))) == INFINITY) {
        constexpr uint32_t kInf = kBf16 ? 0x7f80u : 0x7c00u;
#pragma unroll
        for (int n = 0; n < 4; ++n) out[n] -= ((out[n] & 0x7fffu) == kInf ? 1u : 0u) + ((out[n] >> 16 & 0x7fffu) == kInf ? 0x10000u : 0u);
      }
      __stcs(reinterpret_cast<uint4*>((kv ? a.v : a.k) + at + g * kKvGroup), make_uint4(out[0], out[1], out[2], out[3]));
    }
}

cudaError_t launch_kv_append(const KvView& c, const KvAppendArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st) {
  const int heads = kStTurns * 4 / (2 * (head_dim / kKvGroup));
  const long long tasks = (long long)a.rows * ((c.n_kv + heads - 1) / heads);
  const long long want = (tasks + kStThreads / 32 - 1) / (kStThreads / 32), most = (3LL * sms + c.n_seq - 1) / c.n_seq;
  const dim3 grid((unsigned)(want < most ? want : most), c.n_seq);       // three blocks an SM
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(kStThreads), 0, st, c, a); };
  if (head_dim == 64) return bf16 ? go(kv_append_kernel<64, true>) : go(kv_append_kernel<64, false>);
  return bf16 ? go(kv_append_kernel<128, true>) : go(kv_append_kernel<128, false>);
}
cudaError_t launch_kv_read(const KvView& c, const KvReadArgs& a, int head_dim, bool bf16, cudaStream_t st) {
  const long long tasks = ((long long)a.n + 3) / 4 * c.n_kv;
  const dim3 grid((unsigned)((tasks + kStThreads / 32 - 1) / (kStThreads / 32)), c.n_seq);
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(kStThreads), 0, st, c, a); };
  if (head_dim == 64) return bf16 ? go(kv_read_kernel<64, true>) : go(kv_read_kernel<64, false>);
  return bf16 ? go(kv_read_kernel<128, true>) : go(kv_read_kernel<128, false>);
}

cudaError_t preload_kv_store_kernels() {
  cudaError_t e;
  if ((e = preload_kernel(kv_append_kernel<64, true>)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_append_kernel<64, false>)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_append_kernel<128, true>)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_append_kernel<128, false>)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_read_kernel<64, true>)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_read_kernel<64, false>)) != cudaSuccess) return e;
  if ((e = preload_kernel(kv_read_kernel<128, true>)) != cudaSuccess) return e;
  return preload_kernel(kv_read_kernel<128, false>);
}

}  // namespace oilbird
