// Storing into the 4-bit cache and reading it back.
//
// append: eight lanes take the 64 channels of one group (16 bytes each), agree on its minimum
// and maximum with three shuffles, and write one word of codes each and one word of scale and
// offset; a token's group costs 128 bytes in and 36 out.  read: the same lanes, the other way.
// Both are bound by memory on long inputs and by the launch on a decoding step's few rows.
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

template <int D, bool kBf16>
__global__ void __launch_bounds__(kStThreads)
kv_append_kernel(const KvView c, const KvAppendArgs a) {
  constexpr int G = D / kKvGroup, kUnits = 2 * G;        // units of eight lanes per (token, head)
  pdl_enter();
  KvWork* work = reinterpret_cast<KvWork*>(c.work);
  const int lane8 = threadIdx.x & 7;
  const int page = 1 << c.page_shift;
  const size_t block = 2 * (size_t)kv_part_bytes(D, page);
  const long long total = (long long)c.n_seq * a.rows * c.n_kv * kUnits;
  const long long step = (long long)gridDim.x * (kStThreads / 8);
  // (a warp's four units take part in the shuffles together: the loop bound is the warp's)
  for (long long u0 = (long long)blockIdx.x * (kStThreads / 8) + (threadIdx.x >> 5) * 4; u0 < total; u0 += step) {
    const long long u = u0 + ((threadIdx.x & 31) >> 3);
    bool live = u < total;
    const long long row = live ? u / kUnits : 0;         // (sequence, row, head)
    const int part = (int)(live ? u - row * kUnits : 0), kv = part / G, grp = part % G;
    const int head = (int)(row % c.n_kv);
    const long long sr = row / c.n_kv;
    const int s = (int)(sr / a.rows), j = (int)(sr - (long long)s * a.rows);
    const int n = a.n_new ? a.n_new[s] : a.rows;
    live = live && j < n;
    int src = j;
    if (live && a.select) src = a.select[(size_t)s * a.rows + j];
    const int before = c.seq_len[s];
    const long long slot = (long long)(before < 0 ? 0 : before) + j;
    const int p = live ? page_of(c, s, slot) : -1;
    const bool store = live && p >= 0 && src >= 0 && src < a.m;
    if (live && !store && part == 0 && head == 0 && lane8 == 0) atomicAdd(&work->dropped, 1ull);
    uint32_t w[4] = {0, 0, 0, 0};
    if (store) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>((kv ? a.v : a.k).at(s, src, head) + grp * kKvGroup + lane8 * 8);
    float x[8];
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = half_lo<kBf16>(w[e]);
      x[2 * e + 1] = half_hi<kBf16>(w[e]);
    }
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
      bad |= !(fabsf(x[e]) < INFINITY);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    bad = (__ballot_sync(0xffffffffu, bad) >> (threadIdx.x & 24) & 0xffu) != 0;
    // halves: the difference of two finite elements cannot overflow
    uint32_t meta = pack16<kBf16>((hi * 0.5f - lo * 0.5f) / 7.5f, lo);
    const float half = half_lo<kBf16>(meta) * 0.5f, base = lo * 0.5f;
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float q = rintf((x[e] * 0.5f - base) / half);
      q = half > 0.f ? fminf(fmaxf(q, 0.f), 15.f) : 0.f;
      codes |= (uint32_t)(int)q << (4 * (e >> 1) + 16 * (e & 1));
    }
    if (bad) { codes = 0; meta = kBf16 ? 0x7fc07fc0u : 0x7e007e00u; }
    if (store) {
      const int in = (int)(slot & (page - 1));
      unsigned char* b = c.pages + ((size_t)p * c.n_kv + head) * block + kv * (block / 2);
      *reinterpret_cast<uint32_t*>(b + ((size_t)grp * page + in) * 32 + lane8 * 4) = codes;
      if (lane8 == 0) *reinterpret_cast<uint32_t*>(b + (size_t)G * page * 32 + ((size_t)in * G + grp) * 4) = meta;
      if (part == 0 && lane8 == 1) {
        const size_t at = ((size_t)p * c.n_kv + head) * page + in;
        c.weight[at] = a.weight ? a.weight[((size_t)s * c.n_kv + head) * a.m + src] : 0.f;
        c.pos[at] = c.n_pos[s] + j;
      }
    }
  }
  if (last_block(&work->arrivals, gridDim.x)) {
    const long long room = (long long)c.max_pages << c.page_shift;
    for (int s = threadIdx.x; s < c.n_seq; s += kStThreads) {
      int n = a.n_new ? a.n_new[s] : a.rows;
      n = n < 0 ? 0 : (n > a.rows ? a.rows : n);
      const int before = c.seq_len[s];
      const long long after = (long long)(before < 0 ? 0 : before) + n;
      c.seq_len[s] = (int)(after > room ? room : after);
      c.n_pos[s] += n;
    }
  }
}

template <int D, bool kBf16>
__global__ void __launch_bounds__(kStThreads)
kv_read_kernel(const KvView c, const KvReadArgs a) {
  constexpr int G = D / kKvGroup;
  pdl_enter();
  const int lane8 = threadIdx.x & 7;
  const int page = 1 << c.page_shift;
  const size_t block = 2 * (size_t)kv_part_bytes(D, page);
  // units of eight lanes: (sequence, head, K or V, group, row), rows fastest, so that a warp's
  // loads are contiguous
  const long long total = (long long)c.n_seq * c.n_kv * 2 * G * a.n;
  for (long long u = (long long)blockIdx.x * (kStThreads / 8) + (threadIdx.x >> 3); u < total;
       u += (long long)gridDim.x * (kStThreads / 8)) {
    const long long part = u / a.n;
    const int j = (int)(u - part * a.n);
    const int grp = (int)(part % G), kv = (int)(part / G % 2);
    const long long sh = part / (2 * G);
    const int head = (int)(sh % c.n_kv), s = (int)(sh / c.n_kv);
    const long long slot = (a.start ? (long long)a.start[s] : 0) + j;
    uint32_t out[4] = {0, 0, 0, 0};
    if (slot >= 0 && slot < c.seq_len[s]) {
      const int p = page_of(c, s, slot);
      if (p >= 0) {
        const int in = (int)(slot & (page - 1));
        const unsigned char* b = c.pages + ((size_t)p * c.n_kv + head) * block + kv * (block / 2);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(b + ((size_t)grp * page + in) * 32 + lane8 * 4);
        const uint32_t meta = *reinterpret_cast<const uint32_t*>(b + (size_t)G * page * 32 + ((size_t)in * G + grp) * 4);
        const float sc = half_lo<kBf16>(meta), lo = half_hi<kBf16>(meta);
#pragma unroll
        for (int n = 0; n < 4; ++n)
          out[n] = pack16<kBf16>(fmaf((float)(w >> (4 * n) & 15u), sc, lo), fmaf((float)(w >> (16 + 4 * n) & 15u), sc, lo));
      }
    }
    uint16_t* dst = (kv ? a.v : a.k) + (((size_t)s * a.n + j) * c.n_kv + head) * D + grp * kKvGroup + lane8 * 8;
    *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(out);
  }
}

static int grid_for(long long units, int sms) {          // eight blocks an SM, enough for every unit
  const long long want = (units + kStThreads / 8 - 1) / (kStThreads / 8);
  return (int)(want < 8LL * sms ? (want < 1 ? 1 : want) : 8LL * sms);
}

cudaError_t launch_kv_append(const KvView& c, const KvAppendArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st) {
  const int grid = grid_for((long long)c.n_seq * a.rows * c.n_kv * 2 * (head_dim / kKvGroup), sms);
  auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(kStThreads), 0, st, c, a); };
  if (head_dim == 64) return bf16 ? go(kv_append_kernel<64, true>) : go(kv_append_kernel<64, false>);
  return bf16 ? go(kv_append_kernel<128, true>) : go(kv_append_kernel<128, false>);
}
cudaError_t launch_kv_read(const KvView& c, const KvReadArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st) {
  const int grid = grid_for((long long)c.n_seq * c.n_kv * 2 * (head_dim / kKvGroup) * a.n, sms);
  auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(kStThreads), 0, st, c, a); };
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
