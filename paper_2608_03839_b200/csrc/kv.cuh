// The verifier's 4-bit key/value cache: the format, the views handed to the kernels and the
// device helpers that every kernel over it uses.
//
// Format (the library's reading; the paper names none).  For one slot, one key/value head and
// one of K, V, the channels are taken in groups of 64:
//   lo = min x, hi = max x, scale = rn16((hi - lo) / 15), code_j = rint((x_j - lo) / scale)
// clamped to 0..15; the element stands for scale * code_j + lo.  scale and lo are held in the
// cache's 16-bit type (lo is an element, so it is exact).  4.5 bits a value.  Differences are taken between halves, so
// that the range of two finite elements cannot overflow.  hi == lo, or a scale that rounds to
// zero: code 0.  A group that holds a NaN or an infinity has scale = lo = NaN: all of it reads
// as NaN.
//
// Page block of one key/value head, `page` slots: K codes [group][slot][32 B], K meta
// [slot][group] (one word: scale low half, lo high half), V codes, V meta.  Word w of a
// group's 32 bytes holds channels 8w..8w+7: channel 8w+2n in bits 4n..4n+3, channel 8w+2n+1
// in bits 16+4n..19+4n (n = 0..3).  With that order
//   word & 0x000f000f   is the pair (8w, 8w+1) as two f16 numbers of value code * 2^-24
//   word & 0x00f000f0   is the pair (8w+2, 8w+3) as code * 2^-20
// (f16 subnormals, exact), and (word >> 8) gives the other two pairs: a code costs 0.6
// instructions on its way into a matrix operand, and no arithmetic that could round.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "internal.h"

namespace oilbird {

constexpr int kKvGroup = 64;              // channels that share a scale and an offset
constexpr int kKvMaxSeq = OILBIRD_KV_MAX_SEQ;   // their lengths sit in shared memory
constexpr int kKvMaxCtas = 512;
constexpr float kLog2e = 1.4426950408889634f;

__host__ __device__ inline int kv_part_bytes(int head_dim, int page) {   // K or V of one block
  return head_dim / kKvGroup * page * 36;
}

// Head of the workspace; zeroed once by the caller.
struct KvWork {
  DeviceStats stats;                     // stalled
  unsigned long long dropped;            // appended rows that found no page
  unsigned arrivals;                     // blocks of a running append that have finished
  unsigned pad;
};
constexpr size_t kKvTicketOff = 256;                                  // unsigned [kKvMaxCtas]
constexpr size_t kKvPartOff = kKvTicketOff + 4 * kKvMaxCtas;          // partial results
constexpr int kKvTreeMaxCtas = 160;                                   // of the kernel for many rows
constexpr int kKvPartRows = 2 * kKvTreeMaxCtas * 256;                       // rows of D + 2 floats

struct KvView {
  unsigned char* pages;      // [n_pages, n_kv, block]
  float* weight;             // [n_pages, n_kv, page]
  int32_t* pos;              // [n_pages, n_kv, page]
  const int32_t* table;      // [n_seq, max_pages]
  int32_t* seq_len;          // [n_seq]
  int32_t* n_pos;            // [n_seq]
  unsigned char* work;
  long long n_pages;
  int n_seq, max_pages, page_shift, n_kv;
};

// 16-bit rows [sequence, row, head, channel]; strides in elements
struct KvRows {
  const uint16_t* p;
  long long seq, row, head;
  __host__ __device__ const uint16_t* at(int s, int r, int h) const {
    return p + s * seq + r * row + h * head;
  }
};

struct KvWeighArgs {
  KvRows q, k;               // k.p == nullptr: no new nodes
  float* node_weight;        // [n_seq, n_kv, m] or nullptr
  const float* lse;          // [n_seq, m, n_q] by lse_* strides
  long long lse_seq, lse_row, lse_head;
  const float* row_weight;   // [n_seq, m] or nullptr: one
  const unsigned long long* mask;
  const int32_t* n_new;
  long long mask_stride;
  float scale;
  int m, group;
  int node0, node1;          // rows of this launch: nodes [node0, node1)
};

struct KvAppendArgs {
  KvRows k, v;               // [n_seq, m, n_kv, D]
  const int32_t* n_new;      // [n_seq] or nullptr: `rows` each
  const int32_t* select;     // [n_seq, rows] rows of k and v to take, or nullptr: 0, 1, ...
  const int32_t* first;      // [n_seq + 1] packed: sequence s has rows first[s] .. first[s + 1) of the m; else nullptr
  const float* weight;       // [n_seq, n_kv, m], packed [n_kv, m], or nullptr: 0
  int m, rows;
  // rows that join sequence s, and the first of them
  __device__ __forceinline__ int count(int s, int& base) const {
    base = 0;
    if (!first) return n_new ? min(max(n_new[s], 0), rows) : rows;
    base = min(max(first[s], 0), m);
    return min(max(first[s + 1], base), m) - base;
  }
};
struct KvReadArgs {
  uint16_t *k, *v;           // [n_seq, n, n_kv, D]
  const int32_t* start;      // [n_seq] or nullptr: 0
  int n;
};
struct KvEvictArgs {
  int budget, sink, recent;
  int max_words, held, gather;   // set by the launch
};

struct KvAttendArgs {
  KvRows q, k, v;            // k.p == nullptr: no new nodes
  uint16_t* out;             // [n_seq, m, n_q, D] by out_* strides
  long long out_seq, out_row, out_head;
  float* lse;                // [n_seq, m, n_q] by lse_* strides, or nullptr
  long long lse_seq, lse_row, lse_head;
  const unsigned long long* mask;   // [n_seq] rows of mask_stride words, or nullptr: causal
  const int32_t* n_new;      // [n_seq] or nullptr: m each
  long long mask_stride;
  float scale;
  int m, group;              // nodes per sequence, query heads per key/value head
};

cudaError_t launch_kv_append(const KvView& c, const KvAppendArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st);
cudaError_t launch_kv_read(const KvView& c, const KvReadArgs& a, int head_dim, bool bf16, cudaStream_t st);
cudaError_t launch_kv_attend(const KvView& c, const KvAttendArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st);
cudaError_t launch_kv_tree(const KvView& c, const KvAttendArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st);
cudaError_t launch_kv_weigh(const KvView& c, const KvWeighArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st);
cudaError_t launch_kv_evict(const KvView& c, KvEvictArgs a, int head_dim, int sms, cudaStream_t st);

template <bool kBf16> __device__ __forceinline__ float half_lo(uint32_t w) {
  if (kBf16) return __uint_as_float(w << 16);
  return __half2float(__ushort_as_half((unsigned short)w));
}
template <bool kBf16> __device__ __forceinline__ float half_hi(uint32_t w) {
  if (kBf16) return __uint_as_float(w & 0xffff0000u);
  return __half2float(__ushort_as_half((unsigned short)(w >> 16)));
}
// two floats -> the cache's 16-bit type, the first in the low half
template <bool kBf16> __device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  uint32_t r;
  if (kBf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// pairs of fp32 numbers in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\t"
      "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "mul.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

__device__ __forceinline__ uint32_t kv_smem(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
// 16 bytes global -> shared, past L1; bytes == 0 writes zeros and reads nothing
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// D[16 x 8] += A[16 x 16] B[16 x 8], f16 or bf16 operands, fp32 accumulators
template <bool kBf16>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  if (kBf16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// transpose of an 8 x 8 matrix of 16-bit elements held by the warp
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Query rows enter the products as f16 numbers: a row is multiplied by the power of two that
// brings its largest element to [2^10, 2^11), which is exact, and the power joins the row's
// factor.  (A bf16 element more than 2^20 times smaller than the row's largest becomes an f16
// subnormal and is off by less than 2^-31 of the largest.)
constexpr int kRowTop = 10;
__device__ __forceinline__ int row_exponent(float amax) {
  const int e = (int)(__float_as_uint(amax) >> 23) - 127;
  return e >= 128 ? kRowTop : (e < -110 ? -110 : e);   // infinity, NaN: as they are
}
__device__ __forceinline__ float abs_max(float a, float b) { return fmaxf(a, fabsf(b)); }

// Whole sums over a block's threads in front of each thread (exclusive); `total` of all.
// scratch: one entry per warp.  Every thread calls.
template <int kThreads>
__device__ __forceinline__ long long block_exclusive_scan(long long v, long long* scratch, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) scratch[warp] = x;
  __syncthreads();
  long long before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const long long y = scratch[w];
    if (w < warp) before += y;
    total += y;
  }
  __syncthreads();
  return before + x - v;
}

// ---- tiles ----
// The slots of all (sequence, key head, row block) items, kTile to a tile, are one list: sequence
// by sequence, its items in turn, its tiles in turn.  An item begins with kFront tiles: the new
// nodes in the first of them, nothing in the others.  Nodes come first because their loads
// depend on nothing, and the front stands for what an item costs besides its slots (operands,
// joining), so that a block that gets many short items gets fewer slots.  Items whose rows do
// not exist have one empty tile.
template <int kTile, int kFront, int kFew>
struct TileListOf {
  struct Cursor {
    int s;                // sequence
    int len, nodes;       // its slots and new nodes
    int tiles;            // tiles of each of its items that have rows ...
    int live;             // ... and how many items those are
    int item, head, tile; // head: item modulo the key heads
    __device__ __forceinline__ int slot0() const { return (tile - kFront) * kTile; }
    __device__ __forceinline__ bool cached() const { return item < live && tile >= kFront; }
  };

  long long* cum;       // shared memory: [n_seq + 1] tiles in front of each sequence
  int* len;             // [n_seq], within the table's room
  unsigned char* nodes; // [n_seq], 0..m
  long long total;
  int n_seq, n_kv, items;      // items of every sequence
  int group, rows;             // query heads per key head, rows per block (0: all items live)

  __device__ __forceinline__ int live_items(int n) const {
    return rows == 0 ? items : n_kv * ((n * group + rows - 1) / rows);
  }
  __device__ __forceinline__ int tiles_of(int l) const { return (l + kTile - 1) / kTile + kFront; }
  __device__ __forceinline__ long long tiles_in(int l, int n) const {
    const int live = live_items(n);
    return (long long)live * tiles_of(l) + (items - live);
  }
  // Every thread calls; scratch: a word per warp.
  template <int kThreads>
  __device__ __forceinline__ void build(const KvView& c, const int32_t* n_new, int m, long long* scratch) {
    n_seq = c.n_seq;
    n_kv = c.n_kv;
    const int per = (n_seq + kThreads - 1) / kThreads, tid = threadIdx.x;
    const long long room = (long long)c.max_pages << c.page_shift;
    long long mine = 0;
    for (int i = 0; i < per; ++i) {
      const int s = tid * per + i;
      if (s < n_seq) {
        int l = c.seq_len[s], n = n_new ? n_new[s] : m;
        l = l < 0 ? 0 : (l > room ? (int)room : l);
        n = n < 0 ? 0 : (n > m ? m : n);
        len[s] = l;
        nodes[s] = (unsigned char)n;
        mine += tiles_in(l, n);
      }
    }
    long long at = block_exclusive_scan<kThreads>(mine, scratch, total);
    for (int i = 0; i < per; ++i) {
      const int s = tid * per + i;
      if (s < n_seq) {
        cum[s] = at;
        at += tiles_in(len[s], nodes[s]);
      }
    }
    __syncthreads();
  }
  // Cursors are the same in every lane; the shuffles say so, which moves their arithmetic out of
  // the lanes' registers.
  __device__ __forceinline__ void load(Cursor& k, int s) const {
    k.s = s;
    k.len = __shfl_sync(0xffffffffu, len[s], 0);
    k.nodes = __shfl_sync(0xffffffffu, (int)nodes[s], 0);
    k.tiles = tiles_of(k.len);
    k.live = live_items(k.nodes);
  }
  __device__ __forceinline__ void seek(Cursor& k, long long u) const {   // to list position u
    int lo = 0, hi = n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (cum[mid] <= u) lo = mid; else hi = mid - 1;
    }
    lo = __shfl_sync(0xffffffffu, lo, 0);
    load(k, lo);
    const long long r = u - cum[lo], full = (long long)k.live * k.tiles;
    int item, tile = 0;
    if (r < full) {
      item = full <= 0x7fffffffLL ? (int)((uint32_t)r / (uint32_t)k.tiles) : (int)(r / k.tiles);
      tile = (int)(r - (long long)item * k.tiles);
    } else {
      item = k.live + (int)(r - full);
    }
    k.item = __shfl_sync(0xffffffffu, item, 0);
    k.tile = __shfl_sync(0xffffffffu, tile, 0);
    k.head = k.item % n_kv;
  }
  // The list is cut at raw(b) = total b / n_cta, but not where that would leave a piece of
  // hardly more than an item's first round, or the last few tiles of one: such a cut moves to the item's
  // edge.  (Every block finds the same cuts.)
  // (Where blocks get little, more so: an item's few tiles are better left together.)
  __device__ __forceinline__ int near_end(int n_cta) const { return total < kFew * n_cta ? 4 : 1; }
  __device__ __forceinline__ int near_start(int n_cta) const { return kFront + near_end(n_cta); }
  __device__ __forceinline__ long long cut(Cursor& k, int b, int n_cta) const {
    // (32-bit division wherever the numbers allow: the 64-bit one is a long routine)
    const long long u = total * n_cta <= 0xffffffffLL ? (long long)((uint32_t)total * (uint32_t)b / (uint32_t)n_cta)
                                                      : total * b / n_cta;
    if (u >= total) return total;
    seek(k, u);
    const int tiles = k.item < k.live ? k.tiles : 1;
    if (k.tile <= near_start(n_cta)) { const long long at = u - k.tile; k.tile = 0; return at; }
    if (tiles - k.tile > near_end(n_cta)) return u;
    const int on = tiles - k.tile;
    if (u + on < total) advance(k, on);
    return u + on;
  }
  // Blocks that share the item [i0, i0 + tiles): b0..b1.
  __device__ __forceinline__ void owners(long long i0, int tiles, int n_cta, int& b0, int& b1) const {
    const long long lo = i0 + near_start(n_cta) + 1, hi = i0 + tiles - near_end(n_cta);
    // in front of the first cut behind the start; the last cut before the end
    if ((total + 64) * (n_cta + 1) <= 0xffffffffLL) {
      const uint32_t t = (uint32_t)total, n = (uint32_t)n_cta;
      b0 = (int)(((uint32_t)lo * n + t - 1) / t) - 1;
      b1 = (int)(((uint32_t)hi * n + t - 1) / t) - 1;
    } else {
      b0 = (int)((lo * n_cta + total - 1) / total) - 1;
      b1 = (int)((hi * n_cta + total - 1) / total) - 1;
    }
    if (b1 < b0) b1 = b0;
  }
  __device__ __forceinline__ void advance(Cursor& k, int n) const {      // n tiles on, inside the list
    for (k.tile += n;;) {
      const int here = k.item < k.live ? k.tiles : 1;
      if (k.tile < here) return;
      k.tile -= here;
      if (++k.head == n_kv) k.head = 0;
      if (++k.item == items) { load(k, k.s + 1); k.item = k.head = 0; }
    }
  }
};

constexpr int kKvTile = 64, kKvNodeTile = 32, kKvFront = 8;
using TileList = TileListOf<kKvTile, kKvFront, 64>;
using TileCursor = TileList::Cursor;

// The pages that hold a tile's quarters of 16 slots, lane q the q-th's; -1 where the table names
// none or the quarter has no slot.
__device__ __forceinline__ int tile_pages(const KvView& c, const TileCursor& k, int lane) {
  int p = -1;
  if (k.cached() && lane < 4) {
    const int slot = k.slot0() + lane * 16;
    if (slot < k.len) {
      p = c.table[(size_t)k.s * c.max_pages + (slot >> c.page_shift)];
      p = (uint32_t)p < (uint32_t)c.n_pages ? p : -1;
    }
  }
  return p;
}
// Starts the copies of a tile's keys (kValue 0) or values (1), a whole warp: codes
// [group][slot][32 B] and meta [slot][group].  Quarters without a page are zeroed.
template <int D, int kValue>
__device__ __forceinline__ void copy_tile(const KvView& c, const TileCursor& k, int pages,
                                          unsigned char* dst_ptr, int lane) {
  constexpr int G = D / kKvGroup;
  const uint32_t dst = kv_smem(dst_ptr) + lane * 16;
  const int page = 1 << c.page_shift;
  const size_t block = 2 * (size_t)kv_part_bytes(D, page);
  if (c.page_shift == 6) {                               // the tile is a page
    constexpr int kPart = G * kKvTile * 36, kChunks = kPart / 16;    // as it lies in memory
    const int p = __shfl_sync(0xffffffffu, pages, 0);
    const uint32_t n = p < 0 ? 0 : 16;
    const unsigned char* b = c.pages + ((size_t)(uint32_t)max(p, 0) * c.n_kv + k.head) * block + kValue * kPart + lane * 16;
#pragma unroll
    for (int i = 0; i < kChunks; i += 32)
      if (i + 32 <= kChunks || i + lane < kChunks) cp_async16(dst + i * 16, b + i * 16, n);
    return;
  }
  const int part = G * page * 36;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int p = __shfl_sync(0xffffffffu, pages, q), in = (k.slot0() + q * 16) & (page - 1);
    const unsigned char* b = c.pages + ((size_t)(uint32_t)max(p, 0) * c.n_kv + k.head) * block + kValue * part;
    const uint32_t n = p < 0 ? 0 : 16;
#pragma unroll
    for (int i = 0; i < G; ++i) cp_async16(dst + i * 2048 + q * 512, b + (i * page + in) * 32 + lane * 16, n);
    if (lane < 4 * G) cp_async16(dst + G * 2048 + q * 64 * G, b + (G * page * 8 + in * G) * 4 + lane * 16, n);
  }
}
// bit i: slot i of the tile exists and has a page
__device__ __forceinline__ unsigned long long tile_valid(const TileCursor& k, int pages) {
  const int left = k.len - k.slot0();
  const uint32_t have = __ballot_sync(0xffffffffu, pages >= 0);
  if (left >= 64 && (have & 15u) == 15u) return ~0ull;
  unsigned long long v = left >= 64 ? ~0ull : (1ull << left) - 1ull;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (!(have >> q & 1u)) v &= ~(0xffffull << (16 * q));
  return v;
}
// Zeroes the meta of a tile's slots that are not valid, so that whatever lay there is finite.
template <int G>
__device__ __forceinline__ void clear_meta(unsigned char* meta, unsigned long long valid, int lane) {
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int sl = lane + 32 * e;
    if (!(valid >> sl & 1ull)) {
#pragma unroll
      for (int i = 0; i < G; ++i) reinterpret_cast<uint32_t*>(meta)[sl * G + i] = 0u;
    }
  }
}

// One query row as matrix operands: what lane (row g, t4) of a warp holds of it.  b[step] are
// the pairs of a product step; sum[group] the row's sums (all lanes of the row); returns the
// row's factor exponent.  have == false: zeros.  negate: for a negative scale, so that factors
// are positive and the largest product is the largest score.
template <int D, bool kBf16>
__device__ __forceinline__ int row_operands(const uint16_t* qp, bool have, int t4, bool negate,
                                            uint32_t (&b)[D / 16][2], float (&sum)[D / kKvGroup]) {
  constexpr int G = D / kKvGroup;
  float x[G][16], top = 0.f;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    uint32_t w[8];
    if (have) {
      *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(qp + i * kKvGroup + t4 * 16);
      *reinterpret_cast<uint4*>(w + 4) = *reinterpret_cast<const uint4*>(qp + i * kKvGroup + t4 * 16 + 8);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = 0;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[i][2 * e] = half_lo<kBf16>(w[e]);
      x[i][2 * e + 1] = half_hi<kBf16>(w[e]);
      top = abs_max(abs_max(top, x[i][2 * e]), x[i][2 * e + 1]);
    }
  }
  top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const int e0 = row_exponent(top);
  const float up = negate ? -pow2(kRowTop - e0) : pow2(kRowTop - e0);
#pragma unroll
  for (int i = 0; i < G; ++i) {
    sum[i] = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) { x[i][e] *= up; sum[i] += x[i][e]; }
#pragma unroll
    for (int j = 0; j < 4; ++j) {                        // the odd pairs meet codes times 16
      b[i * 4 + j][0] = pack16<false>(x[i][4 * j], x[i][4 * j + 1]);
      b[i * 4 + j][1] = pack16<false>(x[i][4 * j + 2] * 0.0625f, x[i][4 * j + 3] * 0.0625f);
    }
    sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
    sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
  }
  return e0;
}
// What a score in the products' units is multiplied by to become an exponent of two.
__device__ __forceinline__ float row_factor(float scale, int e0) {
  return fmaxf(fabsf(scale) * kLog2e * (0x1p24f / (float)(1 << kRowTop)) * pow2(e0), 1e-37f);
}
// The scales and offsets of one slot.
template <int G> __device__ __forceinline__ void load_meta(const unsigned char* p, uint32_t (&m)[G]) {
  if (G == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    m[0] = v.x;
    m[G - 1] = v.y;
  } else {
    m[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

}  // namespace oilbird
