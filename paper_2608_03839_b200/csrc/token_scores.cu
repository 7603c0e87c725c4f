// Scores of tokens from logits, in one reading of them: with m = max_j x_j and S = sum_j exp(x_j - m)
//
//   lse = m + ln S,   logp(t) = x_t - lse,   entropy = ln S - sum_j exp(x_j - m) (x_j - m) / S
//
// and the k best tokens by (logit descending, token ascending).
//
// A block of 256 threads goes through a row, or where there are few rows through its part of one: the
// blocks of a row are a cluster and join their sums and lists through shared memory.  Parts begin
// where they fall; 16-byte loads cover what is aligned, single elements the (up to 15) others.  Each thread holds
// sums of its own under a maximum of its own: no thread waits for another to add up.  Exponentials are
// 2^((x - m) log2 e): the difference first, as it is exact where it counts and stays a number for the largest and lowest ones.
//
// The k best.  What reaches a floor is among them or near: the k-th largest of 64 or 128 groups' largest values so far,
// which k elements reach and few pass, found anew after 1, 3, 7, 15, .. loads.  A thread whose load holds something that
// reaches it notes the load and goes on (taking elements out of registers there and then cost 5 us of 135); at the end the
// noted loads are read once more, and their elements that reach the last floor make a list in shared memory.  Otherwise nobody
// waits for anybody in that either; where there turn out to be too many notes or elements (long runs of equal or rising
// values), or too few above -inf, the block goes through its part again, cutting the list to
// its k best each time it is full and raising the floor to the k-th, a composite of value and token.  Cutting
// counts for each entry how many are better, which is its place: no sort, and little code, as what runs
// once a row is bound by fetching it (a bitonic sort and straight-line code for each of a thread's 32
// elements took 15 us a row; a barrier a load 100 us on 2,048 rows).  Blocks that go from row to row, the next one's
// first load under way meanwhile, took 170 us: registers.
//
// Measured, with bf16 logits: 2,048 rows of 152,064 with 5 alternatives in 132 us (623 MB, 4.7 TB/s; 111 us without
// alternatives, 5.6 TB/s), 64 rows of 128,256 in 12 us, one row of 128,256 in fp32 with 20 alternatives in 12 us.  Many rows
// are bound by instructions (two thirds of the issue slots: taking pairs apart, exponentials, three sums) beside
// the memory, few by the chain of a launch, loads, floor, list and join.
#include <cooperative_groups.h>
#include <stdio.h>
#include <string.h>

#include <atomic>

#include "kv.cuh"

namespace cg = cooperative_groups;

namespace oilbird {

namespace {

constexpr int kTsThreads = 256, kTsWarps = kTsThreads / 32, kTsUnroll = 4, kTsList = 1024;
constexpr int kTsMaxParts = 8;
static_assert(OILBIRD_SCORES_MAX_TOP <= kTsList / kTsMaxParts && OILBIRD_SCORES_MAX_TOP <= 64, "the lists of a row's blocks");
constexpr float kTsLn2 = 0.6931471805599453f;
enum { kTsBf16 = OILBIRD_LOGITS_BF16, kTsF16 = OILBIRD_LOGITS_F16, kTsF32 = OILBIRD_LOGITS_F32 };

struct TsArgs {
  const unsigned char* logits;
  long long row_bytes;
  const int32_t* tokens;
  float *logp, *lse, *entropy, *top_logp;
  int32_t* top_id;
  int vocab, part, n_tokens, k;      // part: elements of a row that a block takes
};
struct TsSums {
  float m, s, e;                     // maximum; sums of 2^z and of 2^z z with z = (x - m) log2 e
};
struct TsShared {
  alignas(16) u64 list[kTsList];
  alignas(16) float group[128];
  int seen[kTsList];                 // first reading: which threads' loads hold something for the list
  u64 floor;                         // what is not above it is not among the k best (second reading)
  float floor_x;                     // what is below it is not (first reading)
  int count;                         // of entries (of `seen`, then of the list), and those that found no room
  TsSums sums[kTsWarps];
};

template <int kType> struct TsType {
  static constexpr int kBytes = kType == kTsF32 ? 4 : 2, kPer = 16 / kBytes, kAll = kPer * kTsUnroll;
  static constexpr uint32_t kNone = kType == kTsF32 ? 0xff800000u : kType == kTsF16 ? 0xfc00fc00u : 0xff80ff80u;   // -inf
  static __device__ __forceinline__ float get(const uint4& v, int i) {                      // element i of sixteen bytes
    const uint32_t w = (&v.x)[i * kBytes / 4];
    if (kType == kTsF32) return __uint_as_float(w);
    return i & 1 ? half_hi<kType == kTsBf16>(w) : half_lo<kType == kTsBf16>(w);
  }
  // the largest of sixteen bytes' elements (NaN says nothing); pairs first where a word is one
  static __device__ __forceinline__ float largest(const uint4& v) {
    if (kType == kTsF32) return fmaxf(fmaxf(get(v, 0), get(v, 1)), fmaxf(get(v, 2), get(v, 3)));
    uint32_t r = pair_max(pair_max(v.x, v.y), pair_max(v.z, v.w));
    return fmaxf(half_lo<kType == kTsBf16>(r), half_hi<kType == kTsBf16>(r));
  }
  static __device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b) {
    uint32_t r;
    if (kType == kTsBf16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float one(const unsigned char* p) {
    if (kType == kTsF32) return __ldg(reinterpret_cast<const float*>(p));
    const uint32_t w = __ldg(reinterpret_cast<const unsigned short*>(p));
    return half_lo<kType == kTsBf16>(w);
  }
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// The same sums under a maximum that is not smaller.
__device__ __forceinline__ TsSums brought_to(const TsSums& x, float m) {
  const float d = x.m == m ? 0.f : max_nan((x.m - m) * kLog2e, -400.f);          // (equal infinities are no distance)
  const float f = exp2_approx(d);
  return TsSums{m, f * x.s, f * fmaf(x.s, d, x.e)};
}
__device__ __forceinline__ TsSums joined(const TsSums& a, const TsSums& b) {
  const float m = fmaxf(a.m, b.m);
  const TsSums x = brought_to(a, m), y = brought_to(b, m);
  return TsSums{m, x.s + y.s, x.e + y.e};
}
// Keeps the k best of the list's first n (at most kTsList) entries, in order; every thread calls, behind a barrier.
template <int kMine>
__device__ __forceinline__ void cut_list_of(TsShared& sh, int n, int k) {
  u64 key[kMine];
  int place[kMine];
#pragma unroll
  for (int r = 0; r < kMine; ++r) {
    const int i = r * kTsThreads + threadIdx.x;
    key[r] = i < n ? sh.list[i] : 0ull;
    place[r] = 0;
  }
  const ulonglong2* pairs = reinterpret_cast<const ulonglong2*>(sh.list);
  if (n & 1 && threadIdx.x == 0) sh.list[n] = 0ull;      // (an even place: kTsList is even)
  __syncthreads();
  if (kMine > 1 || threadIdx.x / 32 * 32 < n) {
#pragma unroll 4
    for (int j = 0; j < (n + 1) / 2; ++j) {
      const ulonglong2 y = pairs[j];
#pragma unroll
      for (int r = 0; r < kMine; ++r) place[r] += (y.x > key[r]) + (y.y > key[r]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kMine; ++r)
    if (key[r] != 0ull && place[r] < k) {
      sh.list[place[r]] = key[r];
      if (place[r] == k - 1) sh.floor = key[r];
    }
  if (threadIdx.x == 0) sh.count = min(n, k);
  __syncthreads();
}
__device__ __noinline__ void cut_list(TsShared& sh, int n, int k) {
  if (n <= kTsThreads) cut_list_of<1>(sh, n, k);
  else cut_list_of<kTsList / kTsThreads>(sh, n, k);
}

// The floor that the threads' largest values so far (m) allow, in sh.floor_x; every thread calls.  More groups:
// fewer elements pass, more to count.
__device__ __noinline__ void raise_floor(TsShared& sh, float m, int k) {
  const int tid = threadIdx.x, shares = k <= 32 ? 4 : 2; // threads of a group, each of which counts its share of the groups
  float g = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
  if (shares == 4) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
  const int group = tid / shares, share = kTsThreads / shares / shares;
  if (tid % shares == 0) sh.group[group] = g;
  __syncthreads();
  int better = 0;
  const int j0 = tid % shares * share;
#pragma unroll 4
  for (int j = j0; j < j0 + share; j += 4) {
    const float4 y = *reinterpret_cast<const float4*>(sh.group + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) better += (&y.x)[e] > g || ((&y.x)[e] == g && j + e < group);
  }
  better += __shfl_xor_sync(0xffffffffu, better, 1);
  if (shares == 4) better += __shfl_xor_sync(0xffffffffu, better, 2);
  if (better == k - 1) sh.floor_x = fmaxf(g, -3.402823466e38f);
  __syncthreads();
}
// The list, from the first n noted loads and the single elements: what reaches the last floor; every thread calls, behind a barrier.
template <int kType>
__device__ __noinline__ void collect(TsShared& sh, int n, float m, int k, const unsigned char* x0, int first, int vectors, int single) {
  using E = TsType<kType>;
  constexpr int kOnce = 2;
  if (n > kTsThreads / 2) raise_floor(sh, m, k);
  const float floor_x = sh.floor_x;
  __syncthreads();
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
  auto add = [&](float x, int token) {
    if (x >= floor_x) {
      const int to = atomicAdd(&sh.count, 1);
      if (to < kTsList) sh.list[to] = pack_candidate(x, token);
    }
  };
  if (single >= 0) add(E::one(x0 + (long long)single * E::kBytes), single);
  const uint4* src = reinterpret_cast<const uint4*>(x0 + (long long)first * E::kBytes);
  for (int i0 = threadIdx.x; i0 < n * kTsUnroll; i0 += kOnce * kTsThreads) {
    uint4 w[kOnce];
    int place[kOnce];
#pragma unroll
    for (int r = 0; r < kOnce; ++r) {
      const int i = i0 + r * kTsThreads;
      place[r] = i < n * kTsUnroll ? sh.seen[i / kTsUnroll] + i % kTsUnroll * kTsThreads : vectors;
      w[r] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
      if (place[r] < vectors) w[r] = __ldg(src + place[r]);
    }
#pragma unroll
    for (int r = 0; r < kOnce; ++r)
      if (E::largest(w[r]) >= floor_x) {
#pragma unroll
        for (int e = 0; e < E::kPer; ++e) add(E::get(w[r], e), first + place[r] * E::kPer + e);
      }
  }
  __syncthreads();
}

// The list of a block's elements [lo, hi) from the beginning, for any order of them; every thread calls.
template <int kType>
__device__ __noinline__ void list_again(TsShared& sh, int k, const unsigned char* x0, const uint4* src, int lo, int hi, int first,
                                        int vectors, int behind) {
  using E = TsType<kType>;
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid == 0) { sh.count = 0; sh.floor = 0; }
  __syncthreads();
  // (a round more than there are vectors to go through: the elements in front and behind)
  for (int at = -kTsThreads; at < vectors; at += kTsThreads) {
    uint4 w = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
    int token = first + (at + tid) * E::kPer;
    uint32_t wait = 0;
    if (at < 0) {
      const int one = tid < first - lo ? lo + tid : tid >= 32 && tid - 32 < hi - behind ? behind + tid - 32 : -1;
      if (one >= 0) {
        const float x = E::one(x0 + (long long)one * E::kBytes);
        w.x = kType == kTsF32 ? __float_as_uint(x) : pack16<kType == kTsBf16>(x, x);
        token = one;
        wait = 1;
      }
    } else if (at + tid < vectors) {
      w = ld_stream16(src + at + tid);
      wait = (2u << (E::kPer - 1)) - 1u;
    }
    for (;;) {
      const u64 floor = sh.floor;
#pragma unroll
      for (int e = 0; e < E::kPer; ++e) {
        const float x = E::get(w, e);
        const u64 key = x == x ? pack_candidate(x, token + e) : 0ull;
        if (key <= floor) wait &= ~(1u << e);
        if (wait >> e & 1u) {
          const int to = atomicAdd(&sh.count, 1);
          if (to < kTsList) {
            sh.list[to] = key;
            wait &= ~(1u << e);
          }
        }
      }
      if (!__syncthreads_or(wait != 0)) break;
      cut_list(sh, kTsList, k);
    }
  }
}

}  // namespace

template <int kType, bool kTop>
__global__ void __launch_bounds__(kTsThreads, 4)
token_scores_kernel(const TsArgs a, int parts) {
  using E = TsType<kType>;
  __shared__ TsShared sh;
  pdl_enter();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = parts > 1 ? blockIdx.x % parts : 0;
  const long long row = blockIdx.x / parts;
  const unsigned char* x0 = a.logits + row * a.row_bytes;
  const int lo = min(rank * a.part, a.vocab), hi = min(lo + a.part, a.vocab);
  // [first, first + vectors * kPer): 16 bytes at a time; the elements in front and behind: one each of the first threads
  const int ahead = (int)((16 - ((uintptr_t)(x0 + (long long)lo * E::kBytes) & 15)) & 15) / E::kBytes;
  const int first = min(lo + ahead, hi), vectors = (hi - first) / E::kPer, behind = first + vectors * E::kPer;
  const uint4* src = reinterpret_cast<const uint4*>(x0 + (long long)first * E::kBytes);
  int single = -1;
  if (tid < first - lo) single = lo + tid;
  else if (tid >= 32 && tid - 32 < hi - behind) single = behind + tid - 32;
  if (kTop && tid == 0) { sh.count = 0; sh.floor = 0; sh.floor_x = -INFINITY; }

  uint4 v[kTsUnroll];
  auto load = [&](uint4 (&to)[kTsUnroll], int at) {
#pragma unroll
    for (int i = 0; i < kTsUnroll; ++i) {
      to[i] = make_uint4(E::kNone, E::kNone, E::kNone, E::kNone);
      if (at + i * kTsThreads + tid < vectors) to[i] = ld_stream16(src + at + i * kTsThreads + tid);
    }
  };
  load(v, 0);
  TsSums t = {-INFINITY, 0.f, 0.f};
  float alone = -INFINITY;
  if (single >= 0) alone = E::one(x0 + (long long)single * E::kBytes);

  float floor_x = -INFINITY;
  int at = 0, again = 0;
  do {
    uint4 next[kTsUnroll];
    load(next, at + kTsUnroll * kTsThreads);
    // ---- sums ----
    float high[kTsUnroll], top = alone;
#pragma unroll
    for (int i = 0; i < kTsUnroll; ++i) {
      high[i] = E::largest(v[i]);
      top = fmaxf(top, high[i]);
    }
    if (top > t.m) {
      const float d = max_nan((t.m - top) * kLog2e, -400.f), f = exp2_approx(d);
      t.e = f * fmaf(t.s, d, t.e);
      t.s *= f;
      t.m = top;
    }
    const float base = t.m == -INFINITY ? 0.f : -t.m;
    {
      const float2 l2 = make_float2(kLog2e, kLog2e), b2 = make_float2(base, base);
      float2 s = make_float2(0.f, 0.f), e = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < E::kAll; i += 2) {
        const uint4& w = v[i / E::kPer];
        const float2 z = mul2(add2(make_float2(E::get(w, i % E::kPer), E::get(w, i % E::kPer + 1)), b2), l2);
        const float2 p = make_float2(exp2_approx(z.x), exp2_approx(z.y));
        s = add2(s, p);
        e = fma2(p, z, e);
      }
      if (!(e.x + e.y > -INFINITY)) {                    // 0 times -inf, or something is NaN: again, with care
        s = e = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int i = 0; i < kTsUnroll; ++i) {
          uint4 w = v[0];
#pragma unroll
          for (int j = 1; j < kTsUnroll; ++j)
            if (j == i) w = v[j];
#pragma unroll
          for (int k = 0; k < E::kPer; ++k) {
            const float z = max_nan((E::get(w, k) + base) * kLog2e, -400.f), p = exp2_approx(z);     // (2^-400 is 0)
            s.x += p;
            e.x = fmaf(p, z, e.x);
          }
        }
      }
      t.s += s.x + s.y;
      t.e += e.x + e.y;
      if (single >= 0) {
        const float z = max_nan((alone + base) * kLog2e, -400.f), p = exp2_approx(z);
        t.s += p;
        t.e = fmaf(p, z, t.e);
      }
    }
    // ---- the k best ----
    if (kTop) {
      if (at == again && (at == 0 || vectors - at > at / 2)) {     // (a floor for little that is left does not pay)
        again = 2 * (at + kTsUnroll * kTsThreads);
        raise_floor(sh, t.m, a.k);
        floor_x = sh.floor_x;
      }
      if (top >= floor_x) {
        const int to = atomicAdd(&sh.count, 1);
        if (to < kTsList) sh.seen[to] = at + tid;
      }
    }
    single = -1;
    alone = -INFINITY;
    at += kTsUnroll * kTsThreads;
#pragma unroll
    for (int i = 0; i < kTsUnroll; ++i) v[i] = next[i];
  } while (at < vectors);

  // ---- joined: threads, warps, blocks ----
  const float own = t.m;
  {
    float m = own;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    t = brought_to(t, m);
    t.s = warp_sum(t.s);
    t.e = warp_sum(t.e);
  }
  if (lane == 0) sh.sums[warp] = t;
  __syncthreads();
  if (kTop) {
    const int lone = tid < first - lo ? lo + tid : tid >= 32 && tid - 32 < hi - behind ? behind + tid - 32 : -1;
    int n = sh.count;                                    // (all that follows has a barrier before its first change)
    if (n <= kTsList) {
      collect<kType>(sh, n, own, a.k, x0, first, vectors, lone);
      n = sh.count;
    }
    if (n > kTsList || n < min(a.k, hi - lo)) list_again<kType>(sh, a.k, x0, src, lo, hi, first, vectors, behind);
    // (short lists of a row's blocks are cut together)
    if (parts == 1 || sh.count * parts > kTsThreads) cut_list(sh, sh.count, a.k);
  }
  t = sh.sums[0];
#pragma unroll
  for (int w = 1; w < kTsWarps; ++w) t = joined(t, sh.sums[w]);
  if (parts > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    __syncthreads();
    if (tid == 0) sh.sums[0] = t;
    cluster.sync();
    if (rank == 0) {
      for (int p = 1; p < parts; ++p) t = joined(t, cluster.map_shared_rank(&sh, p)->sums[0]);
      if (kTop) {                                        // of at most kTsList / kTsMaxParts each
        int n = sh.count;
        for (int p = 1; p < parts; ++p) {
          const TsShared* other = cluster.map_shared_rank(&sh, p);
          const int more = other->count;
          for (int i = tid; i < more; i += kTsThreads) sh.list[n + i] = other->list[i];
          n += more;
        }
        __syncthreads();
        cut_list(sh, n, a.k);
      }
    }
    cluster.sync();                                      // (nobody leaves while its shared memory is read)
    if (rank != 0 || warp != 0) return;
  } else if (warp != 0) {
    return;
  }
  // ---- out: warp 0 of the row's first block ----
  const bool empty = t.m == -INFINITY && t.s == 0.f;     // every logit is -inf
  const float ls = log2f(t.s);
  if (lane == 0) {
    if (a.lse) a.lse[row] = empty ? -INFINITY : fmaf(ls, kTsLn2, t.m);
    if (a.entropy) a.entropy[row] = empty ? 0.f : (ls - t.e / t.s) * kTsLn2;
  }
  auto logp = [&](float x) {
    if (empty || x == -INFINITY) return t.s == t.s ? -INFINITY : t.s;
    return fmaf(ls, -kTsLn2, x - t.m);
  };
  for (int i = lane; i < a.n_tokens; i += 32) {
    const int tok = a.tokens[row * a.n_tokens + i];
    const bool is = tok >= 0 && tok < a.vocab;
    a.logp[row * a.n_tokens + i] = is ? logp(E::one(x0 + (long long)tok * E::kBytes)) : -INFINITY;
  }
  if (kTop)
    for (int i = lane; i < a.k; i += 32) {
      const u64 key = i < sh.count ? sh.list[i] : 0ull;
      a.top_id[row * a.k + i] = key ? candidate_row(key) : -1;
      a.top_logp[row * a.k + i] = key ? logp(candidate_score(key)) : -INFINITY;
    }
}

namespace {

template <int kType, bool kTop>
cudaError_t run_scores(const TsArgs& a, int rows, int parts, cudaStream_t st) {
  return launch_cluster(token_scores_kernel<kType, kTop>, (unsigned)rows * (unsigned)parts, kTsThreads, 0, parts, st, a, parts);
}
template <int kType>
cudaError_t run_type(TsArgs a, int rows, int sms, cudaStream_t st) {
  // Blocks: four an SM.  A row is cut while its parts still fill a block's loads twice and all
  // blocks run at once.
  int parts = 1;
  const long long bytes = (long long)a.vocab * TsType<kType>::kBytes;
  while (parts < kTsMaxParts && (long long)rows * parts * 2 <= 4LL * sms && bytes / (parts * 2) >= 2 * 16 * kTsUnroll * kTsThreads) parts *= 2;
  a.part = (a.vocab + parts - 1) / parts;
  return a.k > 0 ? run_scores<kType, true>(a, rows, parts, st) : run_scores<kType, false>(a, rows, parts, st);
}

thread_local char g_scores_err[256] = "";
int refuse(const char* why) {
  snprintf(g_scores_err, sizeof g_scores_err, "%s", why);
  return OILBIRD_EINVAL;
}
int fail(cudaError_t e, const char* what) {
  snprintf(g_scores_err, sizeof g_scores_err, "%s: %s", what, cudaGetErrorString(e));
  return e == cudaErrorMemoryAllocation ? OILBIRD_ENOMEM : OILBIRD_ECUDA;
}
bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
struct Back {                          // the caller's device, current again behind the call
  int before = -1;
  ~Back() { if (before >= 0) cudaSetDevice(before); }
};

}  // namespace

cudaError_t preload_token_scores_kernels() {
  cudaError_t e;
  if ((e = preload_kernel(token_scores_kernel<kTsBf16, false>)) != cudaSuccess) return e;
  if ((e = preload_kernel(token_scores_kernel<kTsBf16, true>)) != cudaSuccess) return e;
  if ((e = preload_kernel(token_scores_kernel<kTsF16, false>)) != cudaSuccess) return e;
  if ((e = preload_kernel(token_scores_kernel<kTsF16, true>)) != cudaSuccess) return e;
  if ((e = preload_kernel(token_scores_kernel<kTsF32, false>)) != cudaSuccess) return e;
  return preload_kernel(token_scores_kernel<kTsF32, true>);
}

}  // namespace oilbird

using namespace oilbird;

extern "C" {

const char* oilbird_token_scores_error(void) { return g_scores_err; }

int oilbird_token_scores(const void* logits, int64_t row_stride, int32_t rows, int32_t vocab, int32_t dtype,
                         const int32_t* tokens, int32_t n_tokens, int32_t k, const oilbird_scores_out* out,
                         int32_t device, void* cuda_stream) {
  if (dtype != kTsBf16 && dtype != kTsF16 && dtype != kTsF32) return refuse("dtype: OILBIRD_LOGITS_BF16, _F16 or _F32");
  if (rows < 0 || rows > (1 << 24)) return refuse("rows: 0 to 2^24");
  if (vocab < 1 || vocab > OILBIRD_SCORES_MAX_VOCAB) return refuse("vocab: 1 to OILBIRD_SCORES_MAX_VOCAB");
  if (k < 0 || k > OILBIRD_SCORES_MAX_TOP) return refuse("k: 0 to OILBIRD_SCORES_MAX_TOP");
  if (n_tokens < 0 || n_tokens > (1 << 20)) return refuse("n_tokens: 0 to 2^20");
  const int size = dtype == kTsF32 ? 4 : 2;
  if (rows > 1 && (row_stride < 0 || row_stride > (1LL << 40))) return refuse("row_stride: 0 to 2^40");
  if (!out) return refuse("no out");
  if (rows == 0) return OILBIRD_OK;
  if (!logits || !aligned(logits, size)) return refuse("logits: aligned to their elements");
  if (n_tokens > 0 && (!tokens || !out->logp)) return refuse("tokens and logp: neither may be missing");
  if (k > 0 && (!out->top_id || !out->top_logp)) return refuse("top_id and top_logp: neither may be missing");
  for (const void* p : {(const void*)tokens, (const void*)out->logp, (const void*)out->lse, (const void*)out->entropy,
                        (const void*)out->top_id, (const void*)out->top_logp})
    if (!aligned(p, 4)) return refuse("tokens and results: 4-byte aligned");
  if (device < 0 || device >= 64) return refuse("device");
  static std::atomic<int> count[64];
  Back back;
  int current = -1;
  if (cudaGetDevice(&current) != cudaSuccess || current != device) {
    const cudaError_t e = cudaSetDevice(device);
    if (e != cudaSuccess) return fail(e, "cudaSetDevice");
    back.before = current;
  }
  int sms = count[device].load(std::memory_order_acquire);
  if (sms == 0) {
    cudaError_t e = preload_all_kernels();
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return fail(e, "loading the library's kernels");
    count[device].store(sms, std::memory_order_release);
  }
  TsArgs a;
  memset(&a, 0, sizeof a);
  a.logits = (const unsigned char*)logits;
  a.row_bytes = rows > 1 ? row_stride * size : 0;
  a.tokens = tokens;
  a.logp = out->logp;
  a.lse = out->lse;
  a.entropy = out->entropy;
  a.top_id = out->top_id;
  a.top_logp = out->top_logp;
  a.vocab = vocab;
  a.n_tokens = n_tokens;
  a.k = k;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = dtype == kTsBf16 ? run_type<kTsBf16>(a, rows, sms, st)
                        : dtype == kTsF16 ? run_type<kTsF16>(a, rows, sms, st) : run_type<kTsF32>(a, rows, sms, st);
  return e == cudaSuccess ? OILBIRD_OK : fail(e, "launch");
}

}  // extern "C"
