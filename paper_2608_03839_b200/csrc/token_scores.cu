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
// The k best.  A list in shared memory takes every element above a floor (a composite of value and token, so
// that equal values are in order too).  The floor is at first the k-th best of 64 groups' best elements of what
// the block holds at the moment, so that few pass it, and again where more than half of the threads would add
// to the list (as behind a long run of masked tokens); when the list is full it is sorted and cut to k, and the floor is the k-th.
#include <cooperative_groups.h>
#include <stdio.h>
#include <string.h>

#include <atomic>

#include "kv.cuh"

namespace cg = cooperative_groups;

namespace oilbird {

namespace {

constexpr int kTsThreads = 256, kTsWarps = kTsThreads / 32, kTsUnroll = 4, kTsList = kTsWarps * 64;
constexpr int kTsMaxParts = 8;
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
  u64 list[kTsList], scratch[kTsList];
  u64 floor;
  int count;
  TsSums sums[kTsWarps];
};

template <int kType> struct TsType {
  static constexpr int kBytes = kType == kTsF32 ? 4 : 2, kPer = 16 / kBytes, kAll = kPer * kTsUnroll;
  static constexpr uint32_t kNone = kType == kTsF32 ? 0xff800000u : kType == kTsF16 ? 0xfc00fc00u : 0xff80ff80u;   // -inf
  static __device__ __forceinline__ float get(const uint4 (&v)[kTsUnroll], int i) {         // element i of the thread's
    const uint32_t w = (&v[i / kPer].x)[i % kPer * kBytes / 4];
    if (kType == kTsF32) return __uint_as_float(w);
    return i & 1 ? half_hi<kType == kTsBf16>(w) : half_lo<kType == kTsBf16>(w);
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
__device__ __forceinline__ TsSums joined(const TsSums& a, const TsSums& b) {
  TsSums r;
  r.m = fmaxf(a.m, b.m);
  r.s = r.e = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const TsSums& x = i ? b : a;
    const float d = x.m == r.m ? 0.f : max_nan((x.m - r.m) * kLog2e, -400.f);       // (equal infinities are no distance)
    const float f = exp2_approx(d);
    r.s = fmaf(f, x.s, r.s);
    r.e = fmaf(f, fmaf(x.s, d, x.e), r.e);
  }
  return r;
}
// Sorts the list's first n (at most kTsList) entries and keeps the k best; every thread calls.  Ends with a barrier.
__device__ __forceinline__ void cut_list(TsShared& sh, int n, int k) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  u64 v[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int i = warp * 64 + r * 32 + lane;
    v[r] = i < n ? sh.list[i] : 0ull;
  }
  if (warp * 64 < n || warp == 0) warp_sort_desc<2>(v, lane);
  block_merge_desc<2>(v, sh.scratch, max(1, (n + 63) / 64));
  __syncthreads();
  if (warp == 0) {
    const u64 last = warp_list_get<2>(v, k - 1);
#pragma unroll
    for (int r = 0; r < 2; ++r)
      if (r * 32 + lane < k) sh.list[r * 32 + lane] = v[r];
    if (lane == 0) {
      sh.count = min(n, k);
      if (n >= k) sh.floor = last;
    }
  }
  __syncthreads();
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
  if (kTop && tid == 0) { sh.count = 0; sh.floor = 0; }

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

  int at = 0;
  do {
    uint4 next[kTsUnroll];
    load(next, at + kTsUnroll * kTsThreads);
    // ---- sums ----
    float top = alone;
#pragma unroll
    for (int i = 0; i < E::kAll; ++i) top = fmaxf(top, E::get(v, i));
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
        float2 z = mul2(add2(make_float2(E::get(v, i), E::get(v, i + 1)), b2), l2);
        z.x = max_nan(z.x, -400.f);                      // (2^-400 is 0; so that 0 times z is, too)
        z.y = max_nan(z.y, -400.f);
        const float2 p = make_float2(exp2_approx(z.x), exp2_approx(z.y));
        s = add2(s, p);
        e = fma2(p, z, e);
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
      const int mine = (at + tid) * E::kPer + first;     // the token of the thread's first element
      auto token = [&](int i) { return mine + i / E::kPer * kTsThreads * E::kPer + i % E::kPer; };
      auto key_of = [&](int i) -> u64 {                  // 0: none (behind the row's end, or NaN)
        const float x = E::get(v, i);
        return token(i) < behind && x == x ? pack_candidate(x, token(i)) : 0ull;
      };
      auto key_alone = [&]() -> u64 { return single >= 0 && alone == alone ? pack_candidate(alone, single) : 0ull; };
      __syncthreads();                                   // the floor of the round before; the list's beginning
      u64 floor = sh.floor;
      bool above = floor == 0ull || top >= candidate_score(floor);
      const int many = __syncthreads_count(above);
      if (many > 0) {
        if (many > kTsThreads / 2) {
          // the k-th best of 64 groups' best
          float x = -INFINITY;
          int tok = -1;
#pragma unroll
          for (int i = 0; i < E::kAll; ++i) {            // (tokens ascend: the first of equal ones stays)
            const float y = E::get(v, i);
            if (token(i) < behind && (y > x || (tok < 0 && y == y))) { x = y; tok = token(i); }
          }
          u64 best = tok >= 0 ? pack_candidate(x, tok) : 0ull;
          if (key_alone() > best) best = key_alone();
#pragma unroll
          for (int o = 1; o < 4; o <<= 1) {
            const u64 y = shfl_xor_u64(best, o);
            best = y > best ? y : best;
          }
          if ((lane & 3) == 0) sh.scratch[tid >> 2] = best;
          __syncthreads();
          if (warp == 0) {
            u64 g[2] = {sh.scratch[lane], sh.scratch[32 + lane]};
            warp_sort_desc<2>(g, lane);
            const u64 kth = warp_list_get<2>(g, a.k - 1);
            // (one below: the k-th itself belongs on the list)
            if (lane == 0 && kth > 0ull && kth - 1 > sh.floor) sh.floor = kth - 1;
          }
          __syncthreads();
          floor = sh.floor;
          above = floor == 0ull || top >= candidate_score(floor);
        }
        uint64_t wait = 0;                               // elements above the floor that are not on the list yet
        if (above) {
#pragma unroll
          for (int i = 0; i < E::kAll; ++i) wait |= (uint64_t)(key_of(i) > floor) << i;
          wait |= (uint64_t)(key_alone() > floor) << E::kAll;
        }
        for (;;) {
          if (wait) {
#pragma unroll
            for (int i = 0; i <= E::kAll; ++i)
              if (wait >> i & 1) {
                const int to = atomicAdd(&sh.count, 1);
                if (to < kTsList) {
                  sh.list[to] = i < E::kAll ? key_of(i < E::kAll ? i : 0) : key_alone();
                  wait &= ~(1ull << i);
                }
              }
          }
          if (!__syncthreads_or(wait != 0)) break;
          cut_list(sh, kTsList, a.k);
          floor = sh.floor;
#pragma unroll
          for (int i = 0; i <= E::kAll; ++i)
            if (wait >> i & 1) {
              const u64 key = i < E::kAll ? key_of(i < E::kAll ? i : 0) : key_alone();
              if (key <= floor) wait &= ~(1ull << i);
            }
        }
      }
    }
    single = -1;
    alone = -INFINITY;
    at += kTsUnroll * kTsThreads;
#pragma unroll
    for (int i = 0; i < kTsUnroll; ++i) v[i] = next[i];
  } while (at < vectors);

  // ---- joined: threads, warps, blocks ----
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    TsSums y;
    y.m = __shfl_xor_sync(0xffffffffu, t.m, o);
    y.s = __shfl_xor_sync(0xffffffffu, t.s, o);
    y.e = __shfl_xor_sync(0xffffffffu, t.e, o);
    t = joined(t, y);
  }
  if (lane == 0) sh.sums[warp] = t;
  __syncthreads();
  if (kTop) cut_list(sh, min(sh.count, kTsList), a.k);
  t = sh.sums[0];
#pragma unroll
  for (int w = 1; w < kTsWarps; ++w) t = joined(t, sh.sums[w]);
  if (parts > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    __syncthreads();
    if (tid == 0) sh.sums[0] = t;
    cluster.sync();
    if (rank == 0 && warp == 0) {
      u64 best[2];
      if (kTop) {
#pragma unroll
        for (int r = 0; r < 2; ++r) best[r] = r * 32 + lane < sh.count ? sh.list[r * 32 + lane] : 0ull;
      }
      for (int p = 1; p < parts; ++p) {
        const TsShared* other = cluster.map_shared_rank(&sh, p);
        t = joined(t, other->sums[0]);
        if (kTop) {
          u64 y[2];
          const int n = other->count;
#pragma unroll
          for (int r = 0; r < 2; ++r) y[r] = r * 32 + lane < n ? other->list[r * 32 + lane] : 0ull;
          warp_merge_desc<2>(best, y, lane);
        }
      }
      if (kTop) {
#pragma unroll
        for (int r = 0; r < 2; ++r) sh.list[r * 32 + lane] = best[r];
        if (lane == 0) sh.count = min(a.k, a.vocab);
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
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows * (unsigned)parts);
  cfg.blockDim = dim3(kTsThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  if (parts > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = parts;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (!tl_pdl_off && pdl_process_ok()) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, token_scores_kernel<kType, kTop>, a, parts);
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
