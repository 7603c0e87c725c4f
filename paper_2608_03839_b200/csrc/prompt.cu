// C-ABI of the operators over whole prompts: argument checks and dispatch.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <atomic>
#include <initializer_list>

#include "prompt.cuh"

using namespace oilbird;

// One per device: how often a wait ran out, and the limit of the waits.
static __device__ DeviceStats g_prompt_stats;

static thread_local char g_prompt_err[256] = "";
static int refuse(const char* why) {
  snprintf(g_prompt_err, sizeof g_prompt_err, "%s", why);
  return OILBIRD_EINVAL;
}
static int fail(cudaError_t e, const char* what) {
  snprintf(g_prompt_err, sizeof g_prompt_err, "%s: %s", what, cudaGetErrorString(e));
  return e == cudaErrorMemoryAllocation ? OILBIRD_ENOMEM : OILBIRD_ECUDA;
}
#define PCU(call)                                         \
  do {                                                    \
    cudaError_t e_ = (call);                              \
    if (e_ != cudaSuccess) return fail(e_, #call);        \
  } while (0)
#define PTRY(call)                          \
  do {                                      \
    const int r_ = (call);                  \
    if (r_ != OILBIRD_OK) return r_;        \
  } while (0)

static bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// The device made current for a call, and the caller's again behind it.
namespace {
struct OnDevice {
  int before = -1, device;
  explicit OnDevice(int d) : device(d) {}
  ~OnDevice() { if (before >= 0 && before != device) cudaSetDevice(before); }
  int enter(int* sms, DeviceStats** stats) {
    static std::atomic<int> count[64];
    static std::atomic<DeviceStats*> where[64];
    if (device < 0 || device >= 64) return refuse("device");
    if (cudaGetDevice(&before) != cudaSuccess) before = -1;
    if (before != device) PCU(cudaSetDevice(device));
    int n = count[device].load(std::memory_order_acquire);
    if (n == 0) {
      PCU(preload_all_kernels());
      void* p = nullptr;
      PCU(cudaGetSymbolAddress(&p, g_prompt_stats));
      PCU(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device));
      where[device].store((DeviceStats*)p, std::memory_order_relaxed);
      count[device].store(n, std::memory_order_release);
    }
    *sms = n;
    *stats = where[device].load(std::memory_order_relaxed);
    return OILBIRD_OK;
  }
};
}  // namespace

static int check_side(const oilbird_prompt_side& s, const char* what, PromptSide* out) {
  if (s.rows < 0 || s.rows > 2147483648LL - 1024 || !aligned(s.first, 4) || !aligned(s.count, 4)) {
    snprintf(g_prompt_err, sizeof g_prompt_err, "%s: 0 to 2^31 - 1024 rows, first and count 4-byte aligned", what);
    return OILBIRD_EINVAL;
  }
  out->first = s.first;
  out->count = s.first ? nullptr : s.count;
  out->rows = (int)s.rows;
  return OILBIRD_OK;
}
static int check_prompt(const oilbird_prompt* p, PromptArgs* a) {
  if (!p) return refuse("no prompt");
  if (p->head_dim != 64 && p->head_dim != 128) return refuse("head_dim: 64 or 128");
  if (p->dtype != OILBIRD_KV_BF16 && p->dtype != OILBIRD_KV_F16) return refuse("dtype: OILBIRD_KV_BF16 or OILBIRD_KV_F16");
  if (p->n_seq < 1 || p->n_seq > OILBIRD_KV_MAX_SEQ) return refuse("n_seq: 1 to OILBIRD_KV_MAX_SEQ");
  if (p->n_kv_heads < 1 || p->n_kv_heads > 1024) return refuse("n_kv_heads: 1 to 1024");
  if (p->n_q_heads < 1 || p->n_q_heads % p->n_kv_heads || p->n_q_heads / p->n_kv_heads > OILBIRD_KV_MAX_GROUP)
    return refuse("n_q_heads: a multiple of n_kv_heads, OILBIRD_KV_MAX_GROUP times as many at most");
  memset(a, 0, sizeof *a);
  PTRY(check_side(p->q, "query rows", &a->qs));
  PTRY(check_side(p->k, "key rows", &a->ks));
  a->n_seq = p->n_seq;
  a->n_kv = p->n_kv_heads;
  a->group = p->n_q_heads / p->n_kv_heads;
  a->pack = a->group & -a->group;
  while (1 << a->log_pack < a->pack) ++a->log_pack;
  return OILBIRD_OK;
}
// The stride of an extent of one is never used, so it may be anything; a packed side has no sequences.
static int check_rows(const oilbird_kv_rows* r, const char* what, const PromptSide& side, int n_seq, int heads, KvRows* out) {
  const bool seqs = !side.first && n_seq > 1;
  if (!r || (!r->data && side.rows > 0)) {
    snprintf(g_prompt_err, sizeof g_prompt_err, "%s is missing", what);
    return OILBIRD_EINVAL;
  }
  out->p = (const uint16_t*)r->data;
  out->seq = seqs ? r->seq_stride : 0;
  out->row = side.rows > 1 ? r->row_stride : 0;
  out->head = heads > 1 ? r->head_stride : 0;
  constexpr int64_t kFar = 1LL << 39;                    // bytes are counted in 40 bits
  for (const int64_t s : {(int64_t)out->seq, (int64_t)out->row, (int64_t)out->head})
    if (!aligned(r->data, 16) || s % 8 || s < 0 || s >= kFar) {
      snprintf(g_prompt_err, sizeof g_prompt_err,
               "%s: 16-byte aligned, with strides that are multiples of 8 elements, not negative and below 2^39", what);
      return OILBIRD_EINVAL;
    }
  return OILBIRD_OK;
}
static int check_scale(float scale, PromptArgs* a) {
  if (!(fabsf(scale) < INFINITY)) return refuse("scale: a finite number");
  // (never zero, as zero times the -inf of what a row does not see is NaN; scores times fp32's smallest number are)
  a->factor = fminf(fmaxf(fabsf(scale) * kLog2e, 1.5e-45f), 3e38f);
  a->negate = scale < 0.f;
  return OILBIRD_OK;
}
static void lse_layout(const oilbird_prompt* p, const int64_t* strides, PromptArgs* a) {
  a->lse_seq = p->q.first ? 0 : strides ? strides[0] : p->q.rows * p->n_q_heads;
  a->lse_row = strides ? strides[1] : p->n_q_heads;
  a->lse_head = strides ? strides[2] : 1;
}

extern "C" {

const char* oilbird_prompt_last_error(void) { return g_prompt_err; }

int oilbird_prompt_attend(const oilbird_prompt* prompt, const oilbird_kv_rows* q, const oilbird_kv_rows* k,
                          const oilbird_kv_rows* v, float scale, const oilbird_kv_rows* out, float* lse,
                          const int64_t* lse_strides, void* cuda_stream) {
  PromptArgs a;
  KvRows o;
  PTRY(check_prompt(prompt, &a));
  PTRY(check_rows(q, "q", a.qs, a.n_seq, prompt->n_q_heads, &a.q));
  PTRY(check_rows(out, "out", a.qs, a.n_seq, prompt->n_q_heads, &o));
  PTRY(check_rows(k, "k", a.ks, a.n_seq, a.n_kv, &a.k));
  PTRY(check_rows(v, "v", a.ks, a.n_seq, a.n_kv, &a.v));
  PTRY(check_scale(scale, &a));
  if (!aligned(lse, 4)) return refuse("lse: 4-byte aligned");
  if (a.qs.rows == 0) return OILBIRD_OK;
  a.out = (uint16_t*)o.p;
  a.out_seq = o.seq;
  a.out_row = o.row;
  a.out_head = o.head;
  a.lse = lse;
  lse_layout(prompt, lse_strides, &a);
  OnDevice dev(prompt->device);
  int sms;
  PTRY(dev.enter(&sms, &a.stats));
  a.wait_limit = &a.stats->wait_limit_ns;
  const cudaError_t e = launch_prompt_attend(a, prompt->head_dim, prompt->dtype == OILBIRD_KV_BF16, sms, (cudaStream_t)cuda_stream);
  if (e == cudaErrorInvalidValue) return refuse("q, k, v: strides that no tensor map takes");
  PCU(e);
  return OILBIRD_OK;
}

int oilbird_prompt_weigh(const oilbird_prompt* prompt, const oilbird_kv_rows* q, const float* lse,
                         const int64_t* lse_strides, const oilbird_kv_rows* k, const float* row_weight, float scale,
                         float* weight, void* cuda_stream) {
  PromptArgs a;
  PTRY(check_prompt(prompt, &a));
  PTRY(check_rows(q, "q", a.qs, a.n_seq, prompt->n_q_heads, &a.q));
  PTRY(check_rows(k, "k", a.ks, a.n_seq, a.n_kv, &a.k));
  PTRY(check_scale(scale, &a));
  if (!aligned(lse, 4) || !aligned(row_weight, 4) || !aligned(weight, 4)) return refuse("lse, row_weight, weight: 4-byte aligned");
  if (a.ks.rows == 0) return OILBIRD_OK;
  if (!weight || (!lse && a.qs.rows > 0)) return refuse("lse and weight: neither may be missing");
  a.lse = const_cast<float*>(lse);
  a.row_weight = row_weight;
  a.weight = weight;
  lse_layout(prompt, lse_strides, &a);
  OnDevice dev(prompt->device);
  int sms;
  PTRY(dev.enter(&sms, &a.stats));
  a.wait_limit = &a.stats->wait_limit_ns;
  const cudaError_t e = launch_prompt_weigh(a, prompt->head_dim, prompt->dtype == OILBIRD_KV_BF16, sms, (cudaStream_t)cuda_stream);
  if (e == cudaErrorInvalidValue) return refuse("q, k: strides that no tensor map takes");
  PCU(e);
  return OILBIRD_OK;
}

int oilbird_prompt_status(int32_t device, void* cuda_stream) {
  OnDevice dev(device);
  int sms;
  DeviceStats *stats, got;
  PTRY(dev.enter(&sms, &stats));
  PCU(cudaMemcpyAsync(&got, stats, sizeof got, cudaMemcpyDeviceToHost, (cudaStream_t)cuda_stream));
  PCU(cudaStreamSynchronize((cudaStream_t)cuda_stream));
  // The device counts on and nothing is cleared (what another stream's call adds meanwhile would be lost); a count beyond
  // the last one reported, by whichever thread, is news.
  static std::atomic<int> reported[64];
  int was = reported[device].load();
  while ((int)((unsigned)got.stalled - (unsigned)was) > 0)
    if (reported[device].compare_exchange_weak(was, got.stalled)) return OILBIRD_ESTALL;
  return OILBIRD_OK;
}

int oilbird_prompt_set_wait_limit(int32_t device, uint64_t limit_ns, void* cuda_stream) {
  OnDevice dev(device);
  int sms;
  DeviceStats* stats;
  PTRY(dev.enter(&sms, &stats));
  // (pageable host memory: the value is taken before the call returns)
  const unsigned long long limit = limit_ns;
  PCU(cudaMemcpyAsync(&stats->wait_limit_ns, &limit, sizeof limit, cudaMemcpyHostToDevice, (cudaStream_t)cuda_stream));
  return OILBIRD_OK;
}

}  // extern "C"
