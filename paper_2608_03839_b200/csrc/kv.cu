// C-ABI of the verifier's 4-bit key/value cache: argument checks and dispatch.
#include <stdio.h>
#include <string.h>

#include <atomic>
#include <initializer_list>

#include "kv.cuh"

using namespace oilbird;

static thread_local char g_kv_err[256] = "";
static int kv_refuse(const char* why) {
  snprintf(g_kv_err, sizeof g_kv_err, "%s", why);
  return OILBIRD_EINVAL;
}
static int kv_fail(cudaError_t e, const char* what) {
  snprintf(g_kv_err, sizeof g_kv_err, "%s: %s", what, cudaGetErrorString(e));
  return e == cudaErrorMemoryAllocation ? OILBIRD_ENOMEM : OILBIRD_ECUDA;
}
#define KCU(call)                                         \
  do {                                                    \
    cudaError_t e_ = (call);                              \
    if (e_ != cudaSuccess) return kv_fail(e_, #call);     \
  } while (0)

static bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

static int check_cache(const oilbird_kv_cache* c, KvView* v) {
  if (!c) return kv_refuse("no cache");
  if (c->head_dim != 64 && c->head_dim != 128) return kv_refuse("head_dim: 64 or 128");
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64) return kv_refuse("page_size: 16, 32 or 64");
  if (c->dtype != OILBIRD_KV_BF16 && c->dtype != OILBIRD_KV_F16) return kv_refuse("dtype: OILBIRD_KV_BF16 or OILBIRD_KV_F16");
  if (c->n_seq < 1 || c->n_seq > OILBIRD_KV_MAX_SEQ) return kv_refuse("n_seq: 1 to OILBIRD_KV_MAX_SEQ");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return kv_refuse("n_kv_heads: 1 to 1024");
  if (c->n_pages < 1 || c->n_pages > 2147483647LL) return kv_refuse("n_pages: 1 to 2^31 - 1");
  // (a tile's worth below 2^31, so that slots and tiles can be counted in 32 bits)
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > 2147483648LL - 1024)
    return kv_refuse("max_pages: at least 1, and max_pages * page_size at most 2^31 - 1024");
  if (!c->pages || !c->weight || !c->pos || !c->page_table || !c->seq_len || !c->n_pos || !c->workspace)
    return kv_refuse("an array of the cache is missing");
  if (!aligned(c->pages, 16) || !aligned(c->workspace, 16)) return kv_refuse("pages and workspace: 16-byte aligned");
  if (!aligned(c->weight, 4) || !aligned(c->pos, 4) || !aligned(c->page_table, 4) || !aligned(c->seq_len, 4) ||
      !aligned(c->n_pos, 4))
    return kv_refuse("weight, pos, page_table, seq_len, n_pos: 4-byte aligned");
  if (c->workspace_bytes < oilbird_kv_workspace_bytes(c->head_dim)) return kv_refuse("workspace: oilbird_kv_workspace_bytes() at least");
  v->pages = (unsigned char*)c->pages;
  v->weight = c->weight;
  v->pos = c->pos;
  v->table = c->page_table;
  v->seq_len = c->seq_len;
  v->n_pos = c->n_pos;
  v->work = (unsigned char*)c->workspace;
  v->n_pages = c->n_pages;
  v->n_seq = c->n_seq;
  v->max_pages = c->max_pages;
  v->page_shift = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : 6;
  v->n_kv = c->n_kv_heads;
  return OILBIRD_OK;
}

// n_seq, rows, heads: the extents; the stride of an extent of one is never used, so it may be anything.
static int check_rows(const oilbird_kv_rows* r, const char* what, int n_seq, int rows, int heads, KvRows* out) {
  if (!r || !r->data) return kv_refuse(what);
  out->p = (const uint16_t*)r->data;
  out->seq = n_seq > 1 ? r->seq_stride : 0;
  out->row = rows > 1 ? r->row_stride : 0;
  out->head = heads > 1 ? r->head_stride : 0;
  if (!aligned(r->data, 16) || out->seq % 8 || out->row % 8 || out->head % 8) {
    snprintf(g_kv_err, sizeof g_kv_err, "%s: 16-byte aligned, with strides that are multiples of 8 elements", what);
    return OILBIRD_EINVAL;
  }
  return OILBIRD_OK;
}
// Arrays of 32-bit elements, each of which may be missing.
static int check_words(const char* what, std::initializer_list<const void*> arrays) {
  for (const void* p : arrays)
    if (!aligned(p, 4)) {
      snprintf(g_kv_err, sizeof g_kv_err, "%s: 4-byte aligned", what);
      return OILBIRD_EINVAL;
    }
  return OILBIRD_OK;
}
static int check_mask(const oilbird_kv_cache* c, const uint64_t* mask, int64_t stride, int m) {
  if (mask && (!aligned(mask, 8) || (c->n_seq > 1 && stride != 0 && stride < m)))
    return kv_refuse("mask: 8-byte aligned, m words a sequence at least, or a stride of 0");
  return OILBIRD_OK;
}

// The device, made current, with the library's kernels loaded; its SM count.
static int on_device(int device, int* sms) {
  static std::atomic<int> count[64];
  int n = 0;
  if (device < 0 || device >= 64) return kv_refuse("device");
  int current = -1;                      // (asking is cheaper than setting)
  if (cudaGetDevice(&current) != cudaSuccess || current != device) KCU(cudaSetDevice(device));
  n = count[device].load(std::memory_order_relaxed);
  if (n == 0) {
    KCU(preload_all_kernels());
    KCU(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device));
    count[device].store(n, std::memory_order_relaxed);
  }
  *sms = n;
  return OILBIRD_OK;
}

static int check_heads(const oilbird_kv_cache* c, int32_t n_q_heads, int32_t m) {
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads || n_q_heads / c->n_kv_heads > OILBIRD_KV_MAX_GROUP)
    return kv_refuse("n_q_heads: a multiple of n_kv_heads, OILBIRD_KV_MAX_GROUP times as many at most");
  if (m < 1 || m > OILBIRD_TREE_MAX_NODES) return kv_refuse("nodes per sequence: 1 to OILBIRD_TREE_MAX_NODES");
  return OILBIRD_OK;
}

#define KTRY(call)                          \
  do {                                      \
    const int r_ = (call);                  \
    if (r_ != OILBIRD_OK) return r_;        \
  } while (0)

extern "C" {

const char* oilbird_kv_last_error(void) { return g_kv_err; }

int64_t oilbird_kv_block_bytes(int32_t head_dim, int32_t page_size) {
  if ((head_dim != 64 && head_dim != 128) || (page_size != 16 && page_size != 32 && page_size != 64)) return 0;
  return 2 * (int64_t)kv_part_bytes(head_dim, page_size);
}

size_t oilbird_kv_workspace_bytes(int32_t head_dim) {
  if (head_dim != 64 && head_dim != 128) return 0;
  return kKvPartOff + (size_t)kKvPartRows * (head_dim + 2) * 4;
}

int oilbird_kv_append(const oilbird_kv_cache* cache, const oilbird_kv_rows* k, const oilbird_kv_rows* v, int32_t m,
                      int32_t rows, const int32_t* n_new, const int32_t* select, const float* weight,
                      void* cuda_stream) {
  KvView c;
  KvAppendArgs a;
  memset(&a, 0, sizeof a);
  KTRY(check_cache(cache, &c));
  if (m < 0 || rows < 0 || rows > (1 << 24)) return kv_refuse("m and rows: not negative, rows at most 2^24");
  if (m == 0 || rows == 0) return OILBIRD_OK;
  if (!select && rows > m) return kv_refuse("rows: m at most without select");
  KTRY(check_rows(k, "k", c.n_seq, m, c.n_kv, &a.k));
  KTRY(check_rows(v, "v", c.n_seq, m, c.n_kv, &a.v));
  KTRY(check_words("n_new, select, weight", {n_new, select, weight}));
  a.n_new = n_new;
  a.select = select;
  a.weight = weight;
  a.m = m;
  a.rows = rows;
  int sms;
  KTRY(on_device(cache->device, &sms));
  KCU(launch_kv_append(c, a, cache->head_dim, cache->dtype == OILBIRD_KV_BF16, sms, (cudaStream_t)cuda_stream));
  return OILBIRD_OK;
}

int oilbird_kv_read(const oilbird_kv_cache* cache, int32_t n, const int32_t* start, void* k, void* v,
                    void* cuda_stream) {
  KvView c;
  KTRY(check_cache(cache, &c));
  if (n < 0 || n > (1 << 24)) return kv_refuse("n: 0 to 2^24");
  if (n == 0) return OILBIRD_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return kv_refuse("k and v: 16-byte aligned");
  KTRY(check_words("start", {start}));
  const KvReadArgs a = {(uint16_t*)k, (uint16_t*)v, start, n};
  int sms;
  KTRY(on_device(cache->device, &sms));
  KCU(launch_kv_read(c, a, cache->head_dim, cache->dtype == OILBIRD_KV_BF16, (cudaStream_t)cuda_stream));
  return OILBIRD_OK;
}

int oilbird_kv_attend(const oilbird_kv_cache* cache, int32_t n_q_heads, int32_t m, const oilbird_kv_rows* q,
                      const oilbird_kv_rows* k_new, const oilbird_kv_rows* v_new, const uint64_t* mask,
                      int64_t mask_stride, const int32_t* n_new, float scale, const oilbird_kv_rows* out, float* lse,
                      const int64_t* lse_strides, void* cuda_stream) {
  KvView c;
  KvAttendArgs a;
  KvRows o;
  memset(&a, 0, sizeof a);
  KTRY(check_cache(cache, &c));
  KTRY(check_heads(cache, n_q_heads, m));
  KTRY(check_rows(q, "q", c.n_seq, m, n_q_heads, &a.q));
  KTRY(check_rows(out, "out", c.n_seq, m, n_q_heads, &o));
  if (!k_new != !v_new) return kv_refuse("k_new and v_new: both or neither");
  if (k_new) {
    KTRY(check_rows(k_new, "k_new", c.n_seq, m, c.n_kv, &a.k));
    KTRY(check_rows(v_new, "v_new", c.n_seq, m, c.n_kv, &a.v));
  }
  KTRY(check_mask(cache, mask, mask_stride, m));
  if (!(scale == scale)) return kv_refuse("scale: a number");
  KTRY(check_words("lse, n_new", {lse, n_new}));
  a.out = (uint16_t*)o.p;
  a.out_seq = o.seq;
  a.out_row = o.row;
  a.out_head = o.head;
  a.lse = lse;
  a.lse_seq = lse_strides ? lse_strides[0] : (int64_t)m * n_q_heads;
  a.lse_row = lse_strides ? lse_strides[1] : n_q_heads;
  a.lse_head = lse_strides ? lse_strides[2] : 1;
  a.mask = (const unsigned long long*)mask;
  a.mask_stride = mask_stride;
  a.n_new = n_new;
  a.scale = scale;
  a.m = m;
  a.group = n_q_heads / c.n_kv;
  int sms;
  KTRY(on_device(cache->device, &sms));
  KCU(launch_kv_attend(c, a, cache->head_dim, cache->dtype == OILBIRD_KV_BF16, sms, (cudaStream_t)cuda_stream));
  return OILBIRD_OK;
}

int oilbird_kv_weigh(const oilbird_kv_cache* cache, int32_t n_q_heads, int32_t m, const oilbird_kv_rows* q,
                     const float* lse, const int64_t* lse_strides, const oilbird_kv_rows* k_new, const uint64_t* mask, int64_t mask_stride,
                     const int32_t* n_new, const float* row_weight, float scale, float* node_weight,
                     void* cuda_stream) {
  KvView c;
  KvWeighArgs a;
  memset(&a, 0, sizeof a);
  KTRY(check_cache(cache, &c));
  KTRY(check_heads(cache, n_q_heads, m));
  KTRY(check_rows(q, "q", c.n_seq, m, n_q_heads, &a.q));
  if (!lse) return kv_refuse("lse");
  KTRY(check_words("lse, n_new, row_weight, node_weight", {lse, n_new, row_weight, node_weight}));
  if (!k_new != !node_weight) return kv_refuse("k_new and node_weight: both or neither");
  if (k_new) KTRY(check_rows(k_new, "k_new", c.n_seq, m, c.n_kv, &a.k));
  KTRY(check_mask(cache, mask, mask_stride, m));
  if (!(scale == scale)) return kv_refuse("scale: a number");
  a.node_weight = node_weight;
  a.lse = lse;
  a.lse_seq = lse_strides ? lse_strides[0] : (int64_t)m * n_q_heads;
  a.lse_row = lse_strides ? lse_strides[1] : n_q_heads;
  a.lse_head = lse_strides ? lse_strides[2] : 1;
  a.row_weight = row_weight;
  a.mask = (const unsigned long long*)mask;
  a.mask_stride = mask_stride;
  a.n_new = n_new;
  a.scale = scale;
  a.m = m;
  a.group = n_q_heads / c.n_kv;
  int sms;
  KTRY(on_device(cache->device, &sms));
  KCU(launch_kv_weigh(c, a, cache->head_dim, cache->dtype == OILBIRD_KV_BF16, sms, (cudaStream_t)cuda_stream));
  return OILBIRD_OK;
}

int oilbird_kv_evict(const oilbird_kv_cache* cache, int32_t budget, int32_t sink, int32_t recent, void* cuda_stream) {
  KvView c;
  KTRY(check_cache(cache, &c));
  if (budget < 1 || sink < 0 || recent < 0 || (int64_t)sink + recent > budget)
    return kv_refuse("budget: at least 1, and at least sink + recent");
  if (((int64_t)c.max_pages << c.page_shift) > OILBIRD_KV_MAX_EVICT_SLOTS)
    return kv_refuse("max_pages * page_size: OILBIRD_KV_MAX_EVICT_SLOTS at most");
  const KvEvictArgs a = {budget, sink, recent, 0, 0, 0};
  int sms;
  KTRY(on_device(cache->device, &sms));
  KCU(launch_kv_evict(c, a, cache->head_dim, sms, (cudaStream_t)cuda_stream));
  return OILBIRD_OK;
}

int oilbird_kv_status(const oilbird_kv_cache* cache, int64_t* dropped, void* cuda_stream) {
  KvView c;
  KTRY(check_cache(cache, &c));
  int sms;
  KTRY(on_device(cache->device, &sms));
  KvWork w;
  KCU(cudaMemcpyAsync(&w, c.work, sizeof w, cudaMemcpyDeviceToHost, (cudaStream_t)cuda_stream));
  KCU(cudaStreamSynchronize((cudaStream_t)cuda_stream));
  if (dropped) *dropped = (int64_t)w.dropped;
  return w.stats.stalled ? OILBIRD_ESTALL : OILBIRD_OK;
}

}  // extern "C"
