// Attention over the 4-bit cache for many query rows per key/value head (whole draft trees):
// tensor cores with accumulators in TMEM.
//
// The formulas are those of kv_attend.cu.  With 128 or 256 rows on a tile of 128 slots the
// products decide (4 D flops for each row and slot), so keys and values are turned into f16 once per tile
// and every row of the block uses them.  One block an SM:
//   warps 0-3, 4-7   softmax: one row per thread.  Two groups of 128 rows A and B, or, where the
//                    block has 128 rows or fewer, the same rows twice: A takes the even tiles
//                    and B the odd ones, each with sums of its own.
//   warps 8-11       decode, a slot per thread: codes from global memory (a tile ahead, each
//                    thread's in a place of its own in shared memory), scales and offsets (two
//                    tiles ahead), to f16 in the 128-byte-swizzled layout the products read:
//                    two places for values, one for both parts of the keys
//   warp 12          issues the products: S = Q K^T (from shared memory) and O += P V (P from
//                    TMEM, where the softmax warps put it over the scores); warps 13-15 only
//                    complete its group, which gives the softmax warps its registers: 192 each,
//                    so that a thread holds its row's 128 scores between the maximum and the
//                    exponentials instead of reading them twice
// While A's scores go through the exponentials the tensor core works on B's tile and the other
// way round.  Keys are the product's N operand as they lie (channels contiguous), values the N operand with
// channels contiguous as well (transposed operand), so both have the same layout and neither
// is transposed by hand.
//
// Numbers.  A decoded value is rounded to f16 once (scale * code + lo as one fused multiply-add,
// 2^-11 of it).  Keys are the sum of two f16 numbers (see key_parts), each multiplied with
// the rows: rounded once they left the logarithms off by 2e-5 of themselves over short
// sequences, in fp32 outputs; now it is 2e-7, for 16 % more time on long ones.  Rows are multiplied by a power of two that brings their largest
// element to [1, 2); a cached tile's keys and values likewise by 2^-Ek and 2^-Ev (below 1).  Ek joins the row's factor,
// Ev the exponent: p = exp2(s + Ev - m + 7) with m the running maximum of s + Ev, so that
// O = sum p (2^-Ev v) and l = sum 2^-Ev p carry no unit of their own and m alone keeps every
// operand in range.  (Without the 7, which f16 has room for, 32,768 slots 17.5 below one other
// in exp's units came out as nothing.)  m is brought up to date only when a row passes it by 2^8 (the
// accumulators are rescaled in TMEM then, once a row's maximum has settled never again).  New
// nodes, which not every row sees, share no scale: each key has a power of two of its own, joined to
// its scores where the mask is applied, and their values are multiplied in the cache's type with probabilities as the sum of two numbers of that type (two copies of 64 nodes
// are a tile of 128 slots).
//
// Work.  The list of tiles of kv.cuh with 128 slots a tile, one run per block.  An item that a
// block has to itself is written out by it; the pieces of the others go to the workspace (sums,
// maxima, fp32 accumulators, rows contiguous so that both sides are coalesced) and a second
// kernel joins them in their order: with 256 rows a piece is 133 KB, which all SMs together
// read back in microseconds and one block would not.
//
// Measured, with 60-node trees under 32 query heads, 8 key/value heads of 128: 65,541 slots in
// 102 us (64.4 GFLOP at 630 TFLOP/s; 39 us at the measured bf16 rate), 8 sequences of 2,048 to
// 4,096 slots in 75 us with the join (59 and 25 us each by itself with cold
// caches).  The kernel spills some 200 bytes a thread.  A tile takes about 5,700 cycles, of which the
// exponentials (2,048), the products (3,072 with both parts of the keys) and the shared
// memory they read (3,300) each fill about half: what bounds it is their chain - products,
// exponentials, products - with two groups to overlap and one place for the keys.
//
// Every wait is bounded (two seconds): a wait that runs out raises the workspace's flag, all roles
// leave, TMEM is freed.
#include "kv.cuh"

namespace oilbird {

namespace {

constexpr int kTrTile = 128, kTrFront = 4;               // slots a tile; see TileListOf
constexpr int kTrDecWarps = 4, kTrIssuer = 12, kTrThreads = 512;
// registers a thread: launched with 128; the four warpgroups' shares add up to 4 x 128
constexpr int kTrSoftRegs = 192, kTrDecRegs = 104, kTrIssueRegs = 24;
static_assert(2 * kTrSoftRegs + kTrDecRegs + kTrIssueRegs == 4 * 128, "more registers than the block was launched with");
using TreeList = TileListOf<kTrTile, kTrFront, 0>;
constexpr float kTrLn2 = 0.6931471805599453f;
// Probabilities are f16 operands in units in which a row's largest lies between 2^7 and 2^15: f16
// ends above that, and what is 2^-21 of the largest still has all its bits, 2^-31 one.
constexpr int kTrRoom = 7, kTrSlack = 8;

// ------------------------------------------------------------------ PTX wrappers ---
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(kv_smem(b)), "r"(n));
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(kv_smem(b)) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(kv_smem(b)), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// Bounded wait; false if it gave up or another role did.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* gave_up, DeviceStats* stats) {
  if (bar_try(b, parity)) return true;
  const unsigned long long t0 = now_ns(), limit = wait_limit_ns(stats);
  for (uint32_t spin = 0;; ++spin) {
    if (bar_try(b, parity)) return true;
    if ((spin & 63u) == 63u) {
      if (*gave_up) return false;
      if (now_ns() - t0 > limit) {
        *gave_up = 1;
        atomicExch(&stats->stalled, 1);
        return false;
      }
    }
  }
}
// the same by a converged warp, one outcome for all lanes
__device__ __forceinline__ bool warp_wait(uint64_t* b, uint32_t parity, volatile int* gave_up, DeviceStats* stats) {
  return __all_sync(0xffffffffu, bar_wait(b, parity, gave_up, stats));
}
__device__ __forceinline__ bool one_lane() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(kv_smem(b)) : "memory");
}
// D[tmem] (+)= A[smem] B[smem], 16-bit operands of one type, fp32 accumulators, M = 128, K = 16
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// the same with A from TMEM (two elements a column)
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// 32 columns of the warp's lanes; the values are there after tmem_wait32 on them
__device__ __forceinline__ void tmem_ask32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_wait32(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :: "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&v)[32]) {
  uint32_t r[32];
  tmem_ask32(addr, r);
  tmem_wait32(r);
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// the largest of three
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Matrix in shared memory, rows of 64 f16 (128 bytes), 128-byte swizzle: descriptor of the
// operand that begins at addr.  Rows are the operand's M or N and the row's channels its K: 8-row
// groups 1024 bytes apart.  Rows are its K and channels its N (transposed): the same groups
// along K, and blocks of 64 channels `block` bytes apart.
__device__ __forceinline__ uint64_t desc128(uint32_t addr, uint32_t block) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(block >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// fp32 accumulators, f16 (or bf16) operands, M = 128, N = n; transposed: B's N is contiguous
__device__ __forceinline__ constexpr uint32_t idesc_16(int n, bool transposed, bool bf16) {
  return (1u << 4) | ((uint32_t)bf16 << 7) | ((uint32_t)bf16 << 10) | ((uint32_t)transposed << 16) |
         ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
struct TileInfo {                    // what the softmax warps need to know of a tile
  uint32_t valid[4];                 // slots that exist (cached tiles)
  float key_scale, value_exp, value_scale;   // 2^Ek, Ev, 2^-Ev
  uint8_t flags[4];                  // by decoding warp; 1: new nodes, 2: some slot is not valid, 4: a value is not finite
  alignas(16) int8_t node_exp[64];   // new nodes: the powers of two their keys were divided by
};
struct TreeShared {
  uint64_t kfull, kfree, vfull[2], vfree[2], sfull[2], pfull[2], pvdone[2], info_full[4], qfull;
  uint64_t meet, peaks[2];           // the softmax warps; the decoding warps, by tile parity
  TileInfo info[4];
  uint32_t peak[4][kTrDecWarps][2];  // by tile: largest key and value bound each decoding warp saw
  uint32_t tmem;
  int gave_up;
  float2 ml[128];                    // group B's sums on their way to A
};

template <int D>
struct Tree {
  static constexpr int kBlocks = D / 64, kMat = kBlocks * kTrTile * 128;     // one tile of K or V in f16
  static constexpr int kQMat = kBlocks * 256 * 128;
  static constexpr int kCum = (kKvMaxSeq + 1) * 8 + 16 * 8 + kKvMaxSeq * 5;
  static constexpr int kCodes = kBlocks * 64 + 16;                           // a slot's codes; spread over the banks
  static constexpr int kBytes = 1024 + 4 * kMat + kQMat + kTrTile * kCodes + (int)sizeof(TreeShared) + 16 + kCum;
  static_assert(kBytes <= 227 * 1024, "shared memory");
  // a piece in the workspace: accumulators [group][D / 4][128 rows][4], then (m, l) [group][128 rows]
  static constexpr size_t kPiece = (size_t)2 * 128 * (D + 2);
};

// One piece of an item, as every role sees it.
struct Piece {
  int s, head, row0, n_rows;         // n_rows: the sequence's
  bool two;                          // more than 128 rows: groups A and B have rows of their own
  bool whole;                        // all of the item
  bool nodes;                        // begins with the new nodes' tile
  int c0, n;                         // first cached tile; tiles in all
};
__device__ __forceinline__ Piece piece_at(const TreeList::Cursor& k, int count, const KvView& c, const KvAttendArgs& a) {
  Piece p;
  p.s = k.s;
  p.head = k.head;
  p.row0 = k.item / c.n_kv * 256;
  p.n_rows = k.nodes * a.group;
  p.two = p.n_rows - p.row0 > 128;
  p.whole = k.tile == 0 && count == (k.item < k.live ? k.tiles : 1);
  const bool live = k.item < k.live;
  p.nodes = live && k.tile == 0 && a.k.p && k.nodes > 0;
  const int first = max(k.tile, kTrFront), last = k.tile + count;
  p.c0 = first - kTrFront;
  p.n = (live && last > first ? last - first : 0) + (p.nodes ? 1 : 0);
  return p;
}

// (largest |element| of a group) as float bits; what reads as NaN says nothing
template <bool kBf16> __device__ __forceinline__ uint32_t meta_peak(uint32_t meta) {
  const float sc = half_lo<kBf16>(meta), lo = half_hi<kBf16>(meta);
  const float x = fmaxf(fabsf(lo), fabsf(fmaf(15.f, sc, lo)));
  return x < INFINITY ? __float_as_uint(x) : 0u;
}
// exponent E with peak < 2^E, as far as 2^E and 2^-E are numbers (the largest peaks come to 4, which
// f16 holds) and sums over long sequences times 2^-E stay in range
__device__ __forceinline__ int peak_exp(uint32_t peak) {
  return min(max((int)(peak >> 23) - 126, -90), 126);
}
__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<__half2*>(&w); }
__device__ __forceinline__ uint32_t as_word(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }

// Eight codes (one word, channels in order) -> eight f16 numbers scale * code + lo.
// code + 1024 (or 16 code + 1024) is an f16 number by its bits; both ways back to the code are exact.
__device__ __forceinline__ uint4 decode8(uint32_t w, __half2 sc, __half2 lo) {
  const uint32_t magic = 0x64006400u;
  const __half2 m1024 = __half2half2(__ushort_as_half(0xE400)), r16 = __half2half2(__ushort_as_half(0x2C00)),
                m64 = __half2half2(__ushort_as_half(0xD400));
  const uint32_t v = w >> 8;
  uint4 r;
  r.x = as_word(__hfma2(__hadd2(as_half2((w & 0x000f000fu) | magic), m1024), sc, lo));
  r.y = as_word(__hfma2(__hfma2(as_half2((w & 0x00f000f0u) | magic), r16, m64), sc, lo));
  r.z = as_word(__hfma2(__hadd2(as_half2((v & 0x000f000fu) | magic), m1024), sc, lo));
  r.w = as_word(__hfma2(__hfma2(as_half2((v & 0x00f000f0u) | magic), r16, m64), sc, lo));
  return r;
}

// The same as the sum of two f16 numbers.  With mid = scale * 8 + lo an element is
// scale (code - 8) + mid.  The scale's five leading bits sh and mid to the last of their places,
// mh, make `hi` = sh (code - 8) + mh, which f16 holds exactly while |mid| < 58 scale (a group whose
// middle lies within four times its range); what both left over makes `rest`, below scale / 2
// and off by 2^-13 scale at most.  (Wider off centre, hi is rounded as one f16 number would be.)
struct KeyParts { __half2 sh, sl, mh, ml; };
__device__ __forceinline__ KeyParts key_parts(float scale, float lo) {
  const uint32_t bits = __float_as_uint(scale);
  const float sh = __uint_as_float(bits & 0xfff80000u), sl = scale - sh, mid = fmaf(8.f, scale, lo);
  const float grid = __uint_as_float((bits & 0x7f800000u) + (19u << 23) | 0x400000u);     // sums with it end at sh's last place
  const float m = __fsub_rn(__fadd_rn(mid, grid), grid);
  KeyParts k;
  k.sh = as_half2(pack16<false>(sh, sh));
  k.sl = as_half2(pack16<false>(sl, sl));
  k.mh = as_half2(pack16<false>(m, m));
  const float ml = mid - __low2float(k.mh);
  k.ml = as_half2(pack16<false>(ml, ml));
  return k;
}
__device__ __forceinline__ void decode8_parts(uint32_t w, const KeyParts& k, uint4& hi, uint4& rest) {
  const uint32_t magic = 0x64006400u;
  const __half2 m1032 = __half2half2(__ushort_as_half(0xE408)), r16 = __half2half2(__ushort_as_half(0x2C00)),
                m72 = __half2half2(__ushort_as_half(0xD480));
  const uint32_t v = w >> 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = i < 2 ? w : v;
    const __half2 c = i & 1 ? __hfma2(as_half2((x & 0x00f000f0u) | magic), r16, m72) : __hadd2(as_half2((x & 0x000f000fu) | magic), m1032);
    (&hi.x)[i] = as_word(__hfma2(c, k.sh, k.mh));
    (&rest.x)[i] = as_word(__hfma2(c, k.sl, k.ml));
  }
}

}  // namespace

template <int D, bool kBf16>
__global__ void __launch_bounds__(kTrThreads, 1)
kv_tree_kernel(const KvView c, const KvAttendArgs a) {
  using T = Tree<D>;
  constexpr int G = T::kBlocks;
  extern __shared__ unsigned char raw_smem[];
  unsigned char* smem = raw_smem + ((1024 - (kv_smem(raw_smem) & 1023)) & 1023);
  unsigned char *vmat = smem, *kmat = smem + 2 * T::kMat, *qmat = smem + 4 * T::kMat;
  unsigned char* codes = qmat + T::kQMat;
  TreeShared& sh = *reinterpret_cast<TreeShared*>(codes + kTrTile * T::kCodes);
  long long* cum = reinterpret_cast<long long*>(codes + kTrTile * T::kCodes + (sizeof(TreeShared) + 15) / 16 * 16);
  long long* scratch = cum + kKvMaxSeq + 1;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  DeviceStats* stats = &reinterpret_cast<KvWork*>(c.work)->stats;
  volatile int* gave_up = &sh.gave_up;

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      bar_init(&sh.vfull[i], kTrDecWarps);
      bar_init(&sh.vfree[i], 1);
      bar_init(&sh.sfull[i], 1);
      bar_init(&sh.pfull[i], 4);
      bar_init(&sh.pvdone[i], 1);
      bar_init(&sh.peaks[i], kTrDecWarps);
    }
    for (int i = 0; i < 4; ++i) bar_init(&sh.info_full[i], kTrDecWarps);
    bar_init(&sh.kfull, kTrDecWarps);
    bar_init(&sh.kfree, 1);
    bar_init(&sh.qfull, 8);
    bar_init(&sh.meet, 8);
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kTrIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(kv_smem(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  pdl_enter();

  TreeList list;
  list.cum = cum;
  list.len = reinterpret_cast<int*>(scratch + 16);
  list.nodes = reinterpret_cast<unsigned char*>(list.len + kKvMaxSeq);
  list.items = c.n_kv * ((a.m * a.group + 255) / 256);
  list.group = a.group;
  list.rows = 256;
  list.build<kTrThreads>(c, a.n_new, a.m, scratch);
  const int n_cta = (int)min((long long)gridDim.x, list.total);
  TreeList::Cursor bc, scrap;
  int u1 = 0;
  if ((int)blockIdx.x < n_cta) {
    const long long end = list.cut(scrap, blockIdx.x + 1, n_cta), begin = list.cut(bc, blockIdx.x, n_cta);
    u1 = (int)(end - begin);
  }
  const int block_bytes = 2 * kv_part_bytes(D, 1 << c.page_shift);
  const int page = 1 << c.page_shift;

  if (warp < 8) {
    // ============================================================ softmax ========
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTrSoftRegs));
    const int wg = warp >> 2, row = tid & 127;           // row of the group
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;   // TMEM lanes of this warp
    const uint32_t s_tm = tmem + lanes + wg * 256, o_tm = s_tm + 128;
    uint32_t kt = 0, su = 0, met = 0;                    // tiles, score tiles of the group, meetings so far
    bool ok = true;
    auto meet = [&]() {                                  // of both groups
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.meet);
      ok = ok && warp_wait(&sh.meet, met++ & 1, gave_up, stats);
      return ok;
    };
    for (int at = 0; at < u1 && ok;) {
      const int n_tiles = bc.item < bc.live ? bc.tiles : 1, count = min(n_tiles - bc.tile, u1 - at);
      const Piece p = piece_at(bc, count, c, a);
      float m = -INFINITY, l = 0.f;
      bool odd_values = false;                           // new nodes' values that are not finite
      const int my_row = p.row0 + (p.two ? wg * 128 : 0) + row;
      const bool have = my_row < p.n_rows;
      const int node = have ? my_row / a.group : 0;
      // (both groups have left the piece before: its scores, its accumulators and its Q are free)
      if (!meet()) break;
      if (p.n > 0) {
        // ---- the row as an operand ----
        // Raw rows are copied to where their f16 will lie (16 bits either way), whole lines at a
        // time, and turned into f16 in place.  Short loops throughout: this code runs once a
        // piece, and fetching straight-line code took longer than the work.  (Group B copies
        // the rows for itself even where A's are the operand: it needs their exponents.)
        unsigned char* my_q = qmat + (wg * 128 + row) * 128;
        {
          // rows are walked by steps: a division for each would take longer than its copy
          constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
          const int chunk = lane % kLanes, first = (warp & 3) * 32 + lane / kLanes;
          int gr = p.row0 + (p.two ? wg * 128 : 0) + first, nd = gr / a.group, sb = gr - nd * a.group;
          unsigned char* dst = qmat + (chunk >> 3) * (256 * 128) + (wg * 128 + first) * 128;
          const uint16_t* src = a.q.at(p.s, 0, p.head * a.group) + chunk * 8;
#pragma unroll 2
          for (int i = 0; i < 32 / kAtOnce; ++i) {
            const bool in = gr < p.n_rows;
            cp_async16(kv_smem(dst + i * kAtOnce * 128 + (((chunk & 7) ^ ((first + i * kAtOnce) & 7)) << 4)),
                       in ? src + nd * a.q.row + sb * a.q.head : src, in ? 16 : 0);
            gr += kAtOnce;
            for (sb += kAtOnce; sb >= a.group; sb -= a.group) ++nd;
          }
        }
        cp_async_commit();
        cp_async_wait<0>();
        __syncwarp();
        float top = 0.f;
#pragma unroll 2
        for (int i = 0; i < D / 8; ++i) {
          const uint4 w = *reinterpret_cast<const uint4*>(my_q + (i >> 3) * (256 * 128) + (((i & 7) ^ (row & 7)) << 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t x = (&w.x)[e];
            top = abs_max(abs_max(top, half_lo<kBf16>(x)), half_hi<kBf16>(x));
          }
        }
        const int e0 = top < INFINITY ? min(row_exponent(top), 126) : 0;
        const float up = a.scale < 0.f ? -pow2(-e0) : pow2(-e0);
        const float f = fmaxf(fabsf(a.scale) * kLog2e * pow2(e0), 1e-37f);
#pragma unroll 2
        for (int i = 0; i < D / 8; ++i) {
          uint4* at_chunk = reinterpret_cast<uint4*>(my_q + (i >> 3) * (256 * 128) + (((i & 7) ^ (row & 7)) << 4));
          uint4 w = *at_chunk;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t x = (&w.x)[e];
            (&w.x)[e] = pack16<false>(half_lo<kBf16>(x) * up, half_hi<kBf16>(x) * up);
          }
          *at_chunk = w;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.qfull);
        const unsigned long long sees =
            !have ? 0ull : a.mask ? a.mask[p.s * a.mask_stride + node] : (2ull << node) - 1ull;

        // ---- tile by tile ----
        const int mine = p.two ? p.n : (p.n + 1 - wg) / 2;
        for (int i = 0; i < mine; ++i, ++su) {
          const uint32_t t = kt + (p.two ? i : 2 * i + wg);
          if (!warp_wait(&sh.info_full[t & 3], (t >> 2) & 1, gave_up, stats) ||
              !warp_wait(&sh.sfull[wg], su & 1, gave_up, stats)) { ok = false; break; }
          fence_after();
          const TileInfo& info = sh.info[t & 3];
          uint32_t flags = *reinterpret_cast<const uint32_t*>(info.flags);
          flags |= flags >> 16;
          flags |= flags >> 8;
          // (never zero, as f is not: zero times the -inf of what the row does not see is NaN; rows and
          // keys this small have scores of zero either way.  Nor infinite: times a score of zero that
          // is NaN too.)
          const float g = fminf(fmaxf(f * info.key_scale, 1e-37f), 3e38f), ev = info.value_exp;
          // which slots count for this row
          uint32_t see[4];
          if (flags & 1) {
            see[0] = (uint32_t)sees & info.valid[0];
            see[1] = (uint32_t)(sees >> 32) & info.valid[1];
            see[2] = see[3] = 0u;
            odd_values |= (flags & 4) != 0;
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) see[k] = info.valid[k];
          }
          const bool masked = __any_sync(0xffffffffu, flags & 3);
          const bool nodes = __any_sync(0xffffffffu, flags & 1);
          if (masked) {                                  // -inf where the row does not look
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
              uint32_t r[16];
              tmem_ld16(s_tm + k * 16, r);
              const uint32_t b = (k < 2 ? see[0] : k < 4 ? see[1] : k < 6 ? see[2] : see[3]) >> (k & 1 ? 16 : 0);
              uint4 ex = make_uint4(0, 0, 0, 0);
              if (nodes && k < 4) ex = *reinterpret_cast<const uint4*>(info.node_exp + k * 16);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float up = pow2((int)(int8_t)((&ex.x)[e >> 2] >> (8 * (e & 3))));
                r[e] = b >> e & 1 ? __float_as_uint(__uint_as_float(r[e]) * up) : 0xff800000u;
              }
              tmem_st16(s_tm + k * 16, r);
            }
            tmem_wait_st();
          }
          uint32_t x[128];                               // the row's scores
#pragma unroll
          for (int k = 0; k < 4; ++k) tmem_ask32(s_tm + k * 32, x + k * 32);
#pragma unroll
          for (int k = 0; k < 4; ++k) tmem_wait32(x + k * 32);
          float y[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 64; ++e) y[e & 3] = max3(y[e & 3], __uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1]));
          float mx = fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]));
          mx = fmaf(mx, g, ev);
          if (__any_sync(0xffffffffu, mx > m + kTrSlack)) {
            // (each row for itself: what its warp's other rows look at changes nothing)
            const float mn = mx > m + kTrSlack ? mx : m, down = mn == -INFINITY ? 1.f : exp2_approx(m - mn);
            m = mn;
            l *= down;
            if (i > 0) {
              if (!warp_wait(&sh.pvdone[wg], (su - 1) & 1, gave_up, stats)) { ok = false; break; }
              fence_after();
#pragma unroll 1
              for (int k = 0; k < D; k += 16) {
                uint32_t r[16];
                tmem_ld16(o_tm + k, r);
#pragma unroll
                for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * down);
                tmem_st16(o_tm + k, r);
              }
            }
          }
          const float shift = ev + kTrRoom - (m == -INFINITY ? 0.f : m);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float2 g2 = make_float2(g, g), shift2 = make_float2(shift, shift);
          if (nodes) {
            // the cache's own type, as the nodes' values are: leading parts, then their rests, which
            // meet the values' second copy
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint32_t w[16], rest[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int i2 = k * 32 + 2 * e;
                const float2 z = fma2(make_float2(__uint_as_float(x[i2]), __uint_as_float(x[i2 + 1])), g2, shift2);
                const float2 pr = make_float2(exp2_approx(z.x), exp2_approx(z.y));
                sum[e & 1] = add2(sum[e & 1], pr);
                w[e] = pack16<kBf16>(pr.x, pr.y);
                rest[e] = pack16<kBf16>(pr.x - half_lo<kBf16>(w[e]), pr.y - half_hi<kBf16>(w[e]));
              }
              tmem_st16(s_tm + k * 16, w);               // over the scores
              tmem_st16(s_tm + 32 + k * 16, rest);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t w[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int i2 = k * 32 + 2 * e;
                const float2 z = fma2(make_float2(__uint_as_float(x[i2]), __uint_as_float(x[i2 + 1])), g2, shift2);
                const float2 pr = make_float2(exp2_approx(z.x), exp2_approx(z.y));
                sum[e & 1] = add2(sum[e & 1], pr);
                w[e] = pack16<false>(pr.x, pr.y);
              }
              tmem_st16(s_tm + k * 16, w);               // over the scores
            }
          }
          sum[0] = add2(sum[0], sum[1]);
          l = fmaf(sum[0].x + sum[0].y, info.value_scale, l);
          tmem_wait_st();
          fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(&sh.pfull[wg]);
        }
        if (!ok) break;
        kt += p.n;
        if (mine > 0) {
          if (!warp_wait(&sh.pvdone[wg], (su - 1) & 1, gave_up, stats)) { ok = false; break; }
          fence_after();
        }
        if (mine == 0) { m = -INFINITY; l = 0.f; }
        m -= kTrRoom;                                    // what l and the accumulators are relative to
      }
      // A thread's 32 accumulators from column k on.  Infinities and NaN of new nodes' values
      // stayed out of the products (0 times a hidden node's would have reached every row): they
      // are added to the rows that see them.
      const bool any = p.n > (p.two ? 0 : wg);           // the group has accumulators
      auto accumulators = [&](int k, float (&x)[32]) {
        tmem_ld32(o_tm + k, x);
        if (odd_values && have) {
          const unsigned long long sees = a.mask ? a.mask[p.s * a.mask_stride + node] : (2ull << node) - 1ull;
          for (int j = 0; j < bc.nodes; ++j)
            if (sees >> j & 1ull) {
              const uint16_t* vp = a.v.at(p.s, j, p.head) + k;
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(vp + 2 * e);
                const float v0 = half_lo<kBf16>(w), v1 = half_hi<kBf16>(w);
                if (!(fabsf(v0) < INFINITY)) x[2 * e] += v0;
                if (!(fabsf(v1) < INFINITY)) x[2 * e + 1] += v1;
              }
            }
        }
      };
      if (!p.whole) {
        // ---- to the workspace ----
        float* part = reinterpret_cast<float*>(c.work + kKvPartOff) + (size_t)(2 * blockIdx.x + (bc.tile == 0 ? 1 : 0)) * T::kPiece;
        __stcg(reinterpret_cast<float2*>(part + (size_t)2 * 128 * D) + wg * 128 + row, make_float2(m, l));
        if (any) {
#pragma unroll 1
          for (int k = 0; k < D; k += 32) {
            float x[32];
            accumulators(k, x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              __stcg(reinterpret_cast<float4*>(part) + ((size_t)wg * (D / 4) + k / 4 + e) * 128 + row,
                     make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]));
          }
        }
      } else {
        // ---- to the output; where both groups had the same rows, B's sums by way of Q's place ----
        float4* swap = reinterpret_cast<float4*>(qmat);
        if (!p.two) {
          if (!meet()) break;                            // all scores are taken
          if (wg == 1) {
            sh.ml[row] = make_float2(m, l);
            if (any) {
#pragma unroll 1
              for (int k = 0; k < D; k += 32) {
                float x[32];
                accumulators(k, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) swap[(k / 4 + e) * 128 + row] = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
              }
            }
          }
          if (!meet()) break;
        }
        // group B has the rows behind the 128 in that case: they do not exist
        const int out_row = p.row0 + wg * 128 + row;
        float ka = 1.f, kb = 0.f;
        if (!p.two && wg == 0 && p.n > 1) {
          const float2 y = sh.ml[row];
          const float big = fmaxf(m, y.x);
          ka = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : exp2_approx(m - big);
          kb = y.x == -INFINITY ? (y.y == 0.f ? 0.f : 1.f) : exp2_approx(y.x - big);
          l = fmaf(ka, l, kb * y.y);
          m = big;
        }
        if (!have || (!p.two && wg == 1)) l = 0.f;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const bool exists = out_row < a.m * a.group;
        const int onode = exists ? out_row / a.group : 0, ohq = p.head * a.group + (exists ? out_row % a.group : 0);
        uint16_t* op = a.out + p.s * a.out_seq + onode * a.out_row + ohq * a.out_head;
#pragma unroll 1
        for (int k = 0; k < D; k += 32) {
          float x[32];
          if (any && (p.two || wg == 0)) {
            accumulators(k, x);
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] *= ka;
            if (kb != 0.f) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float4 y = swap[(k / 4 + e) * 128 + row];
                x[4 * e] = fmaf(kb, y.x, x[4 * e]);
                x[4 * e + 1] = fmaf(kb, y.y, x[4 * e + 1]);
                x[4 * e + 2] = fmaf(kb, y.z, x[4 * e + 2]);
                x[4 * e + 3] = fmaf(kb, y.w, x[4 * e + 3]);
              }
            }
          }
          if (exists) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              uint32_t w[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = l == 0.f ? 0u : pack16<kBf16>(x[8 * h + 2 * e] * inv, x[8 * h + 2 * e + 1] * inv);
              *reinterpret_cast<uint4*>(op + k + 8 * h) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
        if (exists && a.lse)
          a.lse[p.s * a.lse_seq + onode * a.lse_row + ohq * a.lse_head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kTrLn2;
      }
      fence_before();
      at += count;
      if (at < u1) list.advance(bc, count);
    }
  } else if (warp < 8 + kTrDecWarps) {
    // ============================================================ decode =========
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTrDecRegs));
    const int dw = warp - 8, sl = dw * 32 + lane;        // the thread's slot of every tile
    const uint32_t my_codes = kv_smem(codes + sl * T::kCodes);
    uint32_t kt = 0;
    bool ok = true;
    for (int at = 0; at < u1 && ok;) {
      const int n_tiles = bc.item < bc.live ? bc.tiles : 1, count = min(n_tiles - bc.tile, u1 - at);
      const Piece p = piece_at(bc, count, c, a);
      const int32_t* table = c.table + (size_t)p.s * c.max_pages;
      const int first = p.nodes ? -1 : 0, cached = p.n + first;   // tile -1: the new nodes
      auto page_for = [&](int i) {
        const int slot = (p.c0 + i) * kTrTile + sl;
        int q = -1;
        if (i < cached && slot < bc.len) {
          q = table[slot >> c.page_shift];
          q = (uint32_t)q < (uint32_t)c.n_pages ? q : -1;
        }
        return q;
      };
      auto block_of = [&](int q) { return c.pages + ((size_t)max(q, 0) * c.n_kv + p.head) * block_bytes; };
      auto slot_in = [&](int i) { return ((p.c0 + i) * kTrTile + sl) & (page - 1); };
      auto copy_codes = [&](int kv, int q, int i) {
        const unsigned char* b = block_of(q) + slot_in(i) * 32 + kv * (block_bytes / 2);
        if (i < cached)
#pragma unroll
          for (int g = 0; g < G; ++g)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              cp_async16(my_codes + (kv * G + g) * 32 + h * 16, b + g * page * 32 + h * 16, q < 0 ? 0 : 16);
        cp_async_commit();
      };
      auto load_meta_of = [&](uint32_t (&m)[2][G], int q, int i) {
        const unsigned char* b = block_of(q) + (G * page * 8 + slot_in(i) * G) * 4;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          uint32_t w[G];
#pragma unroll
          for (int g = 0; g < G; ++g) w[g] = 0u;
          if (q >= 0) load_meta<G>(b + kv * (block_bytes / 2), w);
#pragma unroll
          for (int g = 0; g < G; ++g) m[kv][g] = w[g];
        }
      };
      // the warp's largest key and value of tile t (counted over pieces) for the other warps
      auto post = [&](uint32_t t, uint32_t pk, uint32_t pv) {
        pk = __reduce_max_sync(0xffffffffu, pk);
        pv = __reduce_max_sync(0xffffffffu, pv);
        if (lane == 0) {
          sh.peak[t & 3][dw][0] = pk;
          sh.peak[t & 3][dw][1] = pv;
          bar_arrive(&sh.peaks[t & 1]);
        }
        __syncwarp();
      };
      auto post_meta = [&](uint32_t t, const uint32_t (&m)[2][G]) {
        uint32_t pk = 0, pv = 0;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          pk = max(pk, meta_peak<kBf16>(m[0][g]));
          pv = max(pv, meta_peak<kBf16>(m[1][g]));
        }
        post(t, pk, pv);
      };
      auto peaks_of = [&](uint32_t t, int& ek, int& ev) {
        uint32_t pk = 0, pv = 0;
#pragma unroll
        for (int w = 0; w < kTrDecWarps; ++w) { pk = max(pk, sh.peak[t & 3][w][0]); pv = max(pv, sh.peak[t & 3][w][1]); }
        ek = peak_exp(pk);
        ev = peak_exp(pv);
      };
      // Ahead of tile i: the codes of i + 1, scales and offsets (and posted peaks) of i + 1 and
      // i + 2, the page of i + 3.
      uint32_t mc[2][G], mn[2][G];
      int page_c = -1, page_n = -1, page_2 = -1;
      if (cached > 0) {
        page_c = page_for(0);
        page_n = page_for(1);
        page_2 = page_for(2);
        copy_codes(0, page_c, 0);                        // in the order of their use below
        copy_codes(1, page_c, 0);
        load_meta_of(mc, page_c, 0);
        load_meta_of(mn, page_n, 1);
        if (!p.nodes) post_meta(kt, mc);
      }
      for (int i = first; i < cached; ++i, ++kt) {
        const int st = kt & 1;
        const uint32_t ph = (kt >> 1) & 1;
        TileInfo& info = sh.info[kt & 3];
        unsigned char *km = kmat, *vm = vmat + st * T::kMat;
        if (i >= 0) {
          if (i + 1 < cached) post_meta(kt + 1, mn);
          uint32_t m2[2][G];
          load_meta_of(m2, page_2, i + 2);
          const int page_3 = page_for(i + 3);
          const uint32_t ballot = __ballot_sync(0xffffffffu, page_c >= 0);
          // The keys, whose one place is free once the last tile's scores are there, then the values.
          // (With the keys' place, four tiles back, the place of the tile's info is free.)
          int ek = 0, ev = 0;
#pragma unroll 1
          for (int part = 0; part < 2 && ok; ++part) {
            // (one body that the compiler cannot take apart into two: those took 118 us for 99)
            int which = part;
            asm volatile("" : "+r"(which));
            const bool values = which != 0;
            ok = warp_wait(values ? &sh.vfree[st] : &sh.kfree, (values ? ph : kt & 1) ^ 1, gave_up, stats);
            if (ok && !values) {
              ok = warp_wait(&sh.peaks[st], ph, gave_up, stats);
              peaks_of(kt, ek, ev);
              if (lane == 0) {
                info.valid[dw] = ballot;
                info.flags[dw] = ballot != 0xffffffffu ? 2 : 0;
                if (dw == 0) {
                  info.key_scale = pow2(ek);
                  info.value_exp = (float)ev;
                  info.value_scale = pow2(-ev);
                }
              }
            }
            if (!ok) break;
            // the codes of this tile, and on to the next one's (a thread reads its own copies alone)
            uint4 code[G][2];
            cp_async_wait<1>();
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                code[g][h] = *reinterpret_cast<const uint4*>(codes + sl * T::kCodes + ((values ? G : 0) + g) * 32 + h * 16);
            copy_codes(values, page_n, i + 1);
            const float down = pow2(-(values ? ev : ek));
            if (values) {
#pragma unroll
              for (int g = 0; g < G; ++g) {
                const uint32_t m1 = mc[1][g];
                const float fs = half_lo<kBf16>(m1) * down, fl = half_hi<kBf16>(m1) * down;
                const __half2 sc = as_half2(pack16<false>(fs, fs)), lo = as_half2(pack16<false>(fl, fl));
                unsigned char* dst = vm + g * (kTrTile * 128) + sl * 128;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                  *reinterpret_cast<uint4*>(dst + ((k ^ (sl & 7)) << 4)) = decode8((&code[g][k >> 2].x)[k & 3], sc, lo);
              }
            } else {
#pragma unroll
              for (int g = 0; g < G; ++g) {
                const uint32_t m1 = mc[0][g];
                const KeyParts parts = key_parts(half_lo<kBf16>(m1) * down, half_hi<kBf16>(m1) * down);
                unsigned char* dst = km + g * (kTrTile * 128) + sl * 128;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  uint4 hi, rest;
                  decode8_parts((&code[g][k >> 2].x)[k & 3], parts, hi, rest);
                  *reinterpret_cast<uint4*>(dst + ((k ^ (sl & 7)) << 4)) = hi;
                  *reinterpret_cast<uint4*>(dst + T::kMat + ((k ^ (sl & 7)) << 4)) = rest;
                }
              }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              bar_arrive(values ? &sh.vfull[st] : &sh.kfull);
              if (!values) bar_arrive(&sh.info_full[kt & 3]);
            }
          }
          if (!ok) break;
          page_c = page_n;
          page_n = page_2;
          page_2 = page_3;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int g = 0; g < G; ++g) { mc[kv][g] = mn[kv][g]; mn[kv][g] = m2[kv][g]; }
        } else {
          // ---- new nodes: 16-bit elements, slots 0..63 of the tile; the rest is zero ----
          // raw rows copied to where they will lie; a thread has one node's key or value.  Keys are
          // turned into f16 in place, each by a power of two of its own, values stay as they are
          // (their products take the cache's type): a hidden node's numbers, however large, take no
          // bits from what the others hold.
          if (!warp_wait(&sh.kfree, (kt & 1) ^ 1, gave_up, stats) || !warp_wait(&sh.vfree[st], ph ^ 1, gave_up, stats)) {
            ok = false;
            break;
          }
          unsigned char* mat = dw < 2 ? km : vm;
          const int r0 = (dw & 1) * 32, j = r0 + lane;
#pragma unroll 2
          for (int x = lane; x < 32 * (D / 8); x += 32) {
            const int r = r0 + x / (D / 8), chunk = x % (D / 8);
            const bool in = r < bc.nodes;
            cp_async16(kv_smem(mat + (chunk >> 3) * (kTrTile * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4)),
                       (dw < 2 ? a.k : a.v).at(p.s, in ? r : 0, p.head) + chunk * 8, in ? 16 : 0);
          }
          cp_async_commit();
          cp_async_wait<0>();
          __syncwarp();
          // (nothing to agree on, but the count of tiles goes on)
          post(kt, 0u, 0u);
          if (cached > 0) post_meta(kt + 1, mc);
          if (!warp_wait(&sh.peaks[st], ph, gave_up, stats)) { ok = false; break; }
          auto my_chunk = [&](int x) {
            return reinterpret_cast<uint4*>(mat + (x >> 3) * (kTrTile * 128) + j * 128 + (((x & 7) ^ (j & 7)) << 4));
          };
          bool odd = false;
          // (bf16 values leave fp32 the room that the probabilities take; f16 ends far below)
          constexpr int kNodeExp = kBf16 ? kTrRoom : 0;
          if (dw < 2) {
            float top = 0.f;
#pragma unroll 2
            for (int x = 0; x < D / 8; ++x) {
              const uint4 w = *my_chunk(x);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const uint32_t y = (&w.x)[e >> 1];
                const float v = fabsf(e & 1 ? half_hi<kBf16>(y) : half_lo<kBf16>(y));
                if (v < INFINITY) top = fmaxf(top, v);
              }
            }
            const int ek = peak_exp(__float_as_uint(top));
            const float down = pow2(-ek);
            info.node_exp[j] = (int8_t)ek;
#pragma unroll 2
            for (int x = 0; x < D / 8; ++x) {
              uint4* at_chunk = my_chunk(x);
              uint4 w = *at_chunk;
#pragma unroll
              for (int e = 0; e < 4; ++e) (&w.x)[e] = pack16<false>(half_lo<kBf16>((&w.x)[e]) * down, half_hi<kBf16>((&w.x)[e]) * down);
              *at_chunk = w;
              at_chunk[64 * 128 / 16] = make_uint4(0, 0, 0, 0);   // slots 64..127 of the tile
              // (f16 holds the keys whole)
              at_chunk[T::kMat / 16] = at_chunk[T::kMat / 16 + 64 * 128 / 16] = make_uint4(0, 0, 0, 0);
            }
          } else {
#pragma unroll 2
            for (int x = 0; x < D / 8; ++x) {            // values that are not finite: see `accumulators`
              uint4 w = *my_chunk(x);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t& v = (&w.x)[e];
                constexpr uint32_t kInf = kBf16 ? 0x7f80u : 0x7c00u;
                if ((v & kInf) == kInf) { odd = true; v &= 0xffff0000u; }
                if ((v >> 16 & kInf) == kInf) { odd = true; v &= 0x0000ffffu; }
                if (kNodeExp) v = pack16<kBf16>(half_lo<kBf16>(v) * pow2(-kNodeExp), half_hi<kBf16>(v) * pow2(-kNodeExp));
              }
              my_chunk(x)[0] = my_chunk(x)[64 * 128 / 16] = w;      // (once for each part of the probabilities)
            }
          }
          odd = __any_sync(0xffffffffu, odd);
          if (lane == 0) {
            info.valid[dw] = dw > 1 ? 0u : (uint32_t)(((bc.nodes >= 64 ? 0ull : 1ull << bc.nodes) - 1ull) >> (32 * dw));
            info.flags[dw] = 1 | (odd ? 4 : 0);
            if (dw == 0) {
              info.key_scale = 1.f;
              info.value_exp = kNodeExp;
              info.value_scale = pow2(-kNodeExp);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            bar_arrive(&sh.kfull);
            bar_arrive(&sh.vfull[st]);
            bar_arrive(&sh.info_full[kt & 3]);
          }
        }
      }
      at += count;
      if (at < u1) list.advance(bc, count);
    }
    cp_async_wait<0>();
  } else {
    // ============================================================ products =======
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTrIssueRegs));
    uint32_t kt = 0, np = 0, pu[2] = {0, 0};
    bool ok = warp == kTrIssuer;
    constexpr uint32_t s_idesc = idesc_16(kTrTile, false, false), o_idesc = idesc_16(D, true, false);
    constexpr uint32_t n_idesc = idesc_16(D, true, kBf16);           // new nodes' values
    // Descriptors are formed here, the same in every lane, and only a constant is added where
    // one lane issues: what that lane computed for itself would have to be moved to uniform
    // registers for every product.
    const uint64_t q_desc = desc128(kv_smem(qmat), 16), k_desc = desc128(kv_smem(kmat), 16),
                   v_desc = desc128(kv_smem(vmat), kTrTile * 128);
    constexpr uint64_t kStage = T::kMat >> 4;
    const bool issuer = one_lane();
    for (int at = 0; at < u1 && ok;) {
      const int n_tiles = bc.item < bc.live ? bc.tiles : 1, count = min(n_tiles - bc.tile, u1 - at);
      const Piece p = piece_at(bc, count, c, a);
      if (p.n > 0) {
        const int steps = p.two ? 2 * p.n : p.n;
        ok = warp_wait(&sh.qfull, np & 1, gave_up, stats);
        ++np;
        auto scores = [&](int u) {
          const uint32_t t = kt + (p.two ? u >> 1 : u);
          const int wg = u & 1;
          if (!p.two || wg == 0) ok = ok && warp_wait(&sh.kfull, t & 1, gave_up, stats);
          if (!ok) return;
          fence_after();
          const uint64_t qd = q_desc + (p.two && wg ? (uint64_t)(128 * 128 >> 4) : 0);
          const uint32_t to = tmem + wg * 256;
          if (issuer) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {           // the keys' leading parts and their rests
              const uint64_t qk = qd + (uint64_t)((k >> 2) * (256 * 128 >> 4) + (k & 3) * 2);
              const uint64_t kk = k_desc + (uint64_t)((k >> 2) * (kTrTile * 128 >> 4) + (k & 3) * 2);
              mma_ss(to, qk, kk, s_idesc, k > 0);
              mma_ss(to, qk, kk + kStage, s_idesc, 1u);
            }
            commit(&sh.sfull[wg]);
            if (!p.two || wg == 1) commit(&sh.kfree);
          }
          __syncwarp();
        };
        scores(0);
        if (steps > 1) scores(1);
        for (int u = 0; u < steps && ok; ++u) {
          const uint32_t t = kt + (p.two ? u >> 1 : u);
          const int st = t & 1, wg = u & 1;
          if (!p.two || wg == 0) ok = warp_wait(&sh.vfull[st], (t >> 1) & 1, gave_up, stats);
          ok = ok && warp_wait(&sh.pfull[wg], pu[wg] & 1, gave_up, stats);
          if (!ok) break;
          const uint32_t pv_idesc = __shfl_sync(0xffffffffu, p.nodes && t == kt ? n_idesc : o_idesc, 0);
          ++pu[wg];
          fence_after();
          const uint64_t vd = v_desc + (st ? kStage : 0);
          const uint32_t to = tmem + wg * 256 + 128, from = tmem + wg * 256, add = u > 1;
          if (issuer) {
#pragma unroll
            for (int k = 0; k < kTrTile / 16; ++k)
              mma_ts(to, from + k * 8, vd + (uint64_t)(k * (2048 >> 4)), pv_idesc, k > 0 ? 1u : add);
            commit(&sh.pvdone[wg]);
            if (!p.two || wg == 1) commit(&sh.vfree[st]);
          }
          __syncwarp();
          if (u + 2 < steps) scores(u + 2);
        }
        kt += p.n;
      }
      at += count;
      if (at < u1) list.advance(bc, count);
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kTrIssuer) {
    // What was issued is done before the memory goes away: the softmax warps waited for the last
    // products, unless somebody gave up.  (Read behind the barrier, when nobody can any more.)
    if (*gave_up) {
      const unsigned long long t0 = now_ns();
      while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// The pieces of every item joined, in their order.  A block: 128 rows of an item, 16 channels;
// a thread: a row, 4 channels.
template <int D, bool kBf16>
__global__ void __launch_bounds__(512)
kv_tree_join_kernel(const KvView c, const KvAttendArgs a, int tree_ctas) {
  using T = Tree<D>;
  extern __shared__ __align__(16) unsigned char smem[];
  long long* cum = reinterpret_cast<long long*>(smem);
  long long* scratch = cum + kKvMaxSeq + 1;
  pdl_enter();
  TreeList list;
  list.cum = cum;
  list.len = reinterpret_cast<int*>(scratch + 16);
  list.nodes = reinterpret_cast<unsigned char*>(list.len + kKvMaxSeq);
  list.items = c.n_kv * ((a.m * a.group + 255) / 256);
  list.group = a.group;
  list.rows = 256;
  list.build<512>(c, a.n_new, a.m, scratch);
  const int n_cta = (int)min((long long)tree_ctas, list.total);
  const int s = blockIdx.x / list.items, item = blockIdx.x % list.items;
  const int head = item % c.n_kv, row0 = item / c.n_kv * 256;
  const int halfb = blockIdx.y & 1, ch0 = (blockIdx.y >> 1) * 16 + (threadIdx.x >> 7) * 4, row = threadIdx.x & 127;
  const int my_row = row0 + halfb * 128 + row;
  if (my_row >= a.m * a.group) return;
  const int node = my_row / a.group, hq = head * a.group + my_row % a.group;
  const int n_rows = list.nodes[s] * a.group;
  if (item >= list.live_items(list.nodes[s])) return;    // its block wrote it, as all items it had whole
  const int tiles = list.tiles_of(list.len[s]);
  int b0, b1;
  list.owners(cum[s] + (long long)item * tiles, tiles, n_cta, b0, b1);
  if (b0 == b1) return;
  float big = -INFINITY, sum = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (my_row < n_rows) {
    const bool two = n_rows - row0 > 128;
    const float* parts = reinterpret_cast<const float*>(c.work + kKvPartOff);
    const int groups = two ? 1 : 2, n_src = (b1 - b0 + 1) * groups;
    constexpr int kBatch = 8;                            // pieces asked for at once
    for (int i0 = 0; i0 < n_src; i0 += kBatch) {
      float2 x[kBatch];
      float4 y[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        x[i] = make_float2(-INFINITY, 0.f);
        if (i0 + i < n_src) {
          const int b = b0 + (i0 + i) / groups, g = two ? halfb : (i0 + i) % groups;
          const float* part = parts + (size_t)(2 * b + (b == b0 ? 1 : 0)) * T::kPiece;
          x[i] = __ldcg(reinterpret_cast<const float2*>(part + (size_t)2 * 128 * D) + g * 128 + row);
          y[i] = __ldcg(reinterpret_cast<const float4*>(part) + ((size_t)g * (D / 4) + ch0 / 4) * 128 + row);
        }
      }
      float top = big;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) top = fmaxf(top, x[i].x);
      const float down = big == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : exp2_approx(big - top);
      big = top;
      sum *= down;
      v.x *= down; v.y *= down; v.z *= down; v.w *= down;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const float k = x[i].x == -INFINITY ? (x[i].y == 0.f ? 0.f : 1.f) : exp2_approx(x[i].x - big);
        sum = fmaf(k, x[i].y, sum);
        if (k != 0.f) {                                  // (a group without tiles left nothing)
          v.x = fmaf(k, y[i].x, v.x);
          v.y = fmaf(k, y[i].y, v.y);
          v.z = fmaf(k, y[i].z, v.z);
          v.w = fmaf(k, y[i].w, v.w);
        }
      }
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<uint2*>(a.out + s * a.out_seq + node * a.out_row + hq * a.out_head + ch0) =
      sum == 0.f ? make_uint2(0u, 0u)
                 : make_uint2(pack16<kBf16>(v.x * inv, v.y * inv), pack16<kBf16>(v.z * inv, v.w * inv));
  if (a.lse && ch0 == 0)
    a.lse[s * a.lse_seq + node * a.lse_row + hq * a.lse_head] = sum == 0.f ? -INFINITY : (big + log2f(sum)) * kTrLn2;
}

template <int D, bool kBf16>
static cudaError_t tree_launch(const KvView& c, const KvAttendArgs& a, int sms, cudaStream_t st) {
  const int grid = sms < kKvTreeMaxCtas ? sms : kKvTreeMaxCtas;
  const cudaError_t e = launch_pdl(kv_tree_kernel<D, kBf16>, dim3(grid), dim3(kTrThreads), Tree<D>::kBytes, st, c, a);
  if (e != cudaSuccess) return e;
  const int items = c.n_seq * c.n_kv * ((a.m * a.group + 255) / 256);
  return launch_pdl(kv_tree_join_kernel<D, kBf16>, dim3(items, 2 * (D / 16)), dim3(512), Tree<D>::kCum, st, c, a, grid);
}

cudaError_t launch_kv_tree(const KvView& c, const KvAttendArgs& a, int head_dim, bool bf16, int sms, cudaStream_t st) {
  if (head_dim == 64) return bf16 ? tree_launch<64, true>(c, a, sms, st) : tree_launch<64, false>(c, a, sms, st);
  return bf16 ? tree_launch<128, true>(c, a, sms, st) : tree_launch<128, false>(c, a, sms, st);
}

template <int D, bool kBf16>
static cudaError_t preload_tree() {
  const cudaError_t e = preload_kernel(kv_tree_kernel<D, kBf16>, true);
  return e != cudaSuccess ? e : preload_kernel(kv_tree_join_kernel<D, kBf16>, true);
}
cudaError_t preload_kv_tree_kernels() {
  cudaError_t e;
  if ((e = preload_tree<64, true>()) != cudaSuccess) return e;
  if ((e = preload_tree<64, false>()) != cudaSuccess) return e;
  if ((e = preload_tree<128, true>()) != cudaSuccess) return e;
  return preload_tree<128, false>();
}

}  // namespace oilbird
