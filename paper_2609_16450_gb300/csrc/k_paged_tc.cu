// Attention over the paged K/V cache with many query rows per K/V head (chunks
// of a prompt, windows of grouped heads) on the 5th-generation tensor cores.
// The mathematics and the treatment of values that are not finite are those of
// k_paged_attn.cu.
//
// A work item is two tiles of up to 128 packed rows of one sequence and K/V
// head; each CTA, one per SM, takes an equal share of all items' steps of 128
// keys (paged.h).  The two tiles run as two streams, S = Q K^T and O += P V of
// one on the tensor cores while the other's softmax runs.  Where a launch's
// sequences have no more rows than one tile, the streams are the same rows over
// alternate steps, put together in the end.
//   TMEM: S of stream 0 and 1 (128 columns each), O of stream 0 and 1 (D
//     each).  P, in bf16, overwrites the S that it came from and is the A
//     operand of P V from there.
//   warps 0-3, 4-7: softmax of stream 0, 1, a thread per row;
//   warps 8-11: 8-bit caches: V's codes become bf16, times their row's scale,
//     and K's exponent bytes become factors of the scores; bf16 ones: only the
//     steps that end in keys which rows do not see;
//   warp 12: loads of q and K; warp 14: loads of V; warps 13, 15: the MMAs of
//     stream 0, 1.
// 8-bit K and q in two e4m3 terms multiply as they are (kind::f8f6f4, at twice the
// rate of bf16: the two terms cost what bf16 would).
//
// Measured: 2 x 1000 rows over 8000 bf16 keys (causal), 28 / 4 heads, 195 to 197 us
// (1100 TFLOP/s, 57 %): two tiles' step of 128 keys takes some 3500 cycles, its MMAs
// 2064, as a stream's S (1450 from its turn), softmax (1620 and more) and P (410)
// follow one another; 61 rows over 60061 8-bit keys 94 us: 4600 a step, V's
// conversion and K's factors sharing the issue slots.  Tried while they took 188 and
// 88: all eight softmax warps on one stream at a time, two threads per row, 189 and
// 103; P handed over in halves 192 and 89.  Scores rounded before the reference is
// taken off, K's factors times the row's first, cost 1 % and 4 %.
#include <cuda_fp16.h>
#include <type_traits>

#include "paged.h"
#include "paged_math.h"
#include "ptx.cuh"

namespace ebd {

namespace {

constexpr int kStep = 1 << kPagedTcStepLog2;     // keys of a step
constexpr int kThreads = 512;
// Steps of a share, at least: 1, 2, 4, 8 take 128 rows over 728 bf16 keys of 32 heads
// 19.6, 18.6, 26.3, 31.0 us, 40 rows over 3040 8-bit keys of 28 / 4 28.2, 25.6, 28.6,
// 37.2, over 740 bf16 keys 17.9, 19.0, 27.9, 34.8.
constexpr int kLeast = 2;
constexpr int kNever = 0x7fffffff;
constexpr uint32_t kTmemCols = 512;
// Notes of values that are not finite, per item in turn.  The warps that take
// them are at most three items ahead of a softmax that reads them: an item is
// begun when every softmax warp has left the steps of the one before, and V is
// loaded two steps ahead, which may be two items.
constexpr int kBads = 4;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2(float x, float y) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
  return r;
}
__device__ __forceinline__ float2 e4m3x2_value(uint32_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(c)));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float scale_value(uint32_t e) { return __uint_as_float(e > 0 ? e << 23 : 1u << 22); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// two 32-bit floats at a time
__device__ __forceinline__ void mul2(float& x, float& y, float a, float b) {
  asm("{\n .reg .b64 v, m;\n mov.b64 v, {%0, %1};\n mov.b64 m, {%2, %3};\n mul.rn.f32x2 v, v, m;\n"
      " mov.b64 {%0, %1}, v;\n}"
      : "+f"(x), "+f"(y)
      : "f"(a), "f"(b));
}
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {
  asm("{\n .reg .b64 v, m;\n mov.b64 v, {%0, %1};\n mov.b64 m, {%2, %3};\n add.rn.f32x2 v, v, m;\n"
      " mov.b64 {%0, %1}, v;\n}"
      : "+f"(x), "+f"(y)
      : "f"(a), "f"(b));
}

// 32 lanes x 32 columns, without the wait
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// Completes the loads above; the values pass through it, so that no use of
// them can be moved ahead.
template <int N>
__device__ __forceinline__ void tmem_ld_wait(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
      "%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
      "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// MMAs with descriptors as low words and a shared high word: bf16 or e4m3 A
// and B from shared memory, and bf16 A from TMEM.
__device__ __forceinline__ void umma_e4m3_lo(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                             uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 ad, bd;\n setp.ne.b32 p, %5, 0;\n"
      " mov.b64 ad, {%1, %3};\n mov.b64 bd, {%2, %3};\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, p;\n}\n" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc));
}
__device__ __forceinline__ void umma_bf16_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                             uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 bd;\n setp.ne.b32 p, %5, 0;\n mov.b64 bd, {%2, %3};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], bd, %4, p;\n}\n" ::"r"(d),
      "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc));
}
__device__ __forceinline__ uint32_t swz(int r, int c) {
  return static_cast<uint32_t>(r * 128 + ((c ^ (r & 7)) << 4));
}
template <int N>
__device__ __forceinline__ void regs_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
// 512 threads start with 128 registers each; the softmax's 256 take 176 and
// the others 80: 256 * 176 + 256 * 80 = 512 * 128.
constexpr int kSoftmaxRegs = 176, kOtherRegs = 80;

template <int D, bool E4M3>
struct Map {
  static constexpr int NB = D / 64;
  static constexpr uint32_t kTile = 128 * D * 2;             // q of a stream: bf16, or its two terms
  static constexpr uint32_t kK = kStep * D * (E4M3 ? 1 : 2);  // a step's K
  static constexpr uint32_t kV = kStep * D * 2;               // a step's V in bf16
  static constexpr int kKs = E4M3 ? 3 : 2, kVs = 2;           // ring slots
  // K's factors.  Step g's are written once K of step g is there, so once S of
  // step g - 3 was computed, so, in either form of the streams, once the softmax
  // is through with step g - 5.
  static constexpr int kFs = 5;
  static constexpr uint32_t kQ = 0;
  static constexpr uint32_t kK0 = kQ + 2 * kTile;
  static constexpr uint32_t kV0 = kK0 + kKs * kK;
  static constexpr uint32_t kRaw = kV0 + kVs * kV;            // 8-bit V as loaded
  static constexpr uint32_t kKe = kRaw + (E4M3 ? kVs * kStep * D : 0);  // exponent bytes
  static constexpr uint32_t kVe = kKe + kKs * kStep;
  static constexpr uint32_t kKf = kVe + kVs * kStep;          // [kFs][kStep] K's factors, f32
  static constexpr uint32_t kRowF = kKf + (E4M3 ? kFs * kStep * 4 : 0);  // [2][128]
  static constexpr uint32_t kMl = kRowF + 2 * 128 * 4;        // [128][2] stream 1's (maximum, sum)
  static constexpr uint32_t kBad = kMl + 128 * 8;             // [kBads][3][D]
  static constexpr uint32_t kBar = kBad + kBads * 3 * D * 4;
  // k full, empty, factors; v full, empty, raw full, raw empty; s, p, o full
  // and o free of 2 streams; q full, ready, empty; drain and turn of 2 streams
  static constexpr int kNBar = 2 * kKs + kFs + 4 * kVs + 8 + 7;
  static constexpr uint32_t kPlan = kBar + kNBar * 8;
  static constexpr uint32_t kMisc = kPlan + sizeof(PagedStart) + (kThreads / 32) * 4;
  static constexpr uint32_t kBytes = kMisc + 32;
  static constexpr uint32_t kDyn = kBytes + 1024;
  static_assert(kDyn <= 227 * 1024 && 2 * kTile >= 128 * 64 * 4 + kTile, "shared memory");
};

template <int D, bool E4M3>
__global__ void __launch_bounds__(kThreads, 1)
    paged_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const PagedParams p, const int one) {
  using L = Map<D, E4M3>;
  constexpr int NB = L::NB;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);  // an offset: accesses stay LDS and STS
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBar);
  uint64_t* kfull = bars;
  uint64_t* kempty = kfull + L::kKs;
  uint64_t* kfact = kempty + L::kKs;
  uint64_t* vfull = kfact + L::kFs;    // V in bf16 (8-bit caches: converted)
  uint64_t* vempty = vfull + L::kVs;
  uint64_t* rfull = vempty + L::kVs;   // 8-bit V as loaded; bf16: V's last rows seen to
  uint64_t* rempty = rfull + L::kVs;
  uint64_t* s_full = rempty + L::kVs;  // [2] by stream
  uint64_t* p_full = s_full + 2;
  uint64_t* o_full = p_full + 2;
  uint64_t* o_free = o_full + 2;
  uint64_t* q_full = o_free + 2;
  uint64_t* q_ready = q_full + 1;
  uint64_t* q_empty = q_ready + 1;
  uint64_t* drain = q_empty + 1;   // [2]
  uint64_t* turn = drain + 2;      // [2]
  PagedStart* plan = reinterpret_cast<PagedStart*>(smem + L::kPlan);
  auto& scan = *reinterpret_cast<unsigned(*)[kThreads / 32]>(smem + L::kPlan + sizeof(PagedStart));
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + L::kMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(smem + L::kMisc + 4);
  int* s_bad = reinterpret_cast<int*>(smem + L::kMisc + 16);  // [kBads] by item
  int* bad = reinterpret_cast<int*>(smem + L::kBad);
  float* rowf = reinterpret_cast<float*>(smem + L::kRowF);

  // rows of a tile: whole tokens, so that its q is a box of (64 columns, heads
  // of the group, tokens)
  const int tile = 128 / p.group * p.group;
  const int T = one ? tile : 2 * tile;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < L::kKs; ++s) {
      mbar_init(&kfull[s], 1);
      mbar_init(&kempty[s], E4M3 ? 6 : 2);  // the two streams' MMAs, and the warps that read its exponents
    }
    for (int s = 0; s < L::kFs; ++s) mbar_init(&kfact[s], 4);
    for (int s = 0; s < L::kVs; ++s) {
      mbar_init(&vfull[s], E4M3 ? 4 : 1);
      mbar_init(&vempty[s], E4M3 ? 2 : 6);  // the two streams' MMAs, and the warps that see to its last rows
      mbar_init(&rfull[s], E4M3 ? 1 : 4);
      mbar_init(&rempty[s], 4);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&s_full[x], 1);
      mbar_init(&p_full[x], 4);
      mbar_init(&o_full[x], 1);
      mbar_init(&o_free[x], 4);
    }
    mbar_init(q_full, 1);
    mbar_init(q_ready, 8);
    mbar_init(q_empty, 10);  // the two streams' MMAs, and the softmax warps
    mbar_init(&drain[0], 1);
    mbar_init(&drain[1], 1);
    mbar_init(&turn[0], 1);
    mbar_init(&turn[1], 1);
    *abort = 0;
    for (int i = 0; i < kBads; ++i) s_bad[i] = 0;
    fence_mbar_init();
  }
  for (int i = tid; i < kBads * 3 * D; i += kThreads) bad[i] = kNever;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == 13) tmem_alloc(tmem_holder, kTmemCols);
  tc_fence_before();
  paged_plan<kThreads>(p, T, kStep, kLeast, plan, scan);  // ends in a barrier of all threads
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  PagedWalk<0, kStep> w;
  const bool work = w.begin(p, *plan, T);
  // no tile to be put together yet (as in k_paged_attn.cu)
  if (tid == 12 * 32) p.cuts[blockIdx.x] = PagedCut{};
  auto gave_up = [&]() {
    if (!*abort) {
      *abort = 1;
      atomicCAS(p.status, 0, EBD_ERR_TIMEOUT);
    }
  };
  // steps of stream x of a piece of n: all of them, or every other one
  auto rows_here = [&]() { return min(T, w.s.n * p.group - w.t * T); };
  auto steps_of = [&](int x, int n) { return one ? (n + 1 - x) / 2 : (x == 0 || rows_here() > tile ? n : 0); };
  // the first and the last of the item's limits
  auto lim_first = [&]() { return paged_limit(p, w.s, paged_row(p, w.t * T)); };
  auto lim_last = [&]() { return paged_limit(p, w.s, paged_row(p, w.t * T + rows_here() - 1)); };

  if (warp >= 12) {
    regs_dec<kOtherRegs>();
    if (work && (warp == 12 || warp == 14)) {
      // ---------------------------------------------------------- loads
      const bool is_k = warp == 12;
      const int slots = is_k ? L::kKs : L::kVs;
      uint64_t* fullb = is_k ? kfull : (E4M3 ? rfull : vfull);
      uint64_t* emptyb = is_k ? kempty : (E4M3 ? rempty : vempty);
      uint8_t* ring = smem + (is_k ? L::kK0 : (E4M3 ? L::kRaw : L::kV0));
      uint8_t* ering = smem + (is_k ? L::kKe : L::kVe);
      const uint32_t op = E4M3 ? kStep * D : L::kV;
      const CUtensorMap* tm = is_k ? &tm_k : &tm_v;
      const uint8_t* scales = is_k ? p.k_scale : p.v_scale;
      const int np_log = 7 - p.box_log2, box = 1 << p.box_log2;
      const int pc = lane & ((1 << np_log) - 1), part = lane >> np_log;
      const int key_in = pc << p.box_log2;
      int n = 0, items = 0;
      bool ok = true;
      do {
        auto load_q = [&]() {
          ok = items == 0 || mbar_wait(q_empty, static_cast<uint32_t>(items - 1) & 1u, p.limit_ns, abort);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) return;
          const int tiles = !one && rows_here() > tile ? 2 : 1;
          if (lane == 0) mbar_arrive_expect_tx(q_full, static_cast<uint32_t>(tiles) * tile * D * 2);
          __syncwarp();
          if (lane < tiles * NB) {
            const int x = lane / NB, hf = lane % NB;
            tma_load_3d(smem + L::kQ + x * L::kTile + hf * 16384, &tm_q, q_full, hf * 64, w.h * p.group,
                        w.s.r0 + paged_row(p, w.t * T + x * tile));
            PagedWalk<0, kStep> next = w;  // the next item's q into L2
            if (next.next(p))
              asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(&tm_q),
                           "r"(hf * 64), "r"(next.h * p.group), "r"(next.s.r0 + paged_row(p, next.t * T + x * tile))
                           : "memory");
          }
          ++items;
        };
        const int lim = lim_last();
        const int* table = p.page_table + static_cast<long long>(w.b) * p.max_pages;
        int win0 = ((w.c0 * kStep) >> p.page_log2) & ~31;  // page ids of 32 pages, one per lane
        int win = win0 + lane < p.max_pages ? table[win0 + lane] : -1;
        for (int c = w.c0; c < w.c1; ++c, ++n) {
          const int key = c * kStep + key_in;
          const int first = (c * kStep) >> p.page_log2;
          if (first >= win0 + 32) {
            win0 = first & ~31;
            win = win0 + lane < p.max_pages ? table[win0 + lane] : -1;
          }
          int page = __shfl_sync(0xffffffffu, win, ((key >> p.page_log2) - win0) & 31);
          const bool mine = part < (E4M3 ? 2 : NB) && key < lim;
          if (mine && (page < 0 || page >= p.n_pages)) {
            atomicCAS(p.status, 0, EBD_ERR_BOUNDS);
            page = 0;
          }
          const int pieces = min(max((lim - c * kStep + box - 1) >> p.box_log2, 0), 1 << np_log);
          const int s = n % slots;
          ok = !p.give_up &&
               (n < slots || mbar_wait(&emptyb[s], static_cast<uint32_t>(n / slots - 1) & 1u, p.limit_ns, abort));
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane == 0)
            mbar_arrive_expect_tx(&fullb[s], static_cast<uint32_t>(pieces) * box * (E4M3 ? D + 1 : 2 * D));
          __syncwarp();
          if (mine) {
            const int off = key & ((1 << p.page_log2) - 1);
            if (E4M3 && part == 1)
              bulk_load(ering + s * kStep + key_in,
                        scales + ((static_cast<long long>(page) * p.Hkv + w.h) << p.page_log2) + off, box, &fullb[s]);
            else
              tma_load_4d(ring + s * op + part * 16384 + key_in * 128, tm, &fullb[s], part * 64, off, w.h, page);
          }
          // K of the item's first steps goes ahead of its q, which waits for the last item's results
          if (is_k && c == min(w.c0 + slots, w.c1) - 1) load_q();
          if (!ok) {
            ++n;
            break;
          }
        }
        if (is_k && lane == 0 && w.u + (w.c1 - w.c0) >= w.u1) w.leave(p, *plan);
      } while (ok && w.next(p));
      if (!ok) {
        if (lane == 0) gave_up();
        // the copies in flight land before the CTA can exit
        for (int j = max(0, n - slots); j < n; ++j)
          mbar_wait(&fullb[j % slots], static_cast<uint32_t>(j / slots) & 1u, p.limit_ns, nullptr);
        if (is_k && items > 0) mbar_wait(q_full, static_cast<uint32_t>(items - 1) & 1u, p.limit_ns, nullptr);
      }
    } else if (work) {
      // ---------------------------------------------------------- MMAs of stream x
      const int x = warp == 13 ? 0 : 1;
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint32_t idesc_s = E4M3 ? (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24) : umma_idesc_bf16(128, 128);
      const uint32_t idesc_o = umma_idesc_bf16(128, D) | (1u << 16);  // B (V) MN-major
      const uint32_t hi = static_cast<uint32_t>(umma_desc_sw128(0) >> 32);
      const uint32_t q_lo = static_cast<uint32_t>(umma_desc_sw128(smem_u32(smem + L::kQ)));
      const uint32_t k_lo0 = static_cast<uint32_t>(umma_desc_sw128(smem_u32(smem + L::kK0)));
      // V: 64-column blocks 16384 bytes apart (leading byte offset)
      const uint32_t v_lo0 = ((smem_u32(smem + L::kV0) >> 4) & 0x3FFFu) | ((16384u >> 4) << 16);
      // A turn is P V of a step and S of the next.  All that it needs is waited
      // for before the probabilities, its last operand.  A warp of its own for
      // each stream, as one warp's waits and issues took as long as its MMAs,
      // which idled meanwhile; and turns alternate, as MMAs of both streams
      // mixed end together, both softmaxes then run at once, and the tensor
      // cores wait for them (4480 cycles a step instead of ~3000).
      const uint32_t ts = __shfl_sync(0xffffffffu, tm + static_cast<uint32_t>(x * 128), 0);
      const uint32_t to = tm + 256u + static_cast<uint32_t>(x * D);
      int kn = 0, en = 0;  // steps, and steps whose V is seen to, before this item
      uint32_t qph = 0, pph = 0, fph = 1, tph = x == 0 ? 1 : 0;  // q, p_full, o_free (free at first), turn (stream 0's)
      bool ok = true;
      // Steps in order: a step that is the other stream's is passed when it has
      // landed, with this stream's share of its slot's release, so that no wait
      // is ever two phases of its barrier away.
      int kpos = 0, vpos = 0;
      auto k_there = [&](int st) {
        return mbar_wait(&kfull[st % L::kKs], static_cast<uint32_t>(st / L::kKs) & 1u, p.limit_ns, abort);
      };
      auto v_there = [&](int st) {
        return mbar_wait(&vfull[st % L::kVs], static_cast<uint32_t>(st / L::kVs) & 1u, p.limit_ns, abort);
      };
      auto pass_k = [&](int to_step) {
        for (; kpos < to_step; ++kpos) {
          ok = ok && __all_sync(0xffffffffu, k_there(kpos));
          if (lane == 0) mbar_arrive(&kempty[kpos % L::kKs]);
        }
      };
      auto pass_v = [&](int to_step) {
        for (; vpos < to_step; ++vpos) {
          ok = ok && __all_sync(0xffffffffu, v_there(vpos));
          if (lane == 0) mbar_arrive(&vempty[vpos % L::kVs]);
        }
      };
      do {
        const int n = w.c1 - w.c0;
        const int mine = steps_of(x, n), turns = steps_of(0, n) + 1;
        const int edge0 = E4M3 ? n : max(0, min(n, lim_first() / kStep - w.c0));  // V steps from here are seen to
        const uint32_t ql = q_lo + (one ? 0u : static_cast<uint32_t>(x) * (L::kTile >> 4));
        ok = __all_sync(0xffffffffu, mbar_wait(E4M3 ? q_ready : q_full, qph, p.limit_ns, abort));
        if (!ok) break;
        qph ^= 1u;
        for (int i = 0; i < turns && ok; ++i) {
          const bool pv = i > 0 && i - 1 < mine, qk = i < mine;
          const int kst = kn + (one ? 2 * i + x : i), vst = kst - (one ? 2 : 1);
          if (qk) pass_k(kst);
          if (pv) pass_v(vst);
          if (mine == 0 && i < n) {
            pass_k(kn + i + 1);
            pass_v(kn + i + 1);
          }
          const int ks = kst % L::kKs, vs = vst % L::kVs;
          const uint32_t v_lo = v_lo0 + static_cast<uint32_t>(vs) * (L::kV >> 4);
          const uint32_t kl = k_lo0 + static_cast<uint32_t>(ks) * (L::kK >> 4);
          bool g = mbar_wait(turn + x, tph, p.limit_ns, abort);
          tph ^= 1u;
          if (qk) g = g && k_there(kst);
          if (pv) {
            g = g && v_there(vst);
            if constexpr (!E4M3) {
              const int e = en + vst - kn - edge0;
              if (vst - kn >= edge0) g = g && mbar_wait(&rfull[e & 1], static_cast<uint32_t>(e >> 1) & 1u, p.limit_ns, abort);
            }
            if (i == 1) {
              g = g && mbar_wait(o_free + x, fph, p.limit_ns, abort);
              fph ^= 1u;
            }
            g = g && mbar_wait(p_full + x, pph, p.limit_ns, abort);
            pph ^= 1u;
          }
          ok = ok && __all_sync(0xffffffffu, g);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            if (pv) {
#pragma unroll
              for (int kk = 0; kk < kStep / 16; ++kk)
                umma_bf16_ts(to, ts + static_cast<uint32_t>(kk * 8), v_lo + static_cast<uint32_t>(kk * (2048 >> 4)), hi,
                             idesc_o, kk != 0 || i > 1 ? 1u : 0u);
              umma_commit(&vempty[vs]);
              if (i == mine) umma_commit(o_full + x);
            }
            if (qk) {
              if constexpr (E4M3) {
#pragma unroll
                for (int term = 0; term < 2; ++term)
#pragma unroll
                  for (int kk = 0; kk < D / 32; ++kk) {
                    if (term == 1 && kk == 0) mbar_arrive(turn + (x ^ 1));
                    umma_e4m3_lo(ts, ql + static_cast<uint32_t>(term * (16384 >> 4) + kk * 2),
                                 kl + static_cast<uint32_t>(kk * 2), hi, idesc_s, term + kk > 0 ? 1u : 0u);
                  }
              } else {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                  if (kk == D / 32) mbar_arrive(turn + (x ^ 1));  // half a product ahead: issue waits on the pipe
                  umma_bf16_lo(ts, ql + static_cast<uint32_t>((kk >> 2) * (16384 >> 4) + (kk & 3) * 2),
                               kl + static_cast<uint32_t>((kk >> 2) * (16384 >> 4) + (kk & 3) * 2), hi, idesc_s,
                               kk > 0 ? 1u : 0u);
                }
              }
              umma_commit(s_full + x);
              umma_commit(&kempty[ks]);
              if (i == mine - 1) umma_commit(q_empty);
            } else {
              mbar_arrive(turn + (x ^ 1));
            }
          }
          __syncwarp();
          if (qk) kpos = kst + 1;
          if (pv) vpos = vst + 1;
        }
        if (!ok) break;
        if (mine == 0) {
          if (lane == 0) mbar_arrive(q_empty);
        }
        pass_k(kn + n);
        pass_v(kn + n);
        kn += n;
        en += n - edge0;
      } while (ok && w.next(p));
      if (!ok) {
        if (lane == 0) gave_up();
        if (elect_one()) umma_commit(drain + x);  // completes once every MMA issued so far is done
        __syncwarp();
        mbar_wait(drain + x, 0, p.limit_ns, nullptr);
      }
    }
  } else if (warp >= 8) {
    // ------------------------------------------------------------ V's codes, K's factors, last rows
    regs_dec<kOtherRegs>();
    const int r = tid - 256;  // key of a step
    int vn = 0, en = 0, items = 0;
    bool ok = work;
    if (work) do {
      const int n = w.c1 - w.c0;
      const int lo = lim_first(), hi = lim_last();
      int* badp = bad + (items % kBads) * 3 * D;
      // Notes of an item long done go first.  The four warps drift by up to two
      // steps, so none may take a note of this item before all have looked:
      // what they see, and the barrier below with it, would differ by warp.
      const bool used = *reinterpret_cast<volatile int*>(&s_bad[items % kBads]) != 0;
      named_barrier(2, 128);
      if (used) {
        for (int i = r; i < 3 * D; i += 128) badp[i] = kNever;
        if (r == 0) *reinterpret_cast<volatile int*>(&s_bad[items % kBads]) = 0;
        named_barrier(2, 128);
      }
      // rows from `hi` on nobody sees; of those from `lo` on, hidden from some
      // rows, what is not finite is kept out and noted for the rows that see it
      auto note = [&](int key, int d, int kind) {
        atomicMin(&badp[kind * D + d], key);
        *reinterpret_cast<volatile int*>(&s_bad[items % kBads]) = 1;
      };
      if constexpr (E4M3) {
        auto factors = [&](int j) {
          const int s = (vn + j) % L::kKs, fs = (vn + j) % L::kFs;
          ok = ok && mbar_wait(&kfull[s], static_cast<uint32_t>((vn + j) / L::kKs) & 1u, p.limit_ns, abort);
          ok = __all_sync(0xffffffffu, ok);
          reinterpret_cast<float*>(smem + L::kKf)[fs * kStep + r] = scale_value((smem + L::kKe)[s * kStep + r]);
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&kfact[fs]);
            mbar_arrive(&kempty[s]);
          }
        };
        factors(0);
        for (int j = 0; j < n; ++j) {
          if (j + 1 < n) factors(j + 1);
          const int s = (vn + j) % L::kVs;
          const uint32_t ph = static_cast<uint32_t>((vn + j) / L::kVs) & 1u;
          ok = ok && mbar_wait(&rfull[s], ph, p.limit_ns, abort);
          if (vn + j >= L::kVs) ok = ok && mbar_wait(&vempty[s], ph ^ 1u, p.limit_ns, abort);
          ok = __all_sync(0xffffffffu, ok);
          const int key = (w.c0 + j) * kStep + r;
          const uint32_t e = (smem + L::kVe)[s * kStep + r];
          // 2^(120 + k): codes moved into place are 2^-120 times their value
          uint32_t m = (min(e, 134u) + 120u) << 7;
          uint32_t m2 = e > 134u ? (e - 7u) << 7 : 0x3F80u;  // past that, the rest of the scale: 2^(e - 134)
          if (e == 255u) m = m2 = 0x7FC0u;
          if (key >= hi) {
            m = 0u;
            m2 = 0x3F80u;
          } else if (e == 255u && key >= lo) {
            for (int d = 0; d < D; ++d) note(key, d, 0);
            m = 0u;
            m2 = 0x3F80u;
          }
          m |= m << 16;
          m2 |= m2 << 16;
          const bool two = __any_sync(0xffffffffu, m2 != 0x3F803F80u);
          const uint8_t* src = smem + L::kRaw + s * kStep * D;
          uint8_t* dst = smem + L::kV0 + s * L::kV;
          uint4 in[D / 16];
#pragma unroll
          for (int c = 0; c < D / 16; ++c) in[c] = *reinterpret_cast<const uint4*>(src + swz(r, c));
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const uint32_t x[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
            uint32_t y[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              // bytes d0, d1, d2, d3 -> (d0, d1), (d2, d3)
              const uint32_t a = __byte_perm(x[i], 0u, 0x1404), b = __byte_perm(x[i], 0u, 0x3424);
              y[2 * i] = mul_bf16x2((a & 0x80008000u) | ((a >> 4) & 0x07F007F0u), m);
              y[2 * i + 1] = mul_bf16x2((b & 0x80008000u) | ((b >> 4) & 0x07F007F0u), m);
            }
            if (two) {
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = mul_bf16x2(y[i], m2);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int ch = 2 * c + i;  // 16 bytes of bf16 columns
              *reinterpret_cast<uint4*>(dst + (ch >> 3) * 16384 + swz(r, ch & 7)) =
                  make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
            }
          }
          fence_async();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&vfull[s]);
            mbar_arrive(&rempty[s]);
          }
        }
      } else {
        // bf16: only the steps that hold keys past `lo`
        const int edge0 = max(0, min(n, lo / kStep - w.c0));
        for (int j = 0; j < n; ++j) {
          const int s = (vn + j) % L::kVs;
          ok = ok && mbar_wait(&vfull[s], static_cast<uint32_t>((vn + j) / L::kVs) & 1u, p.limit_ns, abort);
          ok = __all_sync(0xffffffffu, ok);
          const int key = (w.c0 + j) * kStep + r;
          uint8_t* v = smem + L::kV0 + s * L::kV;
          if (ok && j >= edge0 && key >= lo) {
#pragma unroll 4
            for (int c = 0; c < D / 8; ++c) {
              uint4* q = reinterpret_cast<uint4*>(v + (c >> 3) * 16384 + swz(r, c & 7));
              if (key >= hi) {
                *q = make_uint4(0u, 0u, 0u, 0u);
                continue;
              }
              const uint4 x4 = *q;
              // an exponent of ones carries into the sign's bit
              auto ones = [](uint32_t u) { return (u & 0x7F807F80u) + 0x00800080u; };
              if (((ones(x4.x) | ones(x4.y) | ones(x4.z) | ones(x4.w)) & 0x80008000u) == 0) continue;
              uint16_t* e = reinterpret_cast<uint16_t*>(q);
#pragma unroll 1
              for (int i = 0; i < 8; ++i) {
                const uint32_t u = e[i];
                if ((u & 0x7F80u) != 0x7F80u) continue;
                note(key, c * 8 + i, (u & 0x7Fu) ? 0 : (u & 0x8000u) ? 2 : 1);
                e[i] = 0;
              }
            }
          }
          if (j >= edge0) fence_async();
          __syncwarp();
          if (lane == 0) {
            if (j >= edge0) mbar_arrive(&rfull[(en + j - edge0) & 1]);
            mbar_arrive(&vempty[s]);
          }
        }
        en += n - edge0;
      }
      vn += n;
      ++items;
    } while (w.next(p));
    if (!ok && work && lane == 0) gave_up();
  } else {
    // ------------------------------------------------------------ softmax: stream x, a thread per row
    regs_inc<kSoftmaxRegs>();
    const int x = warp >> 2, row = tid & 127;
    const uint32_t quad = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + quad + static_cast<uint32_t>(x * 128);
    const uint32_t to = tmem + quad + 256u + static_cast<uint32_t>(x * D);
    int kn = 0, items = 0, done = 0, outs = 0;
    bool ok = work;
    if (work) do {
      const int n = w.c1 - w.c0;
      const int mine = steps_of(x, n);
      const int rows = rows_here();
      const int m_row = w.t * T + (one ? 0 : x * tile) + row;  // packed row
      const bool valid = row < tile && (one ? 0 : x * tile) + row < rows;
      const int lim = valid ? paged_limit(p, w.s, paged_row(p, m_row)) : kNever;
      const int lo = lim_first();
      float f = p.scale_log2;
      // also where nothing of q is needed here: a stream without steps must not
      // give q back (below) before the item has it
      ok = ok && mbar_wait(q_full, static_cast<uint32_t>(items) & 1u, p.limit_ns, abort);
      ok = __all_sync(0xffffffffu, ok);
      if constexpr (E4M3) {
        // q as two e4m3 terms, in place, 8 lanes a row: the row's 128 bytes of columns
        // 0..63 become its high terms, those of 64..127 its low ones.  (A thread per
        // row, unrolled, took 14000 cycles, most of them to fetch the instructions.)
        if (x == 0 || (!one && mine > 0)) {
          uint8_t* q = smem + L::kQ + x * L::kTile;
          const int c = lane & 7;
#pragma unroll 1
          for (int r = (warp & 3) * 4 + (lane >> 3); r < 128; r += 16) {
            uint4 v[2];
            uint32_t amax = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              v[k] = *reinterpret_cast<const uint4*>(q + (c >> 2) * 16384 + swz(r, (2 * c + k) & 7));
              const uint32_t u[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
              for (int e = 0; e < 4; ++e) amax = max(amax, max(u[e] & 0x7FFFu, (u[e] >> 16) & 0x7FFFu));
            }
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            const bool finite = amax < 0x7F80u;
            const int e = finite ? max(0, static_cast<int>(amax >> 7) - 8 + ((amax & 0x7Fu) > 0x60u ? 1 : 0)) : 127;
            const float inv = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
            uint32_t h[4], lw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint4 vv = v[k >> 1];
              const uint32_t u0 = k & 1 ? vv.z : vv.x, u1 = k & 1 ? vv.w : vv.y;
              const float a = __uint_as_float(u0 << 16) * inv, b = __uint_as_float(u0 & 0xFFFF0000u) * inv;
              const float cc = __uint_as_float(u1 << 16) * inv, d = __uint_as_float(u1 & 0xFFFF0000u) * inv;
              const uint32_t h0 = e4m3x2(a, b), h1 = e4m3x2(cc, d);
              const float2 f0 = e4m3x2_value(h0), f1 = e4m3x2_value(h1);
              h[k] = finite ? h0 | (h1 << 16) : 0x7F7F7F7Fu;
              lw[k] = e4m3x2(a - f0.x, b - f0.y) | (e4m3x2(cc - f1.x, d - f1.y) << 16);
            }
            *reinterpret_cast<uint4*>(q + swz(r, c)) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4*>(q + 16384 + swz(r, c)) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
            if (c == 0) rowf[x * 128 + r] = scale_value(static_cast<uint32_t>(e)) * p.scale_log2;
          }
          fence_async();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(q_ready);
      }
      // Probabilities are taken against a reference `ref` near the row's running
      // maximum (2^(y - ref), y in log2 units): its first score's half step's
      // maximum, moved up after a step that went more than 8 past it, for the
      // next one.  Only where a row sees its first key, or a score is more than 24
      // past `ref` (sums and O stay far inside 32 bits up to there), is a half
      // step done again, and `ref` moves first: by a whole number, so that
      // what P has of the step's first half scales exactly.  So the maximum is
      // never waited for.  (How far, and why a few moves are enough: paged_math.h.)
      float ref = 0.f, l = 0.f, alpha = 1.f;
      bool started = false, pend = false;  // a key seen; O to be scaled by alpha
      auto rescale = [&](float a) {
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          float o[32];
          uint32_t ob[32];
          tmem_ld32(to + static_cast<uint32_t>(c), o);
          tmem_ld_wait<32>(o);
#pragma unroll
          for (int k = 0; k < 32; ++k) ob[k] = __float_as_uint(o[k] * a);
          tmem_st32(to + static_cast<uint32_t>(c), ob);
        }
        tmem_st_wait();
      };
      for (int i = 0; i < mine; ++i) {
        const int st = one ? 2 * i + x : i;
        const int key0 = (w.c0 + st) * kStep;
        const bool edge = key0 + kStep > lo;
        ok = ok && mbar_wait(&s_full[x], static_cast<uint32_t>(done + i) & 1u, p.limit_ns, abort);
        const int ks = (kn + st) % L::kFs;
        if constexpr (E4M3)
          ok = ok && mbar_wait(&kfact[ks], static_cast<uint32_t>((kn + st) / L::kFs) & 1u, p.limit_ns, abort);
        ok = __all_sync(0xffffffffu, ok);
        if (E4M3 && i == 0) f = rowf[(one ? 0 : x * 128) + row];  // there before S was begun
        tc_fence_after();
        // S(i) is complete, so P V of the step before it is: O may be rescaled
        if (__any_sync(0xffffffffu, pend)) rescale(pend ? alpha : 1.f);
        pend = false;
        // scores 32 c .. 32 c + 31, once loaded: times their factors, which are
        // multiplied first, as either may be past what the other brings back into
        // range; and what the row does not see
        auto finish = [&](int c, float* s) {
          if constexpr (E4M3) {
            const float4* kf = reinterpret_cast<const float4*>(smem + L::kKf + (ks * kStep + 32 * c) * 4);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float4 z = kf[k];
              mul2(z.x, z.y, f, f);
              mul2(z.z, z.w, f, f);
              mul2(s[4 * k], s[4 * k + 1], z.x, z.y);
              mul2(s[4 * k + 2], s[4 * k + 3], z.z, z.w);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 32; k += 2) mul2(s[k], s[k + 1], f, f);
          }
          if (edge) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (key0 + 32 * c + k >= lim) s[k] = -INFINITY;
          }
        };
        float sum = 0.f, top = -INFINITY;
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {  // 64 keys; few instructions, that they stay cached
          uint32_t pk[32];
          float hs, ht;
          for (int moves = 0;; ++moves) {
            float s[2][32];
            tmem_ld32(ts + static_cast<uint32_t>(64 * h), s[0]);
            tmem_ld_wait<32>(s[0]);
            tmem_ld32(ts + static_cast<uint32_t>(64 * h + 32), s[1]);
            float a0 = 0.f, a1 = 0.f, b0 = 0.f, b1 = 0.f, t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float* v = s[c];
              finish(2 * h + c, v);
#pragma unroll
              for (int k = 0; k < 32; k += 4) {
                add2(v[k], v[k + 1], -ref, -ref);
                add2(v[k + 2], v[k + 3], -ref, -ref);
                t0 = max3(t0, v[k], v[k + 1]);
                t1 = max3(t1, v[k + 2], v[k + 3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[k + e] = ex2(v[k + e]);
                add2(a0, a1, v[k], v[k + 1]);
                add2(b0, b1, v[k + 2], v[k + 3]);
                pk[16 * c + k / 2] = bf16x2(v[k], v[k + 1]);
                pk[16 * c + k / 2 + 1] = bf16x2(v[k + 2], v[k + 3]);
              }
              if (c == 0) tmem_ld_wait<32>(s[1]);
            }
            ht = fmaxf(t0, t1);
            hs = (a0 + a1) + (b0 + b1);
            // rows past the tile hold what memory held: they have no say
            const bool again = valid && moves < kPagedMoves && paged_far(ht, started);
            if (!__any_sync(0xffffffffu, again)) break;
            float a = 1.f;
            if (again) {
              const float lost = paged_move(ht, ref, started);
              a = ex2(-lost);
              l *= a;
              sum *= a;
              top -= lost;
            }
            if (__any_sync(0xffffffffu, a != 1.f)) {
              if (i > 0) rescale(a);
              if (h == 1) {  // P of the first half: in place, exactly
                const uint32_t a2 = bf16x2(a, a);
                float q[32];
                tmem_st_wait();  // its store, which loads do not wait for by themselves
                tmem_ld32(ts, q);
                tmem_ld_wait<32>(q);
#pragma unroll
                for (int k = 0; k < 32; ++k) pk[k] = mul_bf16x2(__float_as_uint(q[k]), a2);
                tmem_st32(ts, pk);
                tmem_st_wait();
              }
            }
          }
          tmem_st32(ts + static_cast<uint32_t>(32 * h), pk);
          // The sum is of the unrounded probabilities, but has the half step's largest
          // as P has it: a row that looks at one key has that key's values, exactly, and
          // the error of all outputs is a tenth less.  (An element that this key has no
          // part in is divided by that rounding, too: 2^-8 of it at most.)
          const float pm = ex2(ht);
          sum += hs + (__uint_as_float(bf16x2(pm, 0.f) << 16) - pm);
          top = fmaxf(top, ht);
        }
        l += sum;
        if (valid && top > 8.f && started) {
          alpha = ex2(-top);
          ref += top;
          l *= alpha;
          pend = true;
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[x]);
      }
      kn += n;
      done += mine;
      if (!ok && lane == 0) gave_up();

      // ---- the item's results
      if (mine > 0) ok = ok && mbar_wait(&o_full[x], static_cast<uint32_t>(outs) & 1u, p.limit_ns, abort);
      ok = __all_sync(0xffffffffu, ok);
      outs += mine > 0 ? 1 : 0;
      tc_fence_after();
      const bool whole = w.whole();
      const int rr = (one ? 0 : x * tile) + row;  // row of the item
      const float tail = pend ? alpha : 1.f;
      float m = l == 0.f ? -INFINITY : ref;
      float2* ml1 = reinterpret_cast<float2*>(smem + L::kMl);
      float4* xo = reinterpret_cast<float4*>(smem + L::kQ + L::kTile);  // 64 columns of stream 1's O
      float wa = 1.f, wb = 0.f;
      if (one) {  // the two streams' rows together: stream 1 hands over
        if (x == 1) ml1[row] = make_float2(m, l);
        named_barrier(1, 256);
        if (x == 0) {
          const float2 z = ml1[row];
          const float mm = fmaxf(m, z.x);
          wa = m == -INFINITY ? 0.f : ex2(m - mm);
          wb = z.x == -INFINITY ? 0.f : ex2(z.x - mm);
          l = l * wa + z.y * wb;
          m = mm;
        }
      }
      const bool any_bad = *reinterpret_cast<volatile int*>(&s_bad[items % kBads]) != 0;
      const int* badp = bad + (items % kBads) * 3 * D;
      const float inv = !whole ? 1.f : l > 0.f || l != l ? 1.f / l : 0.f;  // a row that sees nothing: zeros
      // Rows go out through shared memory, a warp's 32 where its part of q lay
      // (every S of the item is complete), so that a store is of whole rows:
      // straight from the row's lane, 16 bytes a row, they took 9 to 18 thousand
      // cycles an item.
      const int i_tok = paged_row(p, m_row), h_grp = m_row - i_tok * p.group;
      const long long at = whole ? (static_cast<long long>(w.s.r0 + i_tok) * p.Hq + w.h * p.group + h_grp) * D
                                 : (static_cast<long long>(w.part()) * p.part_rows + rr) * D;
      uint8_t* stage = smem + L::kQ + (one ? 0 : x * L::kTile) + (warp & 3) * 8192;
      const uint32_t live = __ballot_sync(0xffffffffu, valid && mine > 0 && !*abort);
      // what a row sees of values that are not finite, added: infinities, or NaN
      auto blot = [&](int d) {
        float z = 0.f;
        if (lim > badp[D + d]) z += INFINITY;
        if (lim > badp[2 * D + d]) z -= INFINITY;
        return lim > badp[d] ? NAN : z;
      };
      // 16-byte pieces of 256-byte rows: piece c of row r at c ^ (r % 16)
      auto put = [&](int c, uint4 v) { *reinterpret_cast<uint4*>(stage + lane * 256 + ((c ^ (lane & 15)) << 4)) = v; };
      auto send = [&](auto&& to_global) {
        __syncwarp();
#pragma unroll 4
        for (int k = 0; k < 16; ++k) {
          const int r = 2 * k + (lane >> 4), c = lane & 15;
          const long long o = __shfl_sync(0xffffffffu, at, r);
          if ((live >> r) & 1u) to_global(o, c, *reinterpret_cast<const uint4*>(stage + r * 256 + ((c ^ (r & 15)) << 4)));
        }
        __syncwarp();
      };
#pragma unroll 1
      for (int hf = 0; hf < D / 64; ++hf) {  // few instructions: they are fetched once an item
        if (one) {
          if (x == 1 && mine > 0) {
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
              float o[32];
              tmem_ld32(to + static_cast<uint32_t>(hf * 64 + c), o);
              tmem_ld_wait<32>(o);
#pragma unroll
              for (int k = 0; k < 32; k += 4)
                xo[((c + k) / 4) * 128 + row] =
                    make_float4(o[k] * tail, o[k + 1] * tail, o[k + 2] * tail, o[k + 3] * tail);
            }
          }
          named_barrier(1, 256);
        }
        if ((!one || x == 0) && mine > 0) {
#pragma unroll 1
          for (int c = 0; c < 64; c += 32) {
            float o[32];
            tmem_ld32(to + static_cast<uint32_t>(hf * 64 + c), o);
            tmem_ld_wait<32>(o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] *= tail;
            if (one && n > 1) {
#pragma unroll
              for (int k = 0; k < 32; k += 4) {
                const float4 z = xo[((c + k) / 4) * 128 + row];
                o[k] = fmaf(z.x, wb, o[k] * wa);
                o[k + 1] = fmaf(z.y, wb, o[k + 1] * wa);
                o[k + 2] = fmaf(z.z, wb, o[k + 2] * wa);
                o[k + 3] = fmaf(z.w, wb, o[k + 3] * wa);
              }
            }
            if (any_bad) {
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] += blot(hf * 64 + c + k);
            }
            if (whole) {
#pragma unroll
              for (int k = 0; k < 32; k += 8)
                put((hf * 64 + c + k) / 8,
                    make_uint4(bf16x2(o[k] * inv, o[k + 1] * inv), bf16x2(o[k + 2] * inv, o[k + 3] * inv),
                               bf16x2(o[k + 4] * inv, o[k + 5] * inv), bf16x2(o[k + 6] * inv, o[k + 7] * inv)));
            } else {
#pragma unroll
              for (int k = 0; k < 32; k += 4)
                put((c + k) / 4, make_uint4(__float_as_uint(o[k]), __float_as_uint(o[k + 1]), __float_as_uint(o[k + 2]),
                                            __float_as_uint(o[k + 3])));
            }
          }
          if (!whole)
            send([&](long long o, int c, uint4 v) { *reinterpret_cast<uint4*>(p.part + o + hf * 64 + c * 4) = v; });
        }
        if (one) named_barrier(1, 256);
      }
      if (whole && (!one || x == 0))
        send([&](long long o, int c, uint4 v) { *reinterpret_cast<uint4*>(p.out + o + c * 8) = v; });
      if (!whole && valid && (!one || x == 0))
        *reinterpret_cast<float2*>(p.part_ml + (static_cast<long long>(w.part()) * p.part_rows + rr) * 2) =
            make_float2(m, l);
      tc_fence_before();
      fence_async();  // rows and exchange lay where q is loaded
      __syncwarp();
      if (lane == 0) {
        if (mine > 0) mbar_arrive(&o_free[x]);
        mbar_arrive(q_empty);
      }
      ++items;
    } while (w.next(p));
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 13) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <int D, bool E4M3>
cudaError_t configure() {
  return cudaFuncSetAttribute(paged_tc_kernel<D, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, Map<D, E4M3>::kDyn);
}

}  // namespace

cudaError_t paged_tc_configure() {
  cudaError_t e;
  if ((e = configure<128, false>()) != cudaSuccess) return e;
  return configure<128, true>();
}

cudaError_t launch_paged_tc(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p,
                            bool e4m3, bool one, int sms, cudaStream_t st) {
  if (e4m3)
    return paged_launch(paged_tc_kernel<128, true>, sms, kThreads, Map<128, true>::kDyn, st, q, k, v, p, one ? 1 : 0);
  return paged_launch(paged_tc_kernel<128, false>, sms, kThreads, Map<128, false>::kDyn, st, q, k, v, p, one ? 1 : 0);
}

}  // namespace ebd
