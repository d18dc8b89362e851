// Attention over the paged K/V cache with few query rows per K/V head (single
// tokens, short windows): o_i = sum_j p_ij v_j / sum_j p_ij with p_ij =
// exp2(c q_i k_j - m_i), c = scale * log2 e, over the keys j that row i sees.
//
// A tile is up to 16, 32 or 64 packed rows (row of the sequence, query head of
// the group) of one sequence and K/V head.  Each CTA takes an equal share of
// all tiles' chunks of 64 keys (paged.h).
//   warp 4: loads.  The rows of q, and per chunk K and V as TMA boxes of a
//     page (or a chunk's part of it), each operand into a slot of one ring.
//   warps 0-3: the scores of a quarter of every chunk's keys each; the probabilities
//     meet in shared memory, and each warp multiplies all of them with D / 4
//     columns of V.  A warp's output is then D / 4 columns, not D, which keeps
//     a tile of 32 rows within the registers of two to four CTAs per SM, and
//     no outputs have to meet when a tile ends.  One barrier per chunk.
// Products run on mma.sync with fp32 sums.  The order of the contraction over
// D is free, as long as q and k share it: a lane takes its K in 16-byte pieces
// as they lie in memory, without ldmatrix.
//
// 8-bit cache.  Codes become f16, exactly and in one instruction a pair (an
// e4m3 mma.sync is these conversions too, besides as many again for q).  q
// becomes f16 after its row is scaled by a power of two so that its largest
// element is in [2^14, 2^15): elements above 2^-29 of that are exact.  The key's
// scale, a power of two, multiplies the score; that of a value's row multiplies
// its probability, relative to the largest scale seen so far (a common power of
// two, E0).  A row's probabilities are taken not against its largest score but
// against its largest product of probability and value's scale, which becomes
// 2^kUp: so f16 holds products down to 2^-31 of the row's own largest, whatever
// other keys' values are (scores past 2^22: paged_math.h).  The sum is of the same
// probabilities without the scales, in 32 bits: scales count as 2^-kSpan E0 at
// least in that maximum, and where E0 rises the reference falls no further than
// leaves the sum below 2^kSum.  O is multiplied by E0's power at the end.
// P is rounded to f16 (bf16 where the cache is); its sum is of the unrounded
// values.
//
// The running maximum moves only when a score (a product) exceeds it by more than
// 8 (log2 units), so that exp2 stays below 256 and most chunks rescale nothing.
//
// Measured, 128-wide heads: 64 tokens over ~4096 8-bit keys, 28 / 4 heads, 49.9 us
// (207 MB: at the HBM rate once it streams; four CTAs per SM; with two 12 % more);
// 16 tokens over ~2011 bf16 keys, 32 heads, 68 us (5.8 TB/s, the HBM rate); 64
// windows of 32 rows over ~1056 8-bit keys, 32 heads, 136 us (3.25 TB/s: latencies
// and issue, 1130 cycles a chunk and SM, of which its MMAs are 518; three CTAs per
// SM, with four 13 % more, with two 43 %).
#include <cuda_fp16.h>
#include <type_traits>

#include "paged.h"
#include "paged_math.h"
#include "ptx.cuh"

namespace ebd {

namespace {

constexpr int kThreads = 160;
// Keys of a share, at least: of small calls (1 to 16 sequences of 1 to 32 rows; 32 /
// 32, 28 / 4 and 4 / 4 heads; both caches) over 530 to 3000 keys, 64, 128, 256 and
// 384 take 1.054, 1.002, 1.027 and 1.093 times as long as 192, in the geometric mean
// of 532 calls.  By length 128 and 192 take turns, as chunks divide: 192 is 8 %
// slower at 600 to 640 and 1000 keys, 7 to 11 % faster at 530 to 560 and 900.
constexpr int kLeastKeys = 192;
constexpr int kJoinRows = 4;        // rows of a joining warp
constexpr int kNever = 0x7fffffff;
constexpr float kUp = kPagedUp;     // 8-bit caches: log2 of a row's largest product (2^15 until its reference moves)
constexpr int kSpan = 90;           // and of the scales' span that its reference follows
constexpr float kSum = 100.f;       // and of a lane's sum of probabilities, past which the reference moves

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}
// D += A B, m16n8k16, f16 (bf16) inputs, fp32 accumulators
template <bool F16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// the values of four e4m3 codes, in pairs
__device__ __forceinline__ void e4m3x4_f16(uint32_t c, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}"
      : "=r"(lo), "=r"(hi)
      : "r"(c));
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// 2^(e - 127) of an exponent byte
__device__ __forceinline__ float scale_value(uint32_t e) { return __uint_as_float(max(e << 23, 1u << 22)); }

// CTAs per SM: as many as registers and a ring of two chunks or more allow.
constexpr int ctas_per_sm(bool e4m3, int mb) { return !e4m3 ? 2 : mb == 1 ? 4 : mb == 2 ? 3 : 2; }
// q's fragments of one row block stay in registers where these suffice
constexpr bool q_in_registers(bool e4m3, int mb) { return !e4m3 && mb == 1; }

// Shared memory (offsets from a 1024-byte aligned base).
template <int D, bool E4M3, int MB>
struct Map {
  static constexpr int T = 16 * MB;                               // tile rows
  static constexpr int CH = 1 << kPagedChunkLog2;
  static constexpr uint32_t kOp = CH * D * (E4M3 ? 1 : 2);       // K or V of a chunk
  static constexpr uint32_t kQRow = 2 * D + 16;                   // padded: rows in distinct banks
  static constexpr uint32_t kFrag = q_in_registers(E4M3, MB) ? 0 : T * 2 * D;  // q as fragments
  static constexpr uint32_t kAll = (ctas_per_sm(E4M3, MB) == 4 ? 56 : ctas_per_sm(E4M3, MB) == 3 ? 75 : 113) * 1024 - 1024;
  static constexpr uint32_t kFixed = T * kQRow + kFrag + 4 * T * CH + 3 * D * 4 + 2 * 4 * T * 4 + 4 * T * 4 +
                                     T * 4 + 640;
  static constexpr uint32_t kSlotBytes = kOp + (E4M3 ? CH : 0) + 16;
  static constexpr int S = (kAll - kFixed) / kSlotBytes > 16 ? 16 : (kAll - kFixed) / kSlotBytes;  // ring slots
  static constexpr uint32_t kRing = 0;
  static constexpr uint32_t kP = kRing + S * kOp;                 // [2][64-key blocks][T][128 B]: P of a chunk
  static constexpr uint32_t kScale = kP + 4 * T * CH;
  static constexpr uint32_t kQ = kScale + S * (E4M3 ? CH : 0);
  static constexpr uint32_t kQF = kQ + T * kQRow;                 // [MB][D / 16][32 lanes][16 B]
  static constexpr uint32_t kBad = kQF + kFrag;                   // [3][D]
  static constexpr uint32_t kXl = kBad + 3 * D * 4;               // [2][4][T] sums of the warps
  static constexpr uint32_t kXm = kXl + 2 * 4 * T * 4;            // [4][T] maxima of the warps
  static constexpr uint32_t kRowF = kXm + 4 * T * 4;                     // [T] score factors of the rows
  static constexpr uint32_t kBar = kRowF + T * 4;
  static constexpr int kNBar = 2 * S + 2;
  static constexpr uint32_t kPlan = kBar + kNBar * 8;
  static constexpr uint32_t kMisc = kPlan + sizeof(PagedStart) + 8 * 4;
  static constexpr uint32_t kBytes = kMisc + 16;
  static constexpr uint32_t kDyn = kBytes + 1024;
  static_assert(S >= 3 && kBytes <= kAll && (kP % 1024) == 0 && (kQ % 16) == 0, "shared memory");
};

// What the chunks of a piece need: constant over a piece, or carried along.
template <int MB>
struct Rows {
  float f[MB][2];     // 8-bit caches: the scores' power of two of rows g and g + 8 of each block
  float m[MB][2];     // what is taken off the scores: the running maximum, or near it
  float l[MB][2];     // sum of this lane's probabilities
};

__device__ __forceinline__ bool barrier_or(uint32_t id, uint32_t n, bool pred) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, %3, p;\n"
      " selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)pred), "r"(id), "r"(n)
      : "memory");
  return r != 0;
}

template <int D, bool E4M3, int MB>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(E4M3, MB))
    paged_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                      const PagedParams p) {
  using L = Map<D, E4M3, MB>;
  constexpr int T = L::T, S = L::S, CH = L::CH;
  constexpr int NK = CH / 32;                 // key tiles of a warp
  constexpr int NT = D / 32;                  // output column tiles of a warp
  constexpr int NJ = E4M3 ? D / 64 : D / 32;  // 16-byte pieces of a K row per lane
  constexpr int NB = E4M3 ? 1 : D / 64;       // boxes of 128-byte rows across D
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);  // an offset: accesses stay LDS and STS
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);
  uint64_t* empty = full + S;
  uint64_t* qfull = empty + S;
  uint64_t* qempty = qfull + 1;
  PagedStart* plan = reinterpret_cast<PagedStart*>(smem + L::kPlan);
  auto& scan = *reinterpret_cast<unsigned(*)[kThreads / 32]>(smem + L::kPlan + sizeof(PagedStart));
  volatile int* abort = reinterpret_cast<volatile int*>(smem + L::kMisc);
  int* s_bad = reinterpret_cast<int*>(smem + L::kMisc + 8);
  int* bad = reinterpret_cast<int*>(smem + L::kBad);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 4);
    }
    mbar_init(qfull, 1);
    mbar_init(qempty, 4);
    *abort = 0;
    *s_bad = 0;
    fence_mbar_init();
  }
  for (int i = tid; i < 3 * D; i += kThreads) bad[i] = kNever;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  paged_plan<kThreads>(p, T, CH, kLeastKeys / CH, plan, scan);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // no tile of this CTA's to be put together, until the thread that says so here
  // has seen its share to the end: a share that is given up leaves no other call's
  if (tid == 128) p.cuts[blockIdx.x] = PagedCut{};
  PagedWalk<T, CH> w;
  if (!w.begin(p, *plan, T)) return;

  if (warp == 4) {
    // ------------------------------------------------------------ loads
    const int np_log = kPagedChunkLog2 - p.box_log2, box = 1 << p.box_log2;
    const int pc = lane & ((1 << np_log) - 1), part = lane >> np_log;
    const int key_in = pc << p.box_log2;
    int n = 0, pieces = 0;
    bool ok = true;
    do {
      const int last = min(w.s.n - 1, paged_row(p, w.t * T + T - 1));
      const int rows = min(T, w.s.n * p.group - w.t * T);
      const int lim = paged_limit(p, w.s, last);
      const int* table = p.page_table + static_cast<long long>(w.b) * p.max_pages;
      // page ids of 32 pages, one per lane; the first while q is seen to
      int win0 = ((w.c0 * CH) >> p.page_log2) & ~31;
      int win = win0 + lane < p.max_pages ? table[win0 + lane] : -1;
      {  // q: rows by lane, zeros past the tile's last
        uint8_t* qd = smem + L::kQ;
        ok = !p.give_up &&
             (pieces == 0 || mbar_wait(qempty, static_cast<uint32_t>(pieces - 1) & 1u, p.limit_ns, abort));
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        for (int i = rows * (D / 8) + lane; i < T * (D / 8); i += 32)
          *reinterpret_cast<uint4*>(qd + (i / (D / 8)) * L::kQRow + (i % (D / 8)) * 16) = make_uint4(0u, 0u, 0u, 0u);
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(qfull, static_cast<uint32_t>(rows) * D * 2);
        __syncwarp();
        for (int r = lane; r < rows; r += 32) {
          const int m = w.t * T + r, i = paged_row(p, m), hl = m - i * p.group;
          bulk_load(qd + r * L::kQRow,
                    p.q + (w.s.r0 + i) * p.q_stride + static_cast<long long>(w.h * p.group + hl) * D, D * 2, qfull);
        }
        ++pieces;
      }
      for (int c = w.c0; c < w.c1 && ok; ++c) {
        const int key = c * CH + key_in;
        const int first = (c * CH) >> p.page_log2;
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
        const int pieces_here = min(max((lim - c * CH + box - 1) >> p.box_log2, 0), 1 << np_log);
        const uint32_t bytes = static_cast<uint32_t>(pieces_here) * box * (E4M3 ? D + 1 : 2 * D);
        const int off = key & ((1 << p.page_log2) - 1);
#pragma unroll
        for (int v = 0; v < 2; ++v, ++n) {
          const int s = n % S;
          ok = ok && (n < S || mbar_wait(&empty[s], static_cast<uint32_t>(n / S - 1) & 1u, p.limit_ns, abort));
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(&full[s], bytes);
          __syncwarp();
          if (mine) {
            uint8_t* d = smem + L::kRing + s * L::kOp;
            if (E4M3 && part == 1)
              bulk_load(smem + L::kScale + s * CH + key_in,
                        (v ? p.v_scale : p.k_scale) +
                            ((static_cast<long long>(page) * p.Hkv + w.h) << p.page_log2) + off,
                        box, &full[s]);
            else
              tma_load_4d(d + part * 8192 + key_in * (E4M3 ? D : 128), v ? &tm_v : &tm_k, &full[s], part * 64, off,
                          w.h, page);
          }
        }
      }
      if (lane == 0 && w.u + (w.c1 - w.c0) >= w.u1) w.leave(p, *plan);
    } while (ok && w.next(p));
    if (!ok) {
      if (lane == 0 && !*abort) {
        *abort = 1;
        atomicCAS(p.status, 0, EBD_ERR_TIMEOUT);
      }
      // the copies in flight land before the CTA can exit
      for (int j = max(0, n - S); j < n; ++j)
        mbar_wait(&full[j % S], static_cast<uint32_t>(j / S) & 1u, p.limit_ns, nullptr);
      if (pieces > 0) mbar_wait(qfull, static_cast<uint32_t>(pieces - 1) & 1u, p.limit_ns, nullptr);
    }
    return;
  }

  // -------------------------------------------------------------- products
  const int g = lane >> 2, t4 = lane & 3;
  const int kb = warp * (CH / 4);  // this warp's keys of a chunk
  float* xm = reinterpret_cast<float*>(smem + L::kXm);
  float* xl = reinterpret_cast<float*>(smem + L::kXl);
  float* rowf = reinterpret_cast<float*>(smem + L::kRowF);
  int nchunk = 0;
  bool ok = true;
  int pieces = 0;
  // ring slots of the next K and the next V; they take turns in the ring
  int kslot = 0, vslot = 1;
  uint32_t kphase = 0, vphase = 0;
  auto step = [](int& slot, uint32_t& phase) {
    slot += 2;
    if (slot >= S) {
      slot -= S;
      phase ^= 1u;
    }
  };
  // A wait that finds its operand there costs 150 cycles, most of them the
  // barrier's answer: asked for ahead (peek), it comes beside other work.
  auto peek = [&](int slot, uint32_t phase) { return mbar_test(&full[slot], phase); };
  auto landed = [&](int slot, uint32_t phase, bool there) {
    ok = ok && (there || mbar_wait(&full[slot], phase, p.limit_ns, abort));
    ok = __all_sync(0xffffffffu, ok);
  };
  bool v_there = false, k_there = false;
  do {
    const int m0 = w.t * T;
    const int mtot = w.s.n * p.group;
    const int rows = min(T, mtot - m0);
    const int lim_lo = paged_limit(p, w.s, paged_row(p, m0));
    const int lim_hi = paged_limit(p, w.s, paged_row(p, m0 + rows - 1));
    const int len = w.s.len;
    const int par = pieces & 1;
    [[maybe_unused]] int E0 = 0;  // exponent byte that values' scales are relative to (O with them)
    const uint8_t* qd = smem + L::kQ;
    Rows<MB> R;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int hi = 0; hi < 2; ++hi) {
        R.f[mb][hi] = 1.f;
        R.m[mb][hi] = -INFINITY;
        R.l[mb][hi] = 0.f;
      }
    // keys before this one are seen by row hi * 8 + g of block mb
    auto limit = [&](int mb, int hi) {
      const int m = m0 + mb * 16 + hi * 8 + g;
      return m < mtot ? paged_limit(p, w.s, paged_row(p, m)) : kNever;
    };
    float o[MB][NT][4];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[mb][j][i] = 0.f;

    ok = ok && mbar_wait(qfull, static_cast<uint32_t>(pieces) & 1u, p.limit_ns, abort);
    ok = __all_sync(0xffffffffu, ok);
    // row r in f16: this lane's pieces of 16 elements, (NJ t4 + j) * 16 and on, as
    // 8 words each; returns the row's score factor
    auto f16_row = [&](int r, uint32_t (&y)[NJ][8]) -> float {
      const uint8_t* q = qd + r * L::kQRow;
      uint32_t x[NJ][8], amax = 0;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 v = *reinterpret_cast<const uint4*>(q + ((NJ * t4 + j) * 2 + i) * 16);
          x[j][4 * i] = v.x;
          x[j][4 * i + 1] = v.y;
          x[j][4 * i + 2] = v.z;
          x[j][4 * i + 3] = v.w;
#pragma unroll
          for (int k = 0; k < 4; ++k) amax = max(amax, max(x[j][4 * i + k] & 0x7FFFu, (x[j][4 * i + k] >> 16) & 0x7FFFu));
        }
      amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      const bool finite = amax < 0x7F80u;
      const uint32_t e = finite ? min(268u - (amax >> 7), 254u) : 127u;  // 2^(e - 127) * |largest| in [2^14, 2^15)
      const float up = __uint_as_float(e << 23);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float a = __uint_as_float(x[j][k] << 16) * up, b = __uint_as_float(x[j][k] & 0xFFFF0000u) * up;
          y[j][k] = finite ? f16x2(a, b) : 0x7FFF7FFFu;  // a row with a value that is not finite has NaN scores
        }
      return scale_value(254u - e);
    };
    // q as fragments: word pairs (2 i, 2 i + 1) of a row's pieces are A registers
    // hi and 2 + hi of contraction step i, in registers or shared memory
    constexpr int QW = E4M3 ? 8 : 4;  // words of a piece of q
    constexpr int KS = D / 16;        // contraction steps: QW / 2 per piece
    constexpr bool QREG = q_in_registers(E4M3, MB);
    uint32_t qa[QREG ? KS : 1][4];
    auto row_words = [&](int r, uint32_t (&y)[NJ][QW]) -> float {
      if constexpr (E4M3) {
        return f16_row(r, y);
      } else {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint4 x = *reinterpret_cast<const uint4*>(qd + r * L::kQRow + ((j >> 1) * 8 + 2 * t4 + (j & 1)) * 16);
          y[j][0] = x.x;
          y[j][1] = x.y;
          y[j][2] = x.z;
          y[j][3] = x.w;
        }
        return 1.f;
      }
    };
    if constexpr (QREG) {
#pragma unroll
      for (int hi = 0; hi < 2; ++hi) {
        uint32_t y[NJ][QW];
        R.f[0][hi] = row_words(hi * 8 + g, y);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          qa[i][hi] = y[i / (QW / 2)][2 * (i % (QW / 2))];
          qa[i][2 + hi] = y[i / (QW / 2)][2 * (i % (QW / 2)) + 1];
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(qempty);
    } else {
      // the warps share the rows, one per 4 lanes at a time
#pragma unroll
      for (int r0 = 0; r0 < (MB == 1 ? 8 : T / 4); r0 += 8) {
        if (MB == 1 && warp > 1) break;
        uint32_t y[NJ][QW];
        const int r = (MB == 1 ? warp * 8 : warp * (T / 4) + r0) + g;
        const float f = row_words(r, y);
        uint32_t* qf = reinterpret_cast<uint32_t*>(smem + L::kQF) + ((r >> 4) * KS * 32 + (r & 7) * 4 + t4) * 4 + ((r >> 3) & 1);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          qf[i * 128] = y[i / (QW / 2)][2 * (i % (QW / 2))];
          qf[i * 128 + 2] = y[i / (QW / 2)][2 * (i % (QW / 2)) + 1];
        }
        if (t4 == 0) rowf[r] = f;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(qempty);
      named_barrier(1, 128);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) R.f[mb][hi] = rowf[mb * 16 + hi * 8 + g];
    }

    // scores of this warp's keys of the chunk in ring slot `slot`, rounded in log2
    // units (paged_math.h), but for a power of two per row in 8-bit caches
    auto scores = [&](int slot, float (&s)[MB][NK][4]) {
      const uint8_t* kd = smem + L::kRing + slot * L::kOp;
      // where there are few, two sums of each, so that MMAs wait less for one another
      constexpr bool TWO = MB * NK < 4;
      [[maybe_unused]] float s2[NK][4];
#pragma unroll
      for (int nt = 0; nt < NK; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s2[nt][i] = 0.f;
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) s[mb][nt][i] = 0.f;
        }
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        uint32_t kw[NK][QW];  // K of the piece, in the words of q's type
#pragma unroll
        for (int nt = 0; nt < NK; ++nt) {
          const int row = kb + nt * 8 + g;
          uint32_t at;
          if (E4M3 && D == 64)
            at = row * 64 + t4 * 16;
          else if (E4M3)
            at = row * 128 + (((2 * t4 + j) ^ g) << 4);
          else
            at = (j >> 1) * 8192 + row * 128 + (((2 * t4 + (j & 1)) ^ g) << 4);
          const uint4 x = *reinterpret_cast<const uint4*>(kd + at);
          const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if constexpr (E4M3)
              e4m3x4_f16(u[k], kw[nt][2 * k], kw[nt][2 * k + 1]);
            else
              kw[nt][k] = u[k];
          }
        }
#pragma unroll
        for (int k = 0; k < QW / 2; ++k) {
          const int i = j * (QW / 2) + k;
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            if constexpr (QREG) {
#pragma unroll
              for (int nt = 0; nt < NK; ++nt) mma<E4M3>(TWO && (i & 1) ? s2[nt] : s[0][nt], qa[i], kw[nt][2 * k], kw[nt][2 * k + 1]);
            } else {
              const uint4 x = *reinterpret_cast<const uint4*>(smem + L::kQF + ((mb * KS + i) * 32 + lane) * 16);
              const uint32_t a[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int nt = 0; nt < NK; ++nt) mma<E4M3>(TWO && (i & 1) ? s2[nt] : s[mb][nt], a, kw[nt][2 * k], kw[nt][2 * k + 1]);
            }
          }
        }
      }
      if constexpr (TWO) {
#pragma unroll
        for (int nt = 0; nt < NK; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[0][nt][i] += s2[nt][i];
      }
      if constexpr (E4M3) {
        const uint8_t* sc = smem + L::kScale + slot * CH + kb;
        float ks[NK][2];
#pragma unroll
        for (int nt = 0; nt < NK; ++nt) {
          const uint32_t two = *reinterpret_cast<const uint16_t*>(sc + nt * 8 + 2 * t4);
          ks[nt][0] = scale_value(two & 0xFFu) * p.scale_log2;
          ks[nt][1] = scale_value(two >> 8) * p.scale_log2;
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nt = 0; nt < NK; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[mb][nt][i] *= ks[nt][i & 1];
      } else {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nt = 0; nt < NK; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[mb][nt][i] = __fmul_rn(s[mb][nt][i], p.scale_log2);
      }
    };

    // probabilities of chunk c into shared memory; EDGE where a key of it is past some row's limit
    auto softmax = [&](int c, auto edge_c, bool fresh, float (&s)[MB][NK][4]) {
      constexpr bool EDGE = decltype(edge_c)::value;
      const int key0 = c * CH;
      [[maybe_unused]] uint32_t ve[NK][2];  // exponents of the values' rows
      if constexpr (EDGE) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          const int lim[2] = {limit(mb, 0), limit(mb, 1)};
#pragma unroll
          for (int nt = 0; nt < NK; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + kb + nt * 8 + 2 * t4 + (i & 1) >= lim[i >> 1]) s[mb][nt][i] = -INFINITY;
        }
      }
      // V of the chunk: waited for here, as its rows' scales go into P
      landed(vslot, vphase, v_there);
      k_there = c + 1 < w.c1 && peek(kslot, kphase);
      if constexpr (E4M3) {
        const uint8_t* sc = smem + L::kScale + vslot * CH + kb;
#pragma unroll
        for (int nt = 0; nt < NK; ++nt) {
          const uint32_t two = *reinterpret_cast<const uint16_t*>(sc + nt * 8 + 2 * t4);
          ve[nt][0] = two & 0xFFu;
          ve[nt][1] = two >> 8;
          if constexpr (EDGE) {  // past what is seen nothing is known of them
            if (key0 + kb + nt * 8 + 2 * t4 >= lim_hi) ve[nt][0] = 0u;
            if (key0 + kb + nt * 8 + 2 * t4 + 1 >= lim_hi) ve[nt][1] = 0u;
          }
        }
      }
      auto value_scale = [&](uint32_t e) {  // a row that is NaN: its codes do not say so to P V
        return e == 255u ? NAN : __uint_as_float(static_cast<uint32_t>(max(static_cast<int>(e) - E0 + 127, 0)) << 23);
      };
      // log2 of a value's scale, as the row's reference counts it: a small integer n
      // as the float n, from 1.5 * 2^23 + n (a conversion would be waited for)
      auto value_log2 = [&](uint32_t e) {
        return __int_as_float(0x4B400000 + max(static_cast<int>(e) - E0, -kSpan)) - 12582912.f;
      };
      uint8_t* pd = smem + L::kP + (nchunk & 1) * T * CH * 2;
      // probabilities against the running references, into shared memory, and their
      // sums; the largest of them (8-bit caches: of their products with scales)
      float ls[MB][2];
      auto log2_score = [&](int mb, int hi, int nt, int e, float add) {
        const float y = s[mb][nt][2 * hi + e];
        return E4M3 ? fmaf(y, R.f[mb][hi], add) : __fadd_rn(y, add);
      };
      auto put_p = [&]() {
        float top = 0.f;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) ls[mb][0] = ls[mb][1] = 0.f;
        [[maybe_unused]] float vs[NK][2];
        if constexpr (E4M3) {
#pragma unroll
          for (int nt = 0; nt < NK; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) vs[nt][e] = value_scale(ve[nt][e]);
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int hi = 0; hi < 2; ++hi) {
            const float sub = R.m[mb][hi] == -INFINITY ? 0.f : R.m[mb][hi];
#pragma unroll
            for (int nt = 0; nt < NK; ++nt) {
              float e0 = ex2(log2_score(mb, hi, nt, 0, -sub)), e1 = ex2(log2_score(mb, hi, nt, 1, -sub));
              ls[mb][hi] += e0 + e1;
              if constexpr (E4M3) {
                // what a row does not see stays out, whatever its scale is
                e0 = EDGE && s[mb][nt][2 * hi] == -INFINITY ? 0.f : e0 * vs[nt][0];
                e1 = EDGE && s[mb][nt][2 * hi + 1] == -INFINITY ? 0.f : e1 * vs[nt][1];
              }
              top = max3(top, e0, e1);
              const int r = mb * 16 + hi * 8 + g;
              const int k8 = warp * NK + nt;  // of the chunk's groups of 8 keys
              *reinterpret_cast<uint32_t*>(pd + (k8 >> 3) * T * 128 + r * 128 + (((k8 & 7) ^ g) << 4) + t4 * 4) =
                  E4M3 ? f16x2(e0, e1) : bf16x2(e0, e1);
            }
          }
        return top;
      };
      bool raise = fresh;
      if (!fresh) {
        raise = put_p() > (E4M3 ? 32768.f : 256.f);
        if constexpr (E4M3) {  // scales far past E0 (a NaN row's byte among them: rare enough)
          uint32_t emax = 0;
#pragma unroll
          for (int nt = 0; nt < NK; ++nt) emax = max(emax, max(ve[nt][0], ve[nt][1]));
          raise = raise || static_cast<int>(emax) > E0 + 7;
          // keys whose values are small or zero: their products do not tell, and
          // infinity times such a scale would be NaN
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) raise = raise || fmaxf(ls[mb][0], ls[mb][1]) > 0x1p100f;
        }
      }
      if (barrier_or(1, 128, raise)) {
        // new running maxima, of all warps' scores, and E0
        [[maybe_unused]] float dv[NK][2];
        float down = 1.f, shift = 0.f;
        if constexpr (E4M3) {
          static_assert(CH == 64, "two exponents per lane");
          const uint32_t two = *reinterpret_cast<const uint16_t*>(smem + L::kScale + vslot * CH + 2 * lane);
          uint32_t a = two & 0xFFu, b = two >> 8;
          if (a == 255u || (EDGE && key0 + 2 * lane >= lim_hi)) a = 0u;
          if (b == 255u || (EDGE && key0 + 2 * lane + 1 >= lim_hi)) b = 0u;
          const int e = max(static_cast<int>(__reduce_max_sync(0xffffffffu, max(a, b))), E0);
          down = __uint_as_float(static_cast<uint32_t>(max(E0 - e + 127, 0)) << 23);
          shift = static_cast<float>(min(e - E0, kSpan));
          E0 = e;
#pragma unroll
          for (int nt = 0; nt < NK; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) dv[nt][k] = value_log2(ve[nt][k]);
        }
        // the largest of this warp's keys' scores (8-bit caches: with their values'
        // scales, but for the scores themselves where those are coarse) by row;
        // says whether any is
        auto largest = [&](auto plain_c) {
          constexpr bool PLAIN = decltype(plain_c)::value;
          bool any = false;
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
              float x = -INFINITY;
              if (E4M3 && !PLAIN) x = R.m[mb][hi] + (lg2(R.l[mb][hi]) + (kUp - kSum));  // -inf: no sum yet
#pragma unroll
              for (int nt = 0; nt < NK; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) x = fmaxf(x, log2_score(mb, hi, nt, e, E4M3 && !PLAIN ? dv[nt][e] : 0.f));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
              any = any || fabsf(x) >= kPagedCoarse;  // (-inf with them: then nothing changes)
              float* at = xm + warp * T + mb * 16 + hi * 8 + g;
              if (t4 == 0 && (!PLAIN || paged_coarse(*at))) *at = x;
            }
          return any;
        };
        const bool coarse = largest(std::false_type{});
        if constexpr (E4M3) {
          if (barrier_or(1, 128, coarse)) {
            largest(std::true_type{});
            named_barrier(1, 128);
          }
        } else {
          named_barrier(1, 128);
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int hi = 0; hi < 2; ++hi) {
            const float* q = xm + mb * 16 + hi * 8 + g;
            const float top = fmaxf(fmaxf(q[0], q[T]), fmaxf(q[2 * T], q[3 * T]));
            const float mn = E4M3 ? paged_product_ref(R.m[mb][hi] - shift, top) : fmaxf(R.m[mb][hi], top);
            const float alpha = mn == R.m[mb][hi] ? 1.f : ex2(R.m[mb][hi] - mn);  // 0 from -inf
            R.m[mb][hi] = mn;
            R.l[mb][hi] *= alpha;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              o[mb][j][2 * hi] *= alpha * down;
              o[mb][j][2 * hi + 1] *= alpha * down;
            }
          }
        put_p();
        named_barrier(1, 128);
      }
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) R.l[mb][hi] += ls[mb][hi];
    };

    // P V of chunk c: this warp's D / 4 columns; and the next chunk's scores, whose
    // MMAs fill the gaps between these
    auto values = [&](int c, auto edge_c, float (&s)[MB][NK][4]) {
      constexpr bool EDGE = decltype(edge_c)::value;
      const int key0 = c * CH;
      const bool more = c + 1 < w.c1;
      if (more) landed(kslot, kphase, k_there);
      scores(kslot, s);  // of the last chunk, what the slot holds: not used
      const uint8_t* vd = smem + L::kRing + vslot * L::kOp;
      const uint8_t* pd = smem + L::kP + (nchunk & 1) * T * CH * 2;
      // an element of a key that some row does not see, and that is not finite:
      // kept out of the product and noted, for the rows that do see it (8-bit
      // rows say so by their scale, above)
      [[maybe_unused]] const bool scrub = EDGE && p.causal;
      [[maybe_unused]] auto note = [&](int key, int d, int kind) {
        atomicMin(&bad[kind * D + d], key);
        *reinterpret_cast<volatile int*>(s_bad) = 1;
      };
      const uint32_t pb = smem_u32(pd);
#pragma unroll
      for (int ks = 0; ks < CH / 16; ++ks) {
        if (EDGE && key0 + ks * 16 >= lim_hi) break;
        uint32_t a[MB][4];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          const int row = mb * 16 + (lane & 15);
          ldsm_x4(pb + (ks >> 2) * T * 128 + row * 128 + (((2 * (ks & 3) + (lane >> 4)) ^ (lane & 7)) << 4), a[mb][0],
                  a[mb][1], a[mb][2], a[mb][3]);
        }
        if constexpr (E4M3) {
          uint32_t v[2][2];  // [nt][e]: NT bytes of key ks * 16 + nt * 8 + 2 t4 + e
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int row = ks * 16 + nt * 8 + 2 * t4 + e;
              const int d = warp * (D / 4) + g * NT;
              if constexpr (D == 128)
                v[nt][e] = *reinterpret_cast<const uint32_t*>(vd + row * 128 + (((d >> 4) ^ (row & 7)) << 4) + (d & 15));
              else
                v[nt][e] = *reinterpret_cast<const uint16_t*>(vd + row * 64 + d);
              if constexpr (EDGE) {
                const int key = key0 + row;
                // codes of a NaN row: the probabilities say it, where the row is seen
                const uint32_t nan = ((v[nt][e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
                v[nt][e] &= ~((nan >> 7) * 0xFFu);
                if (key >= len) v[nt][e] = 0u;
              }
            }
#pragma unroll
          for (int hf = 0; hf < NT / 2; ++hf) {
            uint32_t b[2][2];  // [column tile 2 hf + .][nt]
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)  // bytes (key 0, d), (key 1, d), (key 0, d + 1), (key 1, d + 1)
              e4m3x4_f16(__byte_perm(v[nt][0], v[nt][1], hf ? 0x7362 : 0x5140), b[0][nt], b[1][nt]);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int mb = 0; mb < MB; ++mb) mma<true>(o[mb][2 * hf + q], a[mb], b[q][0], b[q][1]);
          }
        } else {
          const uint32_t vb = smem_u32(vd);
          // matrices of an ldmatrix: keys 0-7 and 8-15 of one column tile, then of the next
          const int vrow = ks * 16 + (lane & 15);
#pragma unroll
          for (int j = 0; j < NT; j += 2) {
            uint32_t b[4];
            const int ct = warp * NT + j;  // column tile
            ldsm_x4_t(vb + (ct >> 3) * 8192 + vrow * 128 + ((((ct & 7) + (lane >> 4)) ^ (lane & 7)) << 4), b[0], b[1],
                      b[2], b[3]);
            if constexpr (EDGE) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  const int key = key0 + ks * 16 + (i & 1) * 8 + 2 * t4 + e;
                  const uint32_t x = (b[i] >> (16 * e)) & 0xFFFFu;
                  bool drop = key >= len;
                  if (!drop && scrub && key >= lim_lo && (x & 0x7F80u) == 0x7F80u) {
                    note(key, (ct + (i >> 1)) * 8 + g, (x & 0x7Fu) ? 0 : (x & 0x8000u) ? 2 : 1);
                    drop = true;
                  }
                  if (drop) b[i] &= e ? 0x0000FFFFu : 0xFFFF0000u;
                }
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
              mma<false>(o[mb][j], a[mb], b[0], b[1]);
              mma<false>(o[mb][j + 1], a[mb], b[2], b[3]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&empty[vslot]);
        if (more) mbar_arrive(&empty[kslot]);
      }
      step(vslot, vphase);
      v_there = more && peek(vslot, vphase);
      if (more) step(kslot, kphase);
      ++nchunk;
    };

    float s[MB][NK][4];
    landed(kslot, kphase, false);
    scores(kslot, s);
    v_there = peek(vslot, vphase);
    __syncwarp();
    if (lane == 0) mbar_arrive(&empty[kslot]);
    step(kslot, kphase);
    for (int c = w.c0; c < w.c1; ++c) {
      if ((c + 1) * CH > lim_lo) {
        softmax(c, std::true_type{}, c == w.c0, s);
        values(c, std::true_type{}, s);
      } else {
        softmax(c, std::false_type{}, c == w.c0, s);
        values(c, std::false_type{}, s);
      }
    }
    if (!ok && lane == 0 && !*abort) {
      *abort = 1;
      atomicCAS(p.status, 0, EBD_ERR_TIMEOUT);
    }
    ++pieces;

    // ---- results: this warp's columns; the rows' sums are of all four warps
    float* wl = xl + par * 4 * T;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int hi = 0; hi < 2; ++hi) {
        float l = R.l[mb][hi];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        if (t4 == 0) wl[warp * T + mb * 16 + hi * 8 + g] = l;
      }
    named_barrier(1, 128);
    const bool whole = w.whole();
    const bool any_bad = *reinterpret_cast<volatile int*>(s_bad) != 0;
    float* part = p.part + static_cast<long long>(w.part()) * p.part_rows * D;
    float* part_ml = p.part_ml + static_cast<long long>(w.part()) * p.part_rows * 2;
    if (!*abort) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const int r = mb * 16 + hi * 8 + g;
          if (r >= rows) continue;
          const float l = (wl[r] + wl[T + r]) + (wl[2 * T + r] + wl[3 * T + r]);
          float inv = !whole ? 1.f : l > 0.f || l != l ? 1.f / l : 0.f;  // a row that sees nothing: zeros
          // an 8-bit cache's O is relative to E0: a scale past 1 goes into the divisor,
          // as O may be as small as the sum is large
          const float e0 = E4M3 ? scale_value(static_cast<uint32_t>(E0)) : 1.f;
          if (E4M3 && e0 > 1.f) inv *= e0;
          const float rest = e0 > 1.f ? 1.f : e0;
          // this lane's elements of the row: an 8-bit cache's NT columns of
          // fragment column 2 t4, then those of 2 t4 + 1, which follow on
          // them; a bf16 cache's columns 2 t4 and 2 t4 + 1 of each tile
          float x[2 * NT];
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float z = o[mb][j][2 * hi + e] * inv;
              x[E4M3 ? e * NT + j : 2 * j + e] = E4M3 ? z * rest : z;
            }
          if (any_bad) {
            const int lim = limit(mb, hi);
#pragma unroll
            for (int k = 0; k < 2 * NT; ++k) {
              const int d = warp * (D / 4) + (E4M3 ? 2 * NT * t4 + k : (k >> 1) * 8 + 2 * t4 + (k & 1));
              if (lim > bad[D + d]) x[k] += INFINITY;
              if (lim > bad[2 * D + d]) x[k] -= INFINITY;
              if (lim > bad[d]) x[k] = NAN;
            }
          }
          const int m = m0 + r, i = paged_row(p, m), h = m - i * p.group;
          __nv_bfloat16* od = p.out + (static_cast<long long>(w.s.r0 + i) * p.Hq + w.h * p.group + h) * D + warp * (D / 4);
          float* pd = part + r * D + warp * (D / 4);
          if constexpr (E4M3) {
            if (whole) {
#pragma unroll
              for (int k = 0; k < NT; k += 2)
                *reinterpret_cast<uint2*>(od + 2 * NT * t4 + 2 * k) =
                    make_uint2(bf16x2(x[2 * k], x[2 * k + 1]), bf16x2(x[2 * k + 2], x[2 * k + 3]));
            } else {
#pragma unroll
              for (int k = 0; k < 2 * NT; k += 4)
                *reinterpret_cast<float4*>(pd + 2 * NT * t4 + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
            }
          } else {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              if (whole)
                *reinterpret_cast<uint32_t*>(od + j * 8 + 2 * t4) = bf16x2(x[2 * j], x[2 * j + 1]);
              else
                *reinterpret_cast<float2*>(pd + j * 8 + 2 * t4) = make_float2(x[2 * j], x[2 * j + 1]);
            }
          }
          if (!whole && warp == 0 && t4 == 0) *reinterpret_cast<float2*>(part_ml + 2 * r) = make_float2(R.m[mb][hi], l);
        }
    }
    if (any_bad) {
      named_barrier(1, 128);
      for (int i = tid; i < 3 * D; i += 128) bad[i] = kNever;
      if (tid == 0) *s_bad = 0;
      named_barrier(1, 128);
    }
  } while (w.next(p));
}

// The parts of the tile that CTA blockIdx.x of the attention begins, put
// together in order: kJoinRows rows per warp, their loads all in flight, a lane
// per D / 32 columns, so that a part's row is one load.
template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedParams p) {
  constexpr int V = D / 32, RB = kJoinRows;
  const int lane = threadIdx.x & 31;
  const int r0 = (blockIdx.y * 8 + (threadIdx.x >> 5)) * RB;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the attention's results
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const PagedCut cut = p.cuts[blockIdx.x];
  if (cut.parts == 0 || r0 >= cut.rows) return;
  auto part = [&](int k) { return static_cast<long long>(k == 0 ? 2 * cut.first + 1 : 2 * (cut.first + k)) * p.part_rows; };
  float mx[RB], l[RB], acc[RB][V];
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    mx[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) acc[i][j] = 0.f;
  }
  auto row = [&](int i) { return min(r0 + i, cut.rows - 1); };
  for (int k0 = 0; k0 < cut.parts; k0 += 32) {
    // with the new parts the maximum may rise; -inf: a part that the row sees nothing of
    float2 ml[RB];
    float wgt[RB];
    const bool in = k0 + lane < cut.parts;
#pragma unroll
    for (int i = 0; i < RB; ++i)
      ml[i] = in ? __ldcg(reinterpret_cast<const float2*>(p.part_ml + (part(k0 + lane) + row(i)) * 2))
                 : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      float x = ml[i].x;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
      x = fmaxf(x, mx[i]);
      const float f = mx[i] == -INFINITY ? 0.f : ex2(mx[i] - x);
      mx[i] = x;
      l[i] *= f;
#pragma unroll
      for (int j = 0; j < V; ++j) acc[i][j] *= f;
      wgt[i] = ml[i].x == -INFINITY ? 0.f : ex2(ml[i].x - x);
      l[i] = fmaf(wgt[i], ml[i].y, l[i]);
    }
    const int n = min(32, cut.parts - k0);
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
      const float* z = p.part + part(k0 + k) * D + lane * V;
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const float wk = __shfl_sync(0xffffffffu, wgt[i], k);
        if constexpr (V == 4) {
          const float4 x = __ldcg(reinterpret_cast<const float4*>(z + row(i) * D));
          acc[i][0] = fmaf(wk, x.x, acc[i][0]);
          acc[i][1] = fmaf(wk, x.y, acc[i][1]);
          acc[i][2] = fmaf(wk, x.z, acc[i][2]);
          acc[i][3] = fmaf(wk, x.w, acc[i][3]);
        } else {
          const float2 x = __ldcg(reinterpret_cast<const float2*>(z + row(i) * D));
          acc[i][0] = fmaf(wk, x.x, acc[i][0]);
          acc[i][1] = fmaf(wk, x.y, acc[i][1]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RB; ++i) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
    if (r0 + i >= cut.rows) break;
    const float inv = l[i] > 0.f || l[i] != l[i] ? 1.f / l[i] : 0.f;
    const int m = cut.m0 + r0 + i, n = paged_row(p, m), h = m - n * p.group;
    __nv_bfloat162* od = reinterpret_cast<__nv_bfloat162*>(
        p.out + (static_cast<long long>(cut.r0 + n) * p.Hq + cut.h * p.group + h) * D + lane * V);
#pragma unroll
    for (int k = 0; k < V / 2; ++k) od[k] = __floats2bfloat162_rn(acc[i][2 * k] * inv, acc[i][2 * k + 1] * inv);
  }
}

template <int D, bool E4M3, int MB>
cudaError_t configure() {
  return cudaFuncSetAttribute(paged_attn_kernel<D, E4M3, MB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              Map<D, E4M3, MB>::kDyn);
}
template <int D, bool E4M3>
cudaError_t launch(const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p, int mb, int sms, cudaStream_t st) {
  auto go = [&](auto c) {
    constexpr int MB = decltype(c)::value;
    return paged_launch(paged_attn_kernel<D, E4M3, MB>, sms * ctas_per_sm(E4M3, MB), kThreads, Map<D, E4M3, MB>::kDyn, st,
                        k, v, p);
  };
  if (mb == 1) return go(std::integral_constant<int, 1>{});
  if (mb == 2) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}

}  // namespace

cudaError_t paged_configure() {
  cudaError_t e;
  if ((e = configure<64, false, 1>()) != cudaSuccess) return e;
  if ((e = configure<64, false, 2>()) != cudaSuccess) return e;
  if ((e = configure<64, true, 1>()) != cudaSuccess) return e;
  if ((e = configure<64, true, 2>()) != cudaSuccess) return e;
  if ((e = configure<64, false, 4>()) != cudaSuccess) return e;
  if ((e = configure<64, true, 4>()) != cudaSuccess) return e;
  if ((e = configure<128, false, 4>()) != cudaSuccess) return e;
  if ((e = configure<128, true, 4>()) != cudaSuccess) return e;
  if ((e = configure<128, false, 1>()) != cudaSuccess) return e;
  if ((e = configure<128, false, 2>()) != cudaSuccess) return e;
  if ((e = configure<128, true, 1>()) != cudaSuccess) return e;
  return configure<128, true, 2>();
}

cudaError_t launch_paged_join(const PagedParams& p, int D, int ctas, cudaStream_t st) {
  return paged_launch(D == 64 ? paged_join_kernel<64> : paged_join_kernel<128>, dim3(ctas, p.part_rows / (8 * kJoinRows), 1),
                      256, 0, st, p);
}

int paged_attention_ctas(bool e4m3, int row_blocks, int sms) {
  return sms * ctas_per_sm(e4m3, row_blocks);
}

cudaError_t launch_paged_attention(const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p, int D, bool e4m3,
                                   int row_blocks, int sms, cudaStream_t st) {
  if (D == 64) return e4m3 ? launch<64, true>(k, v, p, row_blocks, sms, st) : launch<64, false>(k, v, p, row_blocks, sms, st);
  return e4m3 ? launch<128, true>(k, v, p, row_blocks, sms, st) : launch<128, false>(k, v, p, row_blocks, sms, st);
}

}  // namespace ebd
