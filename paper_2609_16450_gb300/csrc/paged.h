// The paged K/V cache: launch parameters, and the division of a call's
// attention into equal shares of work.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "ebd.h"

namespace ebd {

constexpr int kPagedMaxBatch = 4096;  // sequences of a paged attention (as many as rows)

// ------------------------------------------------------------------ rows in and out
struct PagedRowsParams {
  int B, R, Hkv, D;
  int page_log2, n_pages, max_pages, e4m3;
  long long page_stride;       // bytes of the pools from page to page
  const int* cu_rows;
  const int* row_pos;
  const int* page_table;       // [B][max_pages]
  uint8_t *k_pool, *v_pool;    // [n_pages][Hkv][page][D]
  uint8_t *k_scale, *v_scale;  // [n_pages][Hkv][page]
  __nv_bfloat16 *k, *v;        // rows
  long long kv_stride;         // elements from row to row
  const uint8_t* skip;         // [R] or null
};
// Every kernel of the paged cache is a programmatic dependent of the one before
// it on the stream: it reads global memory only after griddepcontrol.wait, and
// lets the next one's blocks in as soon as it has read its plan.  A kernel before
// it that is such a dependent itself has to complete after its own prior one (it
// waits for it as here does every thread, or see complete_after_prior in k_attn.cu).
template <class... A>
cudaError_t paged_launch(void (*kernel)(A...), dim3 grid, int threads, uint32_t smem, cudaStream_t st, const A&... a) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a...);
}
cudaError_t launch_paged_write(const PagedRowsParams& p, int sms, cudaStream_t st);
cudaError_t launch_paged_read(const PagedRowsParams& p, int sms, cudaStream_t st);

// ------------------------------------------------------------------ attention
// A tile in parts: the first is part 2 c + 1 of the CTA c that it begins in, the
// k-th after it part 2 (c + k).
struct PagedCut {
  int parts, first;     // their number (0: none), and the CTA of the first
  int rows, m0, r0, h;  // packed rows, the first of them, the sequence's first row, K/V head
};
struct PagedParams {
  int B, R, Hq, Hkv, group;
  unsigned group_inv;          // ceil(2^32 / group): m / group = mulhi(m, group_inv) for m * group < 2^32 (4096 rows, 1024 heads at most)
  int causal;
  int page_log2, n_pages, max_pages;
  int cap;                     // positions of a sequence's pages
  int box_log2;                // keys of a tensor-map box (at most a page)
  int part_rows;               // rows of a partial result
  float scale_log2;            // softmax scale * log2(e)
  const int* cu_rows;
  const int* kv_len;
  const int* page_table;
  const uint8_t *k_scale, *v_scale;
  const __nv_bfloat16* q;
  long long q_stride;          // elements from row to row
  __nv_bfloat16* out;          // [R][Hq][D]
  int uncut;                   // shares end where tiles do: no partial results
  float* part;                 // [CTAs][2][part_rows][D] partial sums of cut tiles,
  float* part_ml;              // [CTAs][2][part_rows][2] their (maximum, sum)
  struct PagedCut* cuts;       // [CTAs] the tile that a CTA's share begins and others end
  int* status;
  uint64_t limit_ns;
  int give_up;                 // tests: loads give up at once, as after a wait that ran out
};
// Rows of a tile and CTAs per SM of the two kernels, at most (their workspace).
constexpr int kPagedRows = 64, kPagedCtasPerSm = 4;  // mma.sync
constexpr int kPagedTcRows = 256;                    // tcgen05, one CTA per SM
constexpr int kPagedTcGroup = 128;                   // query heads of a group that the tcgen05 kernel takes
// Page tables of at most so many positions per sequence: tiles stay whole (32 heads,
// one row over 441 8-bit keys 10.5 us against 12.3, 16 x 32 rows over 472 32.2
// against 37.3; up to 1024, 32 rows over 982 would take 22.8 instead of 19.0).
constexpr int kPagedUncutKeys = 512;
constexpr int kPagedLongKeys = 768, kPagedLongKeysE4m3 = 2048;  // past these caches are long (ebd_paged_attention)
cudaError_t paged_configure();
cudaError_t paged_tc_configure();
// tcgen05, 128-wide heads; one: tiles of at most 128 rows, their steps in two streams
cudaError_t launch_paged_tc(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p,
                            bool e4m3, bool one, int sms, cudaStream_t st);
// the parts of cut tiles put together, a programmatic dependent of either kernel of `ctas` CTAs
cudaError_t launch_paged_join(const PagedParams& p, int D, int ctas, cudaStream_t st);
int paged_attention_ctas(bool e4m3, int row_blocks, int sms);
constexpr int kPagedChunkLog2 = 6;                   // keys of a chunk of the mma.sync kernel
constexpr int kPagedTcStepLog2 = 7;                  // and of a step of the tcgen05 kernel
cudaError_t launch_paged_attention(const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p, int D,
                                   bool e4m3, int row_blocks, int sms, cudaStream_t st);

#ifdef __CUDACC__
// ------------------------------------------------------------------ shares of work
// The tiles of a launch are (sequence, tile of T packed rows, K/V head), a
// packed row being (row of the sequence, query head of the group); a tile's
// work is its chunks of CH keys (one at least).  All chunks, in that order, are
// cut into equal contiguous shares, one per CTA, so that ragged lengths and few
// long sequences load every SM alike; a tile cut by a share's end leaves
// partial results, which a second kernel puts together, a warp per few rows.  (By
// the last of the tile's CTAs instead, 19 parts of 252 rows took 190 us, and 2 or
// 3 parts of 7 rows 2 us more than by the kernel.)  Where no tile has many chunks,
// shares are of whole tiles (uncut), and there is nothing to join.
struct PagedSeq {
  int r0, n, len;  // first row, rows, cached positions
  int tiles;
};
// row of its sequence that packed row m is of
__device__ __forceinline__ int paged_row(const PagedParams& p, int m) {
  return p.group == 1 ? m : static_cast<int>(__umulhi(static_cast<unsigned>(m), p.group_inv));
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedParams& p, int b, int T) {
  PagedSeq s;
  s.r0 = min(max(p.cu_rows[b], 0), p.R);
  s.n = min(max(p.cu_rows[b + 1], s.r0), p.R) - s.r0;
  s.len = min(max(p.kv_len[b], 0), p.cap);
  s.tiles = (s.n * p.group + T - 1) / T;
  return s;
}
// keys that row i of the sequence sees: those before this one
__device__ __forceinline__ int paged_limit(const PagedParams& p, const PagedSeq& s, int i) {
  return p.causal ? min(max(s.len - s.n + i + 1, 0), s.len) : s.len;
}
// chunks of tile t, and units of work: chunks, or tiles where none is cut
__device__ __forceinline__ int paged_chunks(const PagedParams& p, const PagedSeq& s, int t, int T, int CH) {
  const int last = min(s.n - 1, paged_row(p, (t + 1) * T - 1));
  return max(1, (paged_limit(p, s, last) + CH - 1) / CH);
}
__device__ __forceinline__ unsigned paged_units(const PagedParams& p, const PagedSeq& s, int T, int CH) {
  unsigned u = 0;
  if (s.n == 0) return 0;
  if (p.uncut) return s.tiles * p.Hkv;
  if (!p.causal)
    u = s.tiles * static_cast<unsigned>(paged_chunks(p, s, 0, T, CH));
  else
    for (int t = 0; t < s.tiles; ++t) u += paged_chunks(p, s, t, T, CH);
  return u * p.Hkv;
}

// Where a CTA's share begins (in shared memory, written by paged_plan).  With q =
// total / shares and r = total % shares, the first r shares have q + 1 units.
// (The host sees to it that units fit 31 bits.)
struct PagedStart {
  unsigned q, r;
  unsigned u0, u1;          // this CTA's units are [u0, u1)
  int b, t, h, c;           // sequence, tile, head and chunk of u0
};
__device__ __forceinline__ unsigned paged_share(const PagedStart& st, unsigned c) { return c * st.q + min(c, st.r); }
// the CTA whose share holds unit u
__device__ __forceinline__ int paged_owner(const PagedStart& st, unsigned u) {
  const unsigned big = st.r * (st.q + 1);
  return static_cast<int>(u < big ? u / (st.q + 1) : st.r + (u - big) / st.q);
}
// All NT threads of the block.  `least`: chunks of a share, at least, so that
// a small call is not cut into more pieces than it is worth.
template <int NT>
__device__ __forceinline__ void paged_plan(const PagedParams& p, int T, int CH, int least, PagedStart* st,
                                           unsigned (&scan)[NT / 32]) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (p.B + NT - 1) / NT;
  const int b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
  unsigned mine = 0;
  for (int b = b0; b < b1; ++b) mine += paged_units(p, paged_seq(p, b, T), T, CH);
  unsigned inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) scan[warp] = inc;
  __syncthreads();
  unsigned before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    const unsigned v = scan[w];
    if (w < warp) before += v;
    total += v;
  }
  const unsigned most = p.uncut ? total : (total + least - 1) / least;
  const unsigned shares = max(1u, min(most, gridDim.x));
  PagedStart s0{};
  s0.q = total / shares;
  s0.r = total - s0.q * shares;
  if (blockIdx.x < shares) {
    s0.u0 = paged_share(s0, blockIdx.x);
    s0.u1 = paged_share(s0, blockIdx.x + 1);
  }
  if (tid == 0) {
    st->q = s0.q;
    st->r = s0.r;
    st->u0 = s0.u0;
    st->u1 = s0.u1;
  }
  unsigned at = before + inc - mine;
  if (s0.u0 < s0.u1 && s0.u0 >= at && s0.u0 < at + mine) {
    for (int b = b0; b < b1; ++b) {
      const PagedSeq s = paged_seq(p, b, T);
      const unsigned u = paged_units(p, s, T, CH);
      if (s0.u0 >= at + u) {
        at += u;
        continue;
      }
      int t = 0;
      unsigned nch = 1;
      for (;; ++t) {
        nch = p.uncut ? 1 : paged_chunks(p, s, t, T, CH);
        if (s0.u0 < at + nch * p.Hkv) break;
        at += nch * p.Hkv;
      }
      st->b = b;
      st->t = t;
      st->h = static_cast<int>((s0.u0 - at) / nch);
      st->c = static_cast<int>((s0.u0 - at) % nch);
      break;
    }
  }
  __syncthreads();
}

// A walk over a share's pieces of tiles, the same in every warp.  Tiles of CT
// rows (0: of the T that begin is given), chunks of CCH keys.
template <int CT, int CCH>
struct PagedWalk {
  PagedSeq s;
  unsigned u, u1;  // next unit of the share, and its end
  int b, t, h;
  int c0, c1, nch;  // the piece: chunks [c0, c1) of the tile's nch
  int rt;
  __device__ __forceinline__ int T() const { return CT != 0 ? CT : rt; }
  __device__ __forceinline__ void piece(const PagedParams& p, int c) {
    nch = paged_chunks(p, s, t, T(), CCH);
    c0 = c;
    c1 = !p.uncut && u1 - u < static_cast<unsigned>(nch - c) ? c + static_cast<int>(u1 - u) : nch;
  }
  __device__ __forceinline__ bool begin(const PagedParams& p, const PagedStart& st, int T_) {
    rt = T_;
    u = st.u0;
    u1 = st.u1;
    if (u >= u1) return false;
    b = st.b;
    t = st.t;
    h = st.h;
    s = paged_seq(p, b, T());
    piece(p, st.c);
    return true;
  }
  __device__ __forceinline__ bool next(const PagedParams& p) {
    u += p.uncut ? 1 : c1 - c0;
    if (u >= u1) return false;
    if (++h == p.Hkv) {
      h = 0;
      if (++t == s.tiles) {
        t = 0;
        do s = paged_seq(p, ++b, T());
        while (s.tiles == 0);  // ends: chunks are left
      }
    }
    piece(p, 0);
    return true;
  }
  __device__ __forceinline__ bool whole() const { return c0 == 0 && c1 == nch; }
  // where this piece's partial result goes
  __device__ __forceinline__ int part() const { return 2 * static_cast<int>(blockIdx.x) + (c0 == 0 ? 1 : 0); }
  __device__ __forceinline__ PagedCut cut(const PagedParams& p, const PagedStart& st) const {
    PagedCut x;
    x.first = paged_owner(st, u - c0);
    x.parts = paged_owner(st, u - c0 + nch - 1) - x.first + 1;
    x.m0 = t * T();
    x.rows = min(T(), s.n * p.group - x.m0);
    x.r0 = s.r0;
    x.h = h;
    return x;
  }
  // The last piece of a share: the tile that it begins and does not end, to be
  // put together (one thread).
  __device__ __forceinline__ void leave(const PagedParams& p, const PagedStart& st) const {
    PagedCut x{};
    if (c0 == 0 && c1 < nch) x = cut(p, st);
    p.cuts[blockIdx.x] = x;
  }
};

#endif

}  // namespace ebd
