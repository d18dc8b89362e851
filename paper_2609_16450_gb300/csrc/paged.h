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
cudaError_t launch_paged_write(const PagedRowsParams& p, cudaStream_t st);
cudaError_t launch_paged_read(const PagedRowsParams& p, cudaStream_t st);

// ------------------------------------------------------------------ attention
struct PagedParams {
  int B, R, Hq, Hkv, group;
  int causal;
  int page_log2, n_pages, max_pages;
  int box_log2;                // keys of a tensor-map box (at most a page)
  int above, upto;             // sequences with above < rows * group <= upto are this launch's
  float scale_log2;            // softmax scale * log2(e)
  const int* cu_rows;
  const int* kv_len;
  const int* page_table;
  const uint8_t *k_scale, *v_scale;
  const __nv_bfloat16* q;
  long long q_stride;          // elements from row to row
  __nv_bfloat16* out;          // [R][Hq][D]
  float* part;                 // [CTAs][2][tile rows][D] partial sums of split tiles,
  float* part_ml;              // [CTAs][2][tile rows][2] their (maximum, sum)
  int* tickets;                // [CTAs] by the CTA that a split tile begins in; zero between launches
  int* status;
  uint64_t limit_ns;
};
// tile rows and CTAs of the two kernels (their workspace)
constexpr int kPagedRows = 64;      // mma.sync kernel: at most, per tile
constexpr int kPagedCtasPerSm = 3;  // at most
cudaError_t paged_configure();
cudaError_t launch_paged_attention(const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p, int D,
                                   bool e4m3, int row_blocks, int sms, cudaStream_t st);

#ifdef __CUDACC__
// ------------------------------------------------------------------ shares of work
// The tiles of a launch are (sequence, tile of T packed rows, K/V head), a
// packed row being (row of the sequence, query head of the group); a tile's
// work is its chunks of CH keys (one at least).  All chunks, in that order, are
// cut into equal contiguous shares, one per CTA, so that ragged lengths and few
// long sequences load every SM alike; a tile cut by a share's end leaves
// partial results, which the last CTA of the tile to finish puts together.
struct PagedSeq {
  int r0, n, len;  // first row, rows (0: not of this launch), cached positions
  int tiles;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedParams& p, int b, int T) {
  PagedSeq s;
  s.r0 = min(max(p.cu_rows[b], 0), p.R);
  s.n = min(max(p.cu_rows[b + 1], s.r0), p.R) - s.r0;
  const long long cap = static_cast<long long>(p.max_pages) << p.page_log2;
  const int len = p.kv_len[b];
  s.len = len < 0 ? 0 : (len > cap ? static_cast<int>(cap) : len);
  const long long m = static_cast<long long>(s.n) * p.group;
  if (m <= p.above || m > p.upto) s.n = 0;
  s.tiles = static_cast<int>((static_cast<long long>(s.n) * p.group + T - 1) / T);
  return s;
}
// keys that row i of the sequence sees: those before this one
__device__ __forceinline__ int paged_limit(const PagedParams& p, const PagedSeq& s, int i) {
  return p.causal ? min(max(s.len - s.n + i + 1, 0), s.len) : s.len;
}
// chunks of tile t
__device__ __forceinline__ int paged_chunks(const PagedParams& p, const PagedSeq& s, int t, int T, int CH) {
  const int last = min(s.n - 1, static_cast<int>(((static_cast<long long>(t) + 1) * T - 1) / p.group));
  return max(1, (paged_limit(p, s, last) + CH - 1) / CH);
}
__device__ __forceinline__ long long paged_units(const PagedParams& p, const PagedSeq& s, int T, int CH) {
  long long u = 0;
  if (s.n == 0) return 0;
  if (!p.causal) return static_cast<long long>(s.tiles) * p.Hkv * paged_chunks(p, s, 0, T, CH);
  for (int t = 0; t < s.tiles; ++t) u += paged_chunks(p, s, t, T, CH);
  return u * p.Hkv;
}

// Where a CTA's share begins (in shared memory, written by paged_plan).
struct PagedStart {
  long long total, u0, u1;  // chunks in all; this CTA's are [u0, u1)
  int shares;               // CTAs that have one
  int b, t, h, c;           // sequence, tile, head and chunk of u0
};
// All NT threads of the block.  `least`: chunks of a share, at least, so that
// a small call is not cut into more pieces than it is worth.
template <int NT>
__device__ __forceinline__ void paged_plan(const PagedParams& p, int T, int CH, int least, PagedStart* st,
                                           long long (&scan)[NT / 32 + 1]) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (p.B + NT - 1) / NT;
  const int b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += paged_units(p, paged_seq(p, b, T), T, CH);
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) scan[warp] = inc;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    if (w < warp) before += scan[w];
    total += scan[w];
  }
  const long long most = (total + least - 1) / least;
  const int shares = most < gridDim.x ? static_cast<int>(most) : static_cast<int>(gridDim.x);
  long long u0 = 0, u1 = 0;
  if (static_cast<int>(blockIdx.x) < shares) {
    u0 = total * blockIdx.x / shares;
    u1 = total * (blockIdx.x + 1) / shares;
  }
  if (tid == 0) {
    st->total = total;
    st->shares = shares;
    st->u0 = u0;
    st->u1 = u1;
  }
  long long at = before + inc - mine;
  if (u0 < u1 && u0 >= at && u0 < at + mine) {
    for (int b = b0; b < b1; ++b) {
      const PagedSeq s = paged_seq(p, b, T);
      const long long u = paged_units(p, s, T, CH);
      if (u0 < at + u) {
        int t = 0;
        for (; t < s.tiles; ++t) {
          const long long w = static_cast<long long>(paged_chunks(p, s, t, T, CH)) * p.Hkv;
          if (u0 < at + w) break;
          at += w;
        }
        const int nch = paged_chunks(p, s, t, T, CH);
        st->b = b;
        st->t = t;
        st->h = static_cast<int>((u0 - at) / nch);
        st->c = static_cast<int>((u0 - at) % nch);
        break;
      }
      at += u;
    }
  }
  __syncthreads();
}

// A walk over a share's pieces of tiles, the same in every warp.
struct PagedWalk {
  PagedSeq s;
  long long u, u1;  // next chunk of the share, and its end
  int b, t, h;
  int c0, c1, nch;  // the piece: chunks [c0, c1) of the tile's nch
  int T, CH;
  __device__ __forceinline__ void piece(const PagedParams& p, int c) {
    nch = paged_chunks(p, s, t, T, CH);
    c0 = c;
    c1 = u1 - u < nch - c ? c + static_cast<int>(u1 - u) : nch;
  }
  __device__ __forceinline__ bool begin(const PagedParams& p, const PagedStart& st, int T_, int CH_) {
    T = T_;
    CH = CH_;
    u = st.u0;
    u1 = st.u1;
    if (u >= u1) return false;
    b = st.b;
    t = st.t;
    h = st.h;
    s = paged_seq(p, b, T);
    piece(p, st.c);
    return true;
  }
  __device__ __forceinline__ bool next(const PagedParams& p) {
    u += c1 - c0;
    if (u >= u1) return false;
    if (++h == p.Hkv) {
      h = 0;
      if (++t == s.tiles) {
        t = 0;
        do s = paged_seq(p, ++b, T);
        while (s.tiles == 0);  // ends: chunks are left
      }
    }
    piece(p, 0);
    return true;
  }
  __device__ __forceinline__ bool whole() const { return c0 == 0 && c1 == nch; }
};
// the CTA whose share holds chunk u
__device__ __forceinline__ int paged_owner(const PagedStart& st, long long u) {
  int c = static_cast<int>(u * st.shares / st.total);
  while (c > 0 && st.total * c / st.shares > u) --c;
  while (st.total * (c + 1) / st.shares <= u) ++c;
  return c;
}
#endif

}  // namespace ebd
