// Plan of a step over the paged K/V cache, on the device: pages handed out and taken
// back by what every sequence's length becomes, and the new rows' offsets, positions
// and slots.
//
// Sequence b has len positions in ceil(len / page) pages and comes to max(0, len +
// add).  Pages past what it then needs go onto the stack of free pages, the sequences
// from the last to the first and each from its last page; after that the pages that
// sequences need more come off its top, sequences and pages ascending.  So taking
// back what a call handed out leaves the stack as it was.
//
// One CTA: a plan moves a few KB, and is bound by its chain of loads: lengths ->
// prefix sums (rows, pages out, pages back) -> the pages to move.  Every item finds its
// sequence by a binary search of the prefix sums in shared memory.  Pages that move are
// read once, all at a time, and kept there; slots come from them too.  All that a plan
// asks for is looked at before anything is written: one that cannot be met changes no
// state, and hands out no rows.
#include "internal.h"
#include "paged.h"

namespace ebd {

namespace {

constexpr int kPlanThreads = 512;  // at most
constexpr int kPlanPages = 8192;    // pages out, and back, that shared memory holds

struct Sums {
  long long rows, out, back;
  int bad;   // 1: EBD_ERR_BOUNDS, 2: EBD_ERR_PAGES
  int most;  // new rows of one sequence
};

// Sequence of item i by the prefix sums cu[0 .. n]: the last with cu[b] <= i < cu[b + 1].
__device__ __forceinline__ int sequence_of(const int* cu, int n, int i) {
  int lo = 0, hi = n;  // cu[lo] <= i < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= i)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) paged_plan_kernel(const PagedPlanParams p) {
  extern __shared__ int dyn[];
  int* const rows = dyn;                 // [B + 1] prefix sums of new rows,
  int* const out = rows + p.B + 1;       // of pages to hand out,
  int* const back = out + p.B + 1;       // of pages to take back
  int* const first = back + p.B + 1;     // [B] first page that changes hands
  int* const old = first + p.B;          // [B] length before
  int* const then = old + p.B;           // [B] and after
  int* const now = then + p.B;           // [B] page that the first new row goes into, if it is there
  int* const going = now + p.B;          // [p.pages] pages back,
  int* const coming = going + p.pages;   // and out
  __shared__ Sums warp_sum[kPlanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
  const int page = 1 << p.page_log2;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long n0 = *p.n_free;

  // a run of sequences a thread
  const int per = (p.B + threads - 1) / threads;
  const int b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
  Sums sum{0, 0, 0, 0, 0};
  const long long most = min(static_cast<long long>(p.max_pages) << p.page_log2, 0x7fffffffll);
  auto look = [&](int b, int len, int add) {
    const long long to = max(0ll, static_cast<long long>(len) + add);
    if (len < 0 || len > most || to > most) {
      sum.bad |= len < 0 || len > most ? 1 : 2;
      return;
    }
    const int have = static_cast<int>((static_cast<long long>(len) + page - 1) >> p.page_log2);
    const int need = static_cast<int>((to + page - 1) >> p.page_log2);
    rows[b] = max(add, 0);
    out[b] = max(need - have, 0);
    back[b] = max(have - need, 0);
    first[b] = min(have, need);
    old[b] = len;
    then[b] = static_cast<int>(to);
    sum.rows += max(add, 0);
    sum.out += max(need - have, 0);
    sum.back += max(have - need, 0);
    sum.most = max(sum.most, add);
  };
  for (int b = b0; b < b1; b += 4) {  // four sequences' loads at once
    int len[4], add[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (b + j < b1) len[j] = p.kv_len[b + j], add[j] = p.add[b + j];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (b + j < b1) look(b + j, len[j], add[j]);
  }
  Sums incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long r = __shfl_up_sync(0xffffffffu, incl.rows, o), t = __shfl_up_sync(0xffffffffu, incl.out, o),
                    k = __shfl_up_sync(0xffffffffu, incl.back, o);
    if (lane >= o) {
      incl.rows += r;
      incl.out += t;
      incl.back += k;
    }
  }
  incl.bad = static_cast<int>(__reduce_or_sync(0xffffffffu, static_cast<unsigned>(sum.bad)));
  incl.most = __reduce_max_sync(0xffffffffu, sum.most);
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  Sums at{incl.rows - sum.rows, incl.out - sum.out, incl.back - sum.back, 0, 0}, total{0, 0, 0, 0, 0};
  for (int i = 0; i < threads / 32; ++i) {
    const Sums w = warp_sum[i];
    if (i < warp) at.rows += w.rows, at.out += w.out, at.back += w.back;
    total.rows += w.rows, total.out += w.out, total.back += w.back, total.bad |= w.bad, total.most = max(total.most, w.most);
  }
  int bad = total.bad;  // as all threads see it
  if (n0 < 0 || n0 + total.back > p.n_pages) bad |= 1;
  if (total.out > n0 + total.back || total.rows > 0x7fffffffll) bad |= 2;
  if ((p.row_pos != nullptr || p.slot != nullptr) && total.rows > p.R) bad |= 2;
  const int n_out = static_cast<int>(total.out), n_back = static_cast<int>(total.back);
  const int top = static_cast<int>(n0) + n_back;  // of the stack, once all are back on it
  // Item i of the pages back goes to place top - 1 - i of the stack, which is where item
  // i of the pages out comes from.
  const bool kept = n_out <= p.pages && n_back <= p.pages;
  auto leaves = [&](int i) -> int* {
    const int b = sequence_of(back, p.B, i);
    return p.page_table + static_cast<long long>(b) * p.max_pages + first[b] + i - back[b];
  };
  auto comes = [&](int i) -> int* {
    const int b = sequence_of(out, p.B, i);
    return p.page_table + static_cast<long long>(b) * p.max_pages + first[b] + i - out[b];
  };
  if (!bad) {
    int wrong = 0;
    for (int b = b0; b < b1; ++b) {
      const int r = rows[b], o = out[b], k = back[b], len = old[b];
      rows[b] = static_cast<int>(at.rows), out[b] = static_cast<int>(at.out), back[b] = static_cast<int>(at.back);
      at.rows += r, at.out += o, at.back += k;
      // new rows begin within a page that is there
      if (r > 0 && (len & (page - 1)) != 0) {
        const int e = p.page_table[static_cast<long long>(b) * p.max_pages + (len >> p.page_log2)];
        now[b] = e;
        wrong |= e < 0 || e >= p.n_pages;
      }
    }
    if (tid == 0) rows[p.B] = static_cast<int>(total.rows), out[p.B] = n_out, back[p.B] = n_back;
    __syncthreads();
    for (int i = tid; i < n_back; i += threads) {
      const int e = *leaves(i);
      if (kept) going[i] = e;
      wrong |= e < 0 || e >= p.n_pages;
    }
    for (int i = tid; i < n_out; i += threads) {
      if (i < n_back) continue;  // one of those
      const int e = p.free_pages[top - 1 - i];
      if (kept) coming[i] = e;
      wrong |= e < 0 || e >= p.n_pages;
    }
    if (__syncthreads_or(wrong)) bad = 1;
  }
  if (bad) {
    if (tid == 0) atomicCAS(p.status, 0, (bad & 1) ? EBD_ERR_BOUNDS : EBD_ERR_PAGES);
    if (p.cu_rows != nullptr)
      for (int b = tid; b <= p.B; b += threads) p.cu_rows[b] = 0;
    for (int r = tid; r < p.R; r += threads) {
      if (p.row_pos != nullptr) p.row_pos[r] = -1;
      if (p.slot != nullptr) p.slot[r] = -1;
    }
    return;
  }
  for (int b = b0; b < b1; ++b) p.kv_len[b] = then[b];
  if (tid == 0) *p.n_free = top - n_out;
  if (p.cu_rows != nullptr)
    for (int b = tid; b <= p.B; b += threads) p.cu_rows[b] = rows[b];
  for (int i = tid; i < n_back; i += threads) {
    int* const e = leaves(i);
    p.free_pages[top - 1 - i] = kept ? going[i] : *e;
    *e = -1;
  }
  if (!kept) __syncthreads();  // pages out may be among those on the stack by now
  for (int i = tid; i < n_out; i += threads)
    *comes(i) = !kept ? p.free_pages[top - 1 - i] : i < n_back ? going[i] : coming[i];
  if (!kept) __syncthreads();  // slots read the table
  auto put = [&](int b, int r) {  // row r, of sequence b
    const int pos = old[b] + r - rows[b];
    if (p.row_pos != nullptr) p.row_pos[r] = pos;
    if (p.slot == nullptr) return;
    const int j = pos >> p.page_log2, i = out[b] + j - first[b];  // new pages are from `first` on
    const long long e = !kept          ? p.page_table[static_cast<long long>(b) * p.max_pages + j]
                        : j < first[b] ? now[b]
                        : i < n_back   ? going[i]
                                       : coming[i];
    p.slot[r] = (e << p.page_log2) + (pos & (page - 1));
  };
  // rows by their sequences where those have few, else each looks for its own
  const bool few = total.most <= 4;
  if (p.row_pos == nullptr && p.slot == nullptr) return;
  if (few)
    for (int b = b0; b < b1; ++b)
      for (int r = rows[b]; r < rows[b + 1]; ++r) put(b, r);
  for (int r = few ? static_cast<int>(total.rows) + tid : tid; r < p.R; r += threads) {
    if (r < total.rows) {
      put(sequence_of(rows, p.B, r), r);
      continue;
    }
    if (p.row_pos != nullptr) p.row_pos[r] = -1;
    if (p.slot != nullptr) p.slot[r] = -1;
  }
}

size_t plan_bytes(int B, int pages) {
  return (3 * (static_cast<size_t>(B) + 1) + 4 * static_cast<size_t>(B) + 2 * static_cast<size_t>(pages)) * sizeof(int);
}

}  // namespace

cudaError_t launch_paged_plan(PagedPlanParams p, cudaStream_t st) {
  // A thread for each sequence and row, as far as that goes: fewer start sooner, and
  // meet at barriers sooner.  us for the two calls of 2048 sequences with 128 / 256 / 384 /
  // 512 / 768 / 1024 threads at most: 31.8 / 19.5 / 14.3 / 14.9 / 14.9 / 17.4; of prompts of
  // 2k rows 12.7 / 9.5 / 8.9 / 9.0 / 9.5 / 11.0.
  const int items = p.B > p.R ? p.B : p.R;
  const int threads = items >= kPlanThreads ? kPlanThreads : items <= 128 ? 128 : (items + 31) / 32 * 32;
  // pages that may move: rows and a page more for each sequence, or as many back
  const int pages = p.B + (p.R > p.B ? p.R : p.B);
  p.pages = pages < kPlanPages ? pages : kPlanPages;
  const uint32_t bytes = static_cast<uint32_t>(plan_bytes(p.B, p.pages));
  if (bytes > 40 * 1024) {  // past what a kernel has without being asked, next to its own 2 KB
    const cudaError_t e = cudaFuncSetAttribute(paged_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(plan_bytes(kPagedMaxBatch, kPlanPages)));
    if (e != cudaSuccess) return e;
  }
  return paged_launch(paged_plan_kernel, dim3(1), threads, bytes, st, p);
}

}  // namespace ebd
