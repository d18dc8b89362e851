// Sampling from logits: temperature, top-k, top-p and min-p, one token and its
// probability per row, from a random number given for the row.
//
// With logits l, m their largest, temperature T and w[v] = exp((l[v] - m) / T), the
// tokens are taken by descending logit, ties by ascending index.  Top-k keeps the
// first k of that order, top-p the least prefix of those with at least the share p
// of their sum, min-p those with w >= min_p.  What is kept is a prefix F of the
// order, given by its last logit and index; the token is the first of F by index
// where the running sum passes u times the sum.
//
// Sums are whole numbers of 64 bits (sample_math.h): exact, so that borders do not
// depend on how a row is split or in which order atomics arrive.
//
// A row is one cluster of CTAs; each warp owns a contiguous run of the row's
// 16-byte groups, so that sums by warp are sums by index.  A CTA's slice of the row
// comes into its shared memory once where it fits, else it is read again.
//
// The last logit of a prefix is found without sorting, in one of three ways.
//   - Top-k of few: every thread has the largest logit of each half of its own; the
//     least, over the CTAs, of the (k / CTAs)-th of a CTA's is a bound that k logits
//     reach and not many more.  Those are listed, and one CTA does the rest with them in
//     registers.
//   - Top-p: one sweep counts logits in bins of y = (m - l) log2(e) / T, which bound
//     the sums and so the few bins that the border lies in; a second sums what lies
//     above them and lists what lies within, and again one CTA does the rest.
//   - Where such a list would be too long (ties, most of all): histograms over the
//     logits' ordered bits, each level over the bin that the last one chose.
//
// What bounds it: not the bytes (512 rows of 152064 floats of mixed settings are 311 MB,
// 46 us at the copy rate; 190 us), but the weights, some 40 instructions each (55 % of
// the issue slots are taken then), an atomic operation a logit where bins are counted, and
// for few rows the chain of phases: a row's first bytes 1 us, its largest logit 2 to 3, a
// list and its CTA's work 5 to 8, every barrier of a cluster 1 to 2 (32 rows of 126464 by
// top-k and top-p 20 us; 64 rows at a temperature 24; one row of 4096 6.4).
// Histograms of weights over all of a row instead took 296 us for the 32 rows, 1837 for
// the 512.  A slice of the row in shared memory pays for 16-bit rows (24 rows by
// top-p 61 against 72 us read again from L2), and for floats is no better than L2.
#include <cuda_fp16.h>

#include <climits>
#include <cstring>

#include "internal.h"
#include "ptx.cuh"
#include "sample.h"
#include "sample_math.h"

namespace ebd {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCtas = 8;
constexpr int kBins = 2048;                  // of y, counts
constexpr int kFine = 512, kFineBits = 9;    // of ordered bits, weights and counts
constexpr int kLocal = 1024, kLocalBits = 10;  // of a list
constexpr int kList = 2048, kItems = kList / kThreads;  // listed logits, of a CTA and of a row
constexpr int kListMost = kThreads;           // of a CTA's threads' two values, for a list of top-k's
constexpr int kSliceBytes = 76 * 1024;  // of a row in shared memory

// Loads from a CTA of the cluster; volatile, so none moves across a barrier, and
// several are in flight.
__device__ __forceinline__ uint64_t ld_cluster(const uint64_t* p, uint32_t rank) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(mapa_shared(smem_u32(p), rank)));
  return v;
}
__device__ __forceinline__ int ld_cluster(const int* p, uint32_t rank) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(smem_u32(p), rank)));
  return v;
}
__device__ __forceinline__ uint4 ld_cluster(const uint4* p, uint32_t rank) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(mapa_shared(smem_u32(p), rank))
              );
  return v;
}
__device__ __forceinline__ uint32_t ld_cluster(const uint32_t* p, uint32_t rank) {
  return static_cast<uint32_t>(ld_cluster(reinterpret_cast<const int*>(p), rank));
}
__device__ __forceinline__ uint2 ld_cluster(const uint2* p, uint32_t rank) {
  uint2 v;
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(mapa_shared(smem_u32(p), rank)));
  return v;
}
__device__ __forceinline__ float ld_cluster(const float* p, uint32_t rank) {
  return __int_as_float(ld_cluster(reinterpret_cast<const int*>(p), rank));
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// The logits of a 16-byte group.
template <int TYPE>
struct Group;
template <>
struct Group<EBD_LOGITS_F32> {
  static constexpr int N = 4;
  using T = float;
  __device__ static T masked() { return -INFINITY; }
  __device__ static void get(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
  }
};
template <>
struct Group<EBD_LOGITS_BF16> {
  static constexpr int N = 8;
  using T = uint16_t;
  __device__ static T masked() { return 0xFF80; }
  __device__ static void get(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <>
struct Group<EBD_LOGITS_F16> {
  static constexpr int N = 8;
  using T = uint16_t;
  __device__ static T masked() { return 0xFC00; }
  __device__ static void get(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
};

// A 64-bit sum in shared memory by two 32-bit additions: the 64-bit one is a loop of
// compare and swap, which adds to one place one thread at a time.
__device__ __forceinline__ void add64(uint64_t* to, uint64_t v) {
  uint32_t* w = reinterpret_cast<uint32_t*>(to);
  const uint32_t lo = static_cast<uint32_t>(v), old = atomicAdd(w, lo);
  const uint32_t hi = static_cast<uint32_t>(v >> 32) + (old + lo < old ? 1u : 0u);
  if (hi != 0) atomicAdd(w + 1, hi);
}

__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// sum over this and the lanes before it
__device__ __forceinline__ uint64_t warp_scan(uint64_t x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// Histograms of one level, in turn: every CTA's is read by the whole cluster, which
// is done with it when the next level's are.
struct alignas(16) Hist {
  union {
    uint32_t coarse[kBins];
    struct {
      uint64_t weight[kFine];
      uint32_t count[kFine];
    };
    uint64_t local[kLocal];
  };
};

// y to bins: the lesser of two lines, fine ones up to a knee and coarse ones from there
// on.  Rounding keeps their order.
struct Bins {
  float fine, coarse, shift;
  __device__ __forceinline__ int of(float y) const {
    if (!(y <= kSampleDead)) return kBins;
    return static_cast<int>(__float_as_uint(fminf(fmaf(y, fine, 8388608.f), fmaf(y, coarse, 8388608.f + shift))) & 0x7FFFFFu);
  }
  // where bin b begins
  __device__ __forceinline__ float from(int b) const {
    return fmaxf((static_cast<float>(b) - 0.5f) / fine, (static_cast<float>(b) - 0.5f - shift) / coarse);
  }
};
__device__ __forceinline__ Bins make_bins(float knee) {
  constexpr float kFew = 500.f, kMost = 1540.f;
  if (!(knee < kSampleDead * 0.75f)) return {2040.f / kSampleDead, 2040.f / kSampleDead, 0.f};
  knee = fmaxf(knee, kSampleDead * 2.5e-5f);
  const float fine = kMost / knee, coarse = kFew / (kSampleDead - knee);
  return {fine, coarse, rintf(kMost - knee * coarse)};
}

struct Shared {
  Hist hist[2];
  uint2 list[kList];         // logits (their bits) and indices
  SampleEntry table[kSampleTable];
  uint64_t part[kWarps];     // a warp's sums: of what is kept for sure,
  uint64_t rest[kWarps];     // of all that may be kept;
  uint64_t count[kWarps];    // its elements at the border, or what of it is kept
  uint64_t scan[kWarps];
  uint64_t chunk[kMaxCtas * kWarps];  // what every warp of the cluster has, of what is kept
  float scan_f[kWarps];
  uint64_t bar[kWarps];
  uint64_t before, in, want, total;
  float max[kWarps], low[kWarps];
  int bad[kWarps];
  int first[kWarps];
  float kth;                 // a bound of the row's k-th logit, of this CTA's threads'
  int listed;
  int bin, k_bin, k_whole, k_before, alone, index, owner, last;
  int p_first[3], p_last[3], n_first[3], n_last[3];  // top-p's bins: surely, likely, and still likely
  float value;
  uint32_t bound[8];
  SampleScale scale;
  Bins bins;
  int g1, per_warp;            // the end of this CTA's groups, and a warp's of them
  float floor_hi, floor_lo;  // T ln min_p
};

// Which elements of the row are kept: those above `value`, and those equal to it up
// to `index`.
struct Prefix {
  float value;
  int index;
  __device__ __forceinline__ bool has(float x, int i) const { return x > value || (x == value && i <= index); }
  // what those reach that are kept whatever their index
  __device__ __forceinline__ float cut() const {
    return index == INT_MAX ? value : order_value(order_key(value + 0.f) + 1);
  }
};

// W: logits whose weights a thread works on at once, 4 or 8.
template <int TYPE, bool RESIDENT, int W>
struct Row {
  using G = Group<TYPE>;
  Shared& s;
  const SampleParams& p;
  const uint8_t* data;  // the row's first 16-byte group, in global memory
  int f0, f1;           // this warp's groups that are wholly the row's,
  int ends;             // and whether one before (1) and one after (2) is so in part
  int head, g0;         // elements before the row's in its first group; this CTA's first
  float m = 0.f;
  SampleScale c{};
  int level = 0;

  // What is seldom needed is computed again, or in shared memory: registers are scarce.
  __device__ __forceinline__ static int lane() { return threadIdx.x & 31; }
  __device__ __forceinline__ static int warp() { return threadIdx.x >> 5; }
  __device__ __forceinline__ static int rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return static_cast<int>(r);
  }
  __device__ __forceinline__ int ctas() const { return p.ctas; }
  __device__ __forceinline__ uint4* slice() const {
    extern __shared__ __align__(16) uint8_t dyn[];
    return reinterpret_cast<uint4*>(dyn);
  }
  __device__ __forceinline__ void sync() const {
    if (ctas() == 1)
      __syncthreads();
    else
      cluster_sync_all();
  }
  __device__ __forceinline__ void arrive() const {
    if (ctas() > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  __device__ __forceinline__ void wait() const {
    if (ctas() > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  __device__ __forceinline__ bool whole(int g) const { return g * G::N >= head && (g + 1) * G::N <= head + p.vocab; }
  // a group that is not wholly the row's, element by element
  __device__ __forceinline__ uint4 edge(int g) const {
    uint4 v;
    typename G::T t[G::N];
    for (int j = 0; j < G::N; ++j) {
      const int i = g * G::N + j;
      t[j] = i >= head && i < head + p.vocab ? reinterpret_cast<const typename G::T*>(data)[i] : G::masked();
    }
    memcpy(&v, t, 16);
    return v;
  }
  __device__ __forceinline__ uint4 fetch(int g) const {
    if (RESIDENT) return slice()[g - g0];
    return whole(g) ? __ldg(reinterpret_cast<const uint4*>(data) + g) : edge(g);
  }
  // f(index of the first, four logits) for the logits of the warp's groups; where they
  // are in global memory, AHEAD loads of a thread in flight
  template <int AHEAD, typename F>
  __device__ __forceinline__ void sweep4(F f) const {
    auto four = [&](int g, const uint4& v) {
      float x[G::N];
      G::get(v, x);
#pragma unroll
      for (int j = 0; j < G::N; j += 4) {
        const float y[4] = {x[j], x[j + 1], x[j + 2], x[j + 3]};
        f(g * G::N + j - head, y);
      }
    };
    if (RESIDENT) {
      for (int g = f0 - (ends & 1) + lane(); g < f1 + (ends >> 1); g += 32) four(g, fetch(g));
      return;
    }
    const uint4* d = reinterpret_cast<const uint4*>(data);
    int g = f0 + lane();
    if (AHEAD == 1) {  // the next one while this one is worked on
      uint4 next = make_uint4(0, 0, 0, 0);
      if (g < f1) next = d[g];
      while (g < f1) {
        const uint4 v = next;
        const int at = g;
        g += 32;
        if (g < f1) next = d[g];
        four(at, v);
      }
    } else {
      for (; g + 32 * (AHEAD - 1) < f1; g += 32 * AHEAD) {
        uint4 v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) v[j] = d[g + 32 * j];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) four(g + 32 * j, v[j]);
      }
      for (; g < f1; g += 32) four(g, d[g]);
    }
    if ((ends & 1) != 0 && lane() == 0) four(f0 - 1, edge(f0 - 1));
    if ((ends & 2) != 0 && lane() == 0) four(f1, edge(f1));
  }
  // index of the k-th of W logits, from the first's: floats come in two groups, a
  // warp's apart
  __device__ __forceinline__ static constexpr int at(int k) { return G::N == 8 || k < 4 ? k : k - 4 + 32 * 4; }
  // f(index of the first, W logits), at() apart; -inf where there are none
  template <typename F>
  __device__ __forceinline__ void sweep_wide(F f) const {
    if constexpr (W == 4) {
      sweep4<1>(f);
      return;
    } else {
      constexpr int GROUPS = 8 / G::N;  // of a turn
      const int first = f0 - (RESIDENT ? ends & 1 : 0), end = f1 + (RESIDENT ? ends >> 1 : 0);
      auto load = [&](int g, uint4(&v)[GROUPS]) {
#pragma unroll
        for (int k = 0; k < GROUPS; ++k)
          if (g + 32 * k < end) v[k] = RESIDENT ? slice()[g + 32 * k - g0] : reinterpret_cast<const uint4*>(data)[g + 32 * k];
      };
      auto give = [&](int g, const uint4(&v)[GROUPS], int last) {
        float x[8];
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
          float y[G::N];
          G::get(v[k], y);
#pragma unroll
          for (int j = 0; j < G::N; ++j) x[k * G::N + j] = g + 32 * k < last ? y[j] : -INFINITY;
        }
        f(g * G::N - head, x);
      };
      uint4 next[GROUPS];
      int g = first + lane();
      load(g, next);
      while (g < end) {
        uint4 v[GROUPS];
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) v[k] = next[k];
        const int here = g;
        g += 32 * GROUPS;
        load(g, next);
        give(here, v, end);
      }
      if (!RESIDENT && lane() == 0) {
        uint4 v[GROUPS];
        if ((ends & 1) != 0) {
          v[0] = edge(f0 - 1);
          give(f0 - 1, v, f0);
        }
        if ((ends & 2) != 0) {
          v[0] = edge(f1);
          give(f1, v, f1 + 1);
        }
      }
    }
  }
  // f(index, logit)
  template <int AHEAD = 1, typename F>
  __device__ __forceinline__ void sweep(F f) const {
    sweep4<AHEAD>([&](int i, const float(&x)[4]) {
#pragma unroll
      for (int j = 0; j < 4; ++j) f(i + j, x[j]);
    });
  }
  __device__ __forceinline__ uint64_t weight(float x) const { return sample_weight(m, x, c, s.table); }
  // Adds up the weights of those of W logits that reach `cut`, and of those above
  // `over` (TWO).  Their parts add up exactly as floats.
  template <bool TWO>
  __device__ __forceinline__ void weigh(const float (&x)[W], float cut, float over, uint64_t& sum, uint64_t& above) const {
    if (!(largest(x) >= cut)) return;
    float h[W], r[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const SampleParts w = sample_parts(sample_term(m, x[j], c, s.table));
      h[j] = x[j] >= cut ? w.high : 0.f;
      r[j] = x[j] >= cut ? w.low : 0.f;
    }
    add_up(sum, h, r);
    if (TWO) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        h[j] = x[j] > over ? h[j] : 0.f;
        r[j] = x[j] > over ? r[j] : 0.f;
      }
      add_up(above, h, r);
    }
  }
  __device__ __forceinline__ static float largest(const float (&x)[W]) {
    float y = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    if constexpr (W == 8) y = fmaxf(y, fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    return y;
  }
  // (8 of 1 are 2^24 units of 2^-21, and 4 of 2^-21 2^24 units of 2^-43)
  __device__ __forceinline__ static void add_up(uint64_t& sum, const float (&h)[W], const float (&r)[W]) {
    float a = (h[0] + h[2]) + (h[1] + h[3]);
    int low = __float2int_rn(((r[0] + r[2]) + (r[1] + r[3])) * kSampleUnits);
    if constexpr (W == 8) {
      a += (h[4] + h[6]) + (h[5] + h[7]);
      low += __float2int_rn(((r[4] + r[6]) + (r[5] + r[7])) * kSampleUnits);
    }
    // floats from 4 to 8 have steps of 2^-21
    const int high = W == 4 ? __float_as_int(a + 4.f) - __float_as_int(4.f) : __float2int_rn(a * 2097152.f);
    sum += static_cast<uint64_t>(static_cast<int64_t>(high) * 4194304 + low);
  }
  // how many of W logits are equal to the last kept one, and kept
  __device__ __forceinline__ static int ties(const Prefix& kept, int i, const float (&x)[W]) {
    int n = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) n += x[j] == kept.value && i + at(j) <= kept.index;
    return n;
  }
  // Bin of a logit, by descending logits, and past the last for weights of zero
  __device__ __forceinline__ int bin_of(float x) const { return s.bins.of(sample_depth(m, x, c)); }
  // Least ordered bits from lo on whose logit passes, as all above it do, hi for one (a
  // warp, 32 at a time)
  template <typename F>
  __device__ __forceinline__ uint32_t search(F passes, uint32_t lo, uint32_t hi) const {
    while (lo < hi) {
      const uint32_t step = (hi - lo) / 32 + 1;
      const uint32_t q = hi - lo >= lane() * step ? lo + lane() * step : hi;
      const unsigned hit = __ballot_sync(0xffffffffu, passes(order_value(q)));
      const int f = hit != 0 ? __ffs(hit) - 1 : 32;
      const uint32_t below = __shfl_sync(0xffffffffu, q, f > 0 ? f - 1 : 0);
      if (f < 32) hi = __shfl_sync(0xffffffffu, q, f);
      lo = f > 0 ? min(hi, below + 1) : hi;
    }
    return lo;
  }
  // sum over this and the threads before it, and over all; `upto`: over those before it,
  // which is bit for bit what the thread before this one is given
  template <typename T>
  __device__ __forceinline__ T block_scan(T x, T* part, T& total, T* upto = nullptr) const {
    T incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane() >= o) incl += y;
    }
    __syncthreads();
    if (lane() == 31) part[warp()] = incl;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const T y = part[i];
      if (i < warp()) before += y;
      total += y;
    }
    if (upto != nullptr) {
      const T last = __shfl_up_sync(0xffffffffu, incl, 1);
      *upto = lane() > 0 ? before + last : before;
    }
    return before + incl;
  }
  // f of what every CTA of the cluster has at p, four loads in flight at once
  template <typename T, typename F>
  __device__ __forceinline__ void gather(const T* p, F f) const {
#pragma unroll
    for (int b = 0; b < kMaxCtas; b += 4) {
      if (b >= ctas()) break;
      T v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (b + i < ctas()) v[i] = ld_cluster(p, b + i);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (b + i < ctas()) f(v[i]);
    }
  }
  // sum over the cluster's warps
  __device__ __forceinline__ uint64_t cluster_sum(const uint64_t* of) const {
    uint64_t v = 0;
#pragma unroll
    for (int j = 0; j < kMaxCtas * kWarps / 32; ++j) {
      const int i = j * 32 + lane();
      if (i < ctas() * kWarps) v += ld_cluster(of + i % kWarps, i / kWarps);
    }
    return warp_sum(v);
  }

  // Counts the row's logits by bin; finds top-k's bin (s.k_bin: kBins if all that have
  // weight are wanted) with the number before it, and the bins from p_first to p_last
  // that top-p's border lies in: for sure, by bounds of the sums (where the share's upper
  // bound is past the row's lower one, up to the last bin), and, with weights as in the
  // middle between the bounds and 5 or 2 parts in 10^4 of their sum to either side, in
  // all likelihood.
  __device__ __forceinline__ void count(int k, float share) {
    Hist& h = s.hist[level++ & 1];
    const Bins bins = s.bins;
    sweep([&](int, float x) {
      const int b = bins.of(sample_depth(m, x, c));
      if (b < kBins) atomicAdd(&h.coarse[b], 1u);
    });
    sync();
    constexpr int N = kBins / kThreads;
    static_assert(N == 4, "a thread's bins are one vector");
    uint32_t n[N] = {0, 0, 0, 0};
    gather(reinterpret_cast<const uint4*>(h.coarse) + threadIdx.x,
           [&](const uint4& v) { n[0] += v.x, n[1] += v.y, n[2] += v.z, n[3] += v.w; });
    uint32_t all;
    const uint32_t sum = n[0] + n[1] + n[2] + n[3];
    uint32_t before = block_scan(sum, reinterpret_cast<uint32_t*>(s.scan), all) - sum;
    const uint32_t want = k > 0 ? min(static_cast<uint32_t>(k), all) : all, first = min(before, want);
    if (threadIdx.x < 3) {
      s.k_bin = kBins, s.k_whole = 0;
      s.p_first[threadIdx.x] = s.p_last[threadIdx.x] = kBins - 1;
      s.n_first[threadIdx.x] = 0, s.n_last[threadIdx.x] = static_cast<int>(want);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (k > 0 && k <= all && before < want && before + n[j] >= want) {
        s.k_bin = threadIdx.x * N + j;
        s.k_before = static_cast<int>(before);
        s.k_whole = before + n[j] == want;
      }
      const uint32_t left = want > before ? want - before : 0;
      before += n[j];
      n[j] = min(n[j], left);  // what top-k leaves
    }
    if (share < 1.f) {
      // Sums of weights as they are at most and at least, a bin's all as heavy as where
      // it begins or ends; 10^-4 is far more than all roundings here.
      float most[N], least[N], sum_most = 0.f, sum_least = 0.f, all_most, all_least;
      float edge = exp2f(s.bins.from(threadIdx.x * N) * (-1.f / kSampleTable));
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float next = exp2f(s.bins.from(threadIdx.x * N + j + 1) * (-1.f / kSampleTable));
        sum_most += most[j] = static_cast<float>(n[j]) * edge;
        sum_least += least[j] = static_cast<float>(n[j]) * next;
        edge = next;
      }
      float to_most, to_least;
      const float end_most = block_scan(sum_most, s.scan_f, all_most, &to_most);
      const float end_least = block_scan(sum_least, reinterpret_cast<float*>(s.scan), all_least, &to_least);
      const float from = share * all_least * (1.f - 1e-4f);
      const float upto = fmaxf(share * all_most * (1.f + 1e-4f), 1e-30f);
      const float middle = 0.5f * (all_most + all_least), part = share * middle;
      const float early[2] = {part - 5e-4f * middle, part - 2e-4f * middle};
      const float late[2] = {fminf(part + 5e-4f * middle, middle * (1.f - 1e-6f)), fminf(part + 2e-4f * middle, middle * (1.f - 1e-6f))};
      uint32_t at = first;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int b = threadIdx.x * N + j;
        const uint32_t next_at = at + n[j];
        // a thread's last bin ends where the next thread begins: nothing falls between
        const float next_most = j < N - 1 ? to_most + most[j] : fmaxf(to_most, end_most);
        const float next_least = j < N - 1 ? to_least + least[j] : fmaxf(to_least, end_least);
        const float to = 0.5f * (to_most + to_least), next = 0.5f * (next_most + next_least);
        if ((to_most < from || b == 0) && next_most >= from) s.p_first[0] = b, s.n_first[0] = static_cast<int>(at);
        if (to_least < upto && next_least >= upto) s.p_last[0] = b, s.n_last[0] = static_cast<int>(next_at);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if ((to < early[k] || b == 0) && next >= early[k]) s.p_first[k + 1] = b, s.n_first[k + 1] = static_cast<int>(at);
          if (to < late[k] && next >= late[k]) s.p_last[k + 1] = b, s.n_last[k + 1] = static_cast<int>(next_at);
        }
        at = next_at, to_most = next_most, to_least = next_least;
      }
    }
    __syncthreads();
  }

  // Clears the next level's histograms
  __device__ __forceinline__ void clear() {
    uint4* h = reinterpret_cast<uint4*>(&s.hist[level & 1]);
    for (int i = threadIdx.x; i < static_cast<int>(sizeof(Hist) / 16); i += kThreads) h[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  __device__ static uint32_t key(float x) { return order_key(x + 0.f); }  // -0 counts as 0
  // The largest float with ordered bits up to hi: those of -0, which no logit has
  // (key), stand for what is below 0
  __device__ static float up_to(uint32_t hi) { return order_value(hi == 0x7FFFFFFFu ? hi - 1 : hi); }
  __device__ static int shift_of(uint32_t lo, uint32_t hi) { return max(0, 32 - __clz(hi - lo) - kFineBits); }

  // Takes `kept` down to the elements with ordered bits above hi and, of those within
  // [lo, hi], as many as bring their count or weight (MASS) up to `target`; with
  // `counted` the level's histograms are there.
  template <bool MASS>
  __device__ __forceinline__ void refine(Prefix& kept, uint32_t lo, uint32_t hi, uint64_t target, bool counted) {
    for (;; counted = false) {
      const int shift = shift_of(lo, hi);
      Hist& h = s.hist[level & 1];
      if (!counted) {
        clear();
        const float f_lo = order_value(lo), f_hi = up_to(hi);
        sweep([&](int i, float x) {
          if (x >= f_lo && x <= f_hi && kept.has(x, i)) add<MASS>(h, (hi - key(x)) >> shift, x);
        });
        sync();
      }
      ++level;
      static_assert(kFine == kThreads, "a bin a thread");
      uint64_t n = 0;
      uint32_t one = 0;
      gather(h.count + threadIdx.x, [&](uint32_t v) { one += v; });
      if (MASS)
        gather(h.weight + threadIdx.x, [&](uint64_t v) { n += v; });
      else
        n = one;
      if (threadIdx.x == 0) s.bin = -1;
      uint64_t all;
      const uint64_t before = block_scan(n, s.scan, all) - n;
      if (before < target && before + n >= target) {
        s.bin = threadIdx.x;
        s.before = before;
        s.in = n;
        s.alone = MASS ? one == 1 : before + n == target;
      }
      __syncthreads();
      if (s.bin < 0) return;  // less than target in all
      target -= s.before;
      hi -= static_cast<uint32_t>(s.bin) << shift;
      lo = hi - lo >= 1u << shift ? hi - ((1u << shift) - 1) : lo;
      const bool whole = s.alone != 0;
      if (whole || shift == 0) {
        const float v = order_value(lo);
        const int last = v == kept.value ? kept.index : INT_MAX;
        kept = Prefix{v, whole ? last : first_by_index<MASS>(v, last, target)};
        return;
      }
    }
  }
  // Counts a logit, and its weight
  template <bool MASS>
  __device__ __forceinline__ void add(Hist& h, uint32_t b, float x) const {
    atomicAdd(&h.count[b], 1u);
    if (MASS) add64(&h.weight[b], weight(x));
  }

  // Of the logits equal to v, up to index `last`: the index of the one
  // that brings their count or weight up to `target`; s.in is that of all.
  template <bool MASS>
  __device__ __forceinline__ int first_by_index(float v, int last, uint64_t target) {
    const uint64_t each = MASS ? weight(v) : 1;
    const uint64_t take = (target + each - 1) / each, have = s.in / each;
    if (take >= have) return last;
    uint64_t n = 0;
    sweep([&](int i, float x) { n += x == v && i <= last; });
    n = warp_sum(n);
    if (lane() == 0) s.count[warp()] = n;
    sync();
    uint64_t v4[4], left = take;
    load4(s.count, v4);
    const int at = owner_of(v4, left);  // the warp (of the cluster) that has the last one
    if (at / kWarps == rank()) nth(at % kWarps, left, [&](int i, float x) -> uint64_t { return x == v && i <= last; });
    sync();
    // nobody writes s.index again before the next sync() of all
    return ld_cluster(&s.index, at / kWarps);
  }

  // The index in the run of this CTA's warp `of` at which the sum of f first reaches
  // `want` >= 1, found by all its warps: an iteration of that run each.
  template <typename F>
  __device__ __forceinline__ int nth(int of, uint64_t want, F f) {
    const int r0 = min(s.g1, g0 + of * s.per_warp), r1 = min(s.g1, r0 + s.per_warp);
    for (int base = r0; base < r1; base += 32 * kWarps) {
      const int g = base + 32 * warp() + lane();
      float x[G::N];
      uint64_t v[G::N], sum = 0;
      if (g < r1) {
        G::get(fetch(g), x);
#pragma unroll
        for (int j = 0; j < G::N; ++j) sum += v[j] = f(g * G::N + j - head, x[j]);
      }
      uint64_t all;
      const uint64_t incl = block_scan(sum, s.scan, all);
      if (incl >= want && incl - sum < want) {  // one thread
        uint64_t at = incl - sum;
        int i = -1;
#pragma unroll
        for (int j = 0; j < G::N; ++j) {
          at += v[j];
          if (i < 0 && at >= want) i = g * G::N + j - head;
        }
        s.index = i;
      }
      __syncthreads();
      if (all >= want) return s.index;
      want -= all;
    }
    return -1;
  }
  // Which of the cluster's warps has the sum of v, its warps' values, reach `want` >= 1,
  // and what is left of `want` there (lane i of every warp: v of warps 4 i ..)
  __device__ __forceinline__ int owner_of(const uint64_t (&v)[4], uint64_t& want) const {
    const uint64_t sum = (v[0] + v[1]) + (v[2] + v[3]);
    const uint64_t incl = warp_scan(sum, lane());
    const int l = max(__ffs(__ballot_sync(0xffffffffu, incl >= want)) - 1, 0);
    uint64_t left = want - (incl - sum);
    int at = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (at == j && left > v[j]) {
        left -= v[j];
        at = j + 1;
      }
    want = __shfl_sync(0xffffffffu, left, l);
    return __shfl_sync(0xffffffffu, 4 * lane() + at, l);
  }
  // what the cluster's warps have at `of` + warp
  __device__ __forceinline__ void load4(const uint64_t* of, uint64_t (&v)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = 4 * lane() + j;
      v[j] = i < ctas() * kWarps ? ld_cluster(of + i % kWarps, i / kWarps) : 0;
    }
  }
  // token and probability: this CTA's logit i
  __device__ __forceinline__ void put(int i, float l, uint64_t total) const {
    p.token[blockIdx.x / ctas()] = i;
    const SampleTerm w = sample_term(m, l, c, s.table);
    const double v = static_cast<double>(w.v) * static_cast<double>(kSampleUnits);
    p.prob[blockIdx.x / ctas()] = static_cast<float>((v + v * static_cast<double>(w.x)) / static_cast<double>(total));
  }
  // Draws from what is kept: warp `owner` of the cluster has the one that brings its
  // kept sum up to `want`.
  __device__ __forceinline__ void draw(const Prefix& kept, int owner, uint64_t want, uint64_t total) {
    if (owner / kWarps != rank()) return;
    const int i = nth(owner % kWarps, want, [&](int i, float v) -> uint64_t { return kept.has(v, i) ? weight(v) : 0; });
    if (threadIdx.x == 0 && i >= 0) {
      float v[G::N];
      G::get(fetch((i + head) / G::N), v);
      float l = 0.f;
#pragma unroll
      for (int j = 0; j < G::N; ++j)
        if (j == (i + head) % G::N) l = v[j];
      put(i, l, total);
    }
  }

  // ---- lists: logits of the whole row in one CTA's registers, kItems a thread
  struct Items {
    float x[kItems];
    int i[kItems];
    uint64_t w[kItems];
  };
  __device__ __forceinline__ void push(float x, int i) {
    const int at = atomicAdd(&s.listed, 1);
    if (at < kList) s.list[at] = make_uint2(__float_as_uint(x), static_cast<uint32_t>(i));
  }
  // Numbers of logits that the cluster's CTAs have listed, and their sum
  __device__ __forceinline__ int listed(int (&n)[kMaxCtas]) const {
    int all = 0;
#pragma unroll
    for (int k = 0; k < kMaxCtas; ++k) n[k] = k < ctas() ? ld_cluster(&s.listed, k) : 0;
#pragma unroll
    for (int k = 0; k < kMaxCtas; ++k) all += min(n[k], kList + 1);
    return all;
  }
  // All of them, kList at most; places past them have no weight and -inf
  __device__ __forceinline__ void take(Items& t, const int (&n)[kMaxCtas]) const {
#pragma unroll
    for (int q = 0; q < kItems; ++q) {
      int at = threadIdx.x + q * kThreads, of = 0;
#pragma unroll
      for (int k = 0; k < kMaxCtas - 1; ++k)
        if (of == k && at >= n[k]) {
          at -= n[k];
          of = k + 1;
        }
      t.x[q] = -INFINITY;
      t.i[q] = -1;
      if (of < ctas() && at < min(n[of], kList)) {
        const uint2 v = ld_cluster(&s.list[at], of);
        t.x[q] = __uint_as_float(v.x);
        t.i[q] = static_cast<int>(v.y);
      }
    }
#pragma unroll
    for (int q = 0; q < kItems; ++q) t.w[q] = t.i[q] >= 0 ? weight(t.x[q]) : 0;
  }
  // One level: v by bin; the bin where their sum reaches `target` in s.bin, with the
  // sum before it in s.before and its own in s.in
  template <typename B>
  __device__ __forceinline__ bool level_of(const uint64_t (&v)[kItems], uint64_t target, B bin) {
    static_assert(kLocal == 2 * kThreads, "two bins a thread");
    uint64_t* h = s.hist[1].local;
    reinterpret_cast<uint4*>(h)[threadIdx.x] = make_uint4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kItems; ++q) {
      const int b = v[q] != 0 ? bin(q) : -1;
      if (b < 0) continue;
      add64(h + b, v[q]);
    }
    __syncthreads();
    const uint64_t n0 = h[2 * threadIdx.x], n1 = h[2 * threadIdx.x + 1];
    if (threadIdx.x == 0) s.bin = -1;
    uint64_t all;
    const uint64_t before = block_scan(n0 + n1, s.scan, all) - n0 - n1;
    if (before < target && before + n0 + n1 >= target) {
      const bool second = before + n0 < target;
      s.bin = 2 * threadIdx.x + second;
      s.before = before + (second ? n0 : 0);
      s.in = second ? n1 : n0;
    }
    __syncthreads();
    return s.bin >= 0;
  }
  // A bound that `most` of the threads' two values reach, and few more: by bins of equal
  // width from the largest to the least of them
  __device__ __forceinline__ float threads_kth(float a, float b, int most) {
    float hi = fmaxf(a, b), lo = fminf(a > -INFINITY ? a : INFINITY, b > -INFINITY ? b : INFINITY);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    }
    if (lane() == 0) s.max[warp()] = hi, s.low[warp()] = lo;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWarps; ++i) hi = fmaxf(hi, s.max[i]), lo = fminf(lo, s.low[i]);
    __syncthreads();  // the caller writes them anew
    const float scale = (kLocal - 1.f) / (hi - lo);
    const bool apart = scale < 1e30f && scale > 0.f;  // else one bin for all
    const float x[kItems] = {a, b};
    const uint64_t one[kItems] = {a > -INFINITY ? 1u : 0u, b > -INFINITY ? 1u : 0u};
    if (!level_of(one, static_cast<uint64_t>(most),
                  [&](int q) { return apart ? min(static_cast<int>((hi - x[q]) * scale), kLocal - 1) : 0; }))
      return -3.402823466e38f;  // fewer than `most`: what is wanted may lie below all of them
    if (!apart) return lo;
    const float t = hi - (static_cast<float>(s.bin) + 1.01f) / scale;  // and room for rounding
    return fmaxf(lo, t - (fabsf(hi) + fabsf(t)) * 2.384185791015625e-7f);
  }
  // The index at which the sum of v by index reaches `target`
  __device__ __forceinline__ int list_nth(const Items& t, const uint64_t (&v)[kItems], uint64_t target) {
    int lo = 0, hi = p.vocab - 1;
    for (;;) {
      const int shift = max(0, 32 - __clz(hi - lo) - kLocalBits);
      if (!level_of(v, target, [&](int q) { return t.i[q] >= lo && t.i[q] <= hi ? (t.i[q] - lo) >> shift : -1; })) return -1;
      target -= s.before;
      lo += s.bin << shift;
      hi = min(hi, lo + (1 << shift) - 1);
      if (shift == 0) return lo;
    }
  }
  // refine() of a list
  template <bool MASS>
  __device__ __forceinline__ void list_cut(const Items& t, Prefix& kept, uint32_t lo, uint32_t hi, uint64_t target) {
    uint64_t v[kItems];
    for (;;) {
      const int shift = max(0, 32 - __clz(hi - lo) - kLocalBits);
      const float f_lo = order_value(lo), f_hi = up_to(hi);
#pragma unroll
      for (int q = 0; q < kItems; ++q)
        v[q] = t.i[q] >= 0 && t.x[q] >= f_lo && t.x[q] <= f_hi && kept.has(t.x[q], t.i[q]) ? (MASS ? t.w[q] : 1) : 0;
      if (!level_of(v, target, [&](int q) { return static_cast<int>((hi - key(t.x[q])) >> shift); })) return;
      target -= s.before;
      hi -= static_cast<uint32_t>(s.bin) << shift;
      lo = hi - lo >= 1u << shift ? hi - ((1u << shift) - 1) : lo;
      const float value = order_value(lo), top = up_to(hi);
      int last = value == kept.value ? kept.index : INT_MAX;
      if (!MASS && target == s.in) {  // all of the bin
        kept = Prefix{value, last};
        return;
      }
      if (shift == 0) {
        const uint64_t each = MASS ? weight(value) : 1, take = (target + each - 1) / each, have = s.in / each;
        if (take < have) {
#pragma unroll
          for (int q = 0; q < kItems; ++q) v[q] = v[q] != 0 && t.x[q] == value;
          last = list_nth(t, v, take);
        }
        kept = Prefix{value, last};
        return;
      }
      if (MASS) {
        int n = 0;
#pragma unroll
        for (int q = 0; q < kItems; ++q) n += v[q] != 0 && t.x[q] >= value && t.x[q] <= top;
        const int threads = __syncthreads_count(n > 0);
        if (!__syncthreads_or(n > 1) && threads == 1) {  // one logit, wanted
          kept = Prefix{value, last};
          return;
        }
      }
    }
  }
};

template <int TYPE, bool RESIDENT, int PER_SM>
__global__ void __launch_bounds__(kThreads, PER_SM) sample_kernel(const SampleParams p) {
  constexpr int W = PER_SM == 1 ? 8 : 4;
  using R = Row<TYPE, RESIDENT, W>;
  using G = Group<TYPE>;
  __shared__ Shared s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = p.ctas, rank = static_cast<int>(cluster_ctarank()), r = blockIdx.x / C;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint8_t* row = static_cast<const uint8_t*>(p.logits) + r * p.stride * static_cast<long long>(sizeof(typename G::T));
  const uintptr_t base = reinterpret_cast<uintptr_t>(row) & ~static_cast<uintptr_t>(15);
  const int head = static_cast<int>((reinterpret_cast<uintptr_t>(row) - base) / sizeof(typename G::T));
  const int groups = static_cast<int>((static_cast<long long>(head) + p.vocab + G::N - 1) / G::N);
  const int per = (groups + C - 1) / C, per_warp = (per + kWarps - 1) / kWarps;
  const int g0 = min(groups, rank * per), g1 = min(groups, g0 + per);
  const int w0 = min(g1, g0 + warp * per_warp), w1 = min(g1, w0 + per_warp);
  auto whole = [&](int g) { return g * G::N >= head && (g + 1) * G::N <= head + p.vocab; };
  const int ends = (w0 < w1 && !whole(w0) ? 1 : 0) | (w1 - 1 > w0 && !whole(w1 - 1) ? 2 : 0);
  const int f0 = w0 + (ends & 1), f1 = w1 - (ends >> 1);
  R row_{s, p, reinterpret_cast<const uint8_t*>(base), f0, f1, ends, head, g0};
  R& x = row_;

  const bool loads = RESIDENT && f0 < f1;  // this warp, by a bulk copy
  if (loads && lane == 0) {
    mbar_init(&s.bar[warp], 1);
    fence_mbar_init();
    const uint32_t bytes = static_cast<uint32_t>(f1 - f0) * 16u;
    mbar_arrive_expect_tx(&s.bar[warp], bytes);
    bulk_load(x.slice() + (f0 - g0), x.data + static_cast<size_t>(f0) * 16, bytes, &s.bar[warp]);
  }
  const float T = p.temperature ? p.temperature[r] : 1.f, t = sample_temperature(T), u = p.u[r] + 0.f;  // -0 counts as 0
  const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f;
  const int top_k = p.top_k ? p.top_k[r] : 0;

  if (tid < kSampleTable) s.table[tid] = p.table[tid];
  for (int i = tid; i < static_cast<int>(sizeof(Hist) / 16); i += kThreads)
    reinterpret_cast<uint4*>(&s.hist[0])[i] = make_uint4(0, 0, 0, 0);
  if (tid == 0) s.listed = 0, s.g1 = g1, s.per_warp = per_warp;
  // 64-bit arithmetic is slow here, and is one thread's while the row comes in: by all
  // of them, with the table and the shares, it took 12 of 31 us (47 rows of 57381)
  if (tid == kThreads - 32) s.scale = sample_scale(t);
  if (tid == kThreads - 64 && min_p > 0.f) {
    const double x = static_cast<double>(t) * log(static_cast<double>(fminf(min_p, 1.f)));
    s.floor_hi = static_cast<float>(x);
    s.floor_lo = static_cast<float>(x - s.floor_hi);
  }
  __syncwarp();  // the barrier is there
  int bad = 0;
  if (RESIDENT && w0 < w1) {
    if (lane == 0 && (ends & 1) != 0) x.slice()[w0 - g0] = x.edge(w0);
    if (lane == 1 && (ends & 2) != 0) x.slice()[f1 - g0] = x.edge(f1);
    if (loads && !mbar_wait(&s.bar[warp], 0, p.limit_ns, nullptr)) {
      bad = 2;
      atomicCAS(p.status, 0, EBD_ERR_TIMEOUT);
      mbar_wait(&s.bar[warp], 0, p.limit_ns, nullptr);  // the copy lands before this CTA ends
    }
    __syncwarp();
  }

  // The largest logit; NaN, infinity and rows of nothing are refused.  And the largest
  // of the threads' least: a few in a hundred lie below it, unless more are masked.
  const bool by_k = top_k > 0 && top_k < p.vocab;
  const int most = (top_k + C - 1) / C;  // of a CTA's largest, for a list
  const bool few = by_k && top_k <= kList / 2 && most <= kListMost && T > 0.f;
  float m = -INFINITY, other = -INFINITY, low = INFINITY;  // two halves of a thread's logits
  x.template sweep4<4>([&](int, const float(&v)[4]) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(v[0]));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(other) : "f"(v[1]));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(v[2]));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(other) : "f"(v[3]));
    low = fminf(low, fminf(fminf(v[0], v[1]), fminf(v[2], v[3])));
  });
  bad |= m != m || other != other;
  low = low < INFINITY ? low : -INFINITY;
  if (few) {
    const float kth = x.threads_kth(m, other, most);
    if (tid == 0) s.kth = kth;
  }
  m = fmaxf(m, other);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    low = fmaxf(low, __shfl_xor_sync(0xffffffffu, low, o));
    bad |= __shfl_xor_sync(0xffffffffu, bad, o);
  }
  if (lane == 0) {
    s.max[warp] = m;
    s.low[warp] = low;
    s.bad[warp] = bad;
  }
  x.sync();
#pragma unroll
  for (int j = 0; j < kMaxCtas * kWarps / 32; ++j) {
    const int i = j * 32 + lane;
    if (i >= C * kWarps) continue;
    m = fmaxf(m, ld_cluster(&s.max[i % kWarps], i / kWarps));
    low = fmaxf(low, ld_cluster(&s.low[i % kWarps], i / kWarps));
    bad |= ld_cluster(&s.bad[i % kWarps], i / kWarps);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    low = fmaxf(low, __shfl_xor_sync(0xffffffffu, low, o));
    bad |= __shfl_xor_sync(0xffffffffu, bad, o);
  }
  const bool finite = !bad && m > -INFINITY && m < INFINITY;
  const bool valid = T >= 0.f && T < INFINITY && u >= 0.f && u < 1.f && top_p == top_p && min_p == min_p;
  if (!finite || !valid) {
    if (rank == 0 && tid == 0) {
      atomicCAS(p.status, 0, finite ? EBD_ERR_INVALID_ARG : EBD_ERR_NONFINITE);
      p.token[r] = -1;
      p.prob[r] = __int_as_float(0x7FC00000);
    }
    x.sync();  // the others have read this CTA's shared memory
    return;
  }
  x.m = m;
  if (T == 0.f) {
    int first = INT_MAX;
    x.sweep([&](int i, float v) {
      if (v == m) first = min(first, i);
    });
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0) s.first[warp] = first;
    x.sync();
    if (rank == 0 && warp == 0) {
      for (int i = lane; i < C * kWarps; i += 32) first = min(first, ld_cluster(&s.first[i % kWarps], i / kWarps));
      first = __reduce_min_sync(0xffffffffu, first);
      if (lane == 0) {
        p.token[r] = first;
        p.prob[r] = 1.f;
      }
    }
    x.sync();
    return;
  }

  x.c = s.scale;
  // the least logit that has weight: about 40 / log2(e) = 27.73 T below the largest
  const float near = fabsf(m) * 9.5367431640625e-7f;
  const uint32_t top = x.key(m), dead = order_key(fmaxf(m - 28.f * t - near, -3.402823466e38f));
  const float least = min_p > 0.f ? sample_floor(m, s.floor_hi, s.floor_lo) : -INFINITY;
  bool by_p = top_p < 1.f;
  Prefix kept{-3.402823466e38f, INT_MAX};
  uint64_t sum = 0;

  if (few) {
    float bound = m;
    x.gather(&s.kth, [&](float v) { bound = fminf(bound, v); });
    x.template sweep4<4>([&](int i, const float(&v)[4]) {
      if (!(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) >= bound)) return;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (v[j] >= bound) x.push(v[j], i + j);
    });
    x.sync();
    int n[kMaxCtas];
    if (x.listed(n) <= kList) {
      typename R::Items items;
      if (rank == 0) x.take(items, n);
      x.arrive();
      if (rank != 0) {  // done, once their lists are read
        x.wait();
        return;
      }
      x.template list_cut<false>(items, kept, x.key(bound), top, static_cast<uint64_t>(top_k));
      uint64_t total, v[kItems];
      auto weigh = [&]() {
#pragma unroll
        for (int q = 0; q < kItems; ++q) v[q] = items.i[q] >= 0 && kept.has(items.x[q], items.i[q]) ? items.w[q] : 0;
        x.block_scan((v[0] + v[1]) + (v[2] + v[3]), s.scan, total);
      };
      static_assert(kItems == 4, "the sum above");
      if (by_p) {
        weigh();
        x.template list_cut<true>(items, kept, max(dead, x.key(kept.value)), top, sample_share(top_p, total));
      }
      if (least > kept.value) kept = Prefix{least, INT_MAX};
      weigh();
      const int i = x.list_nth(items, v, sample_point(u, total) + 1);
#pragma unroll
      for (int q = 0; q < kItems; ++q)
        if (items.i[q] == i && i >= 0) x.put(i, items.x[q], total);
      x.wait();
      return;
    }
  }

  // exactly: among the floats about there, or, where they are too fine, by a search
  uint32_t floor = x.key(m - kSampleDead / x.c.hi) - 16;
  const uint32_t here = min(max(floor + lane, dead), top);
  const unsigned alive = __ballot_sync(0xffffffffu, sample_depth(m, order_value(here), x.c) <= kSampleDead);
  if (alive != 0 && (alive & 1) == 0)
    floor = __shfl_sync(0xffffffffu, here, __ffs(alive) - 1);
  else
    floor = x.search([&](float v) { return sample_depth(m, v, x.c) <= kSampleDead; }, dead, top);
  kept.value = order_value(floor);

  if (by_k || by_p) {
    if (tid == 0) s.bins = make_bins(1.5f * sample_depth(m, low, x.c));
    __syncthreads();
    x.count(by_k ? top_k : 0, top_p);
    const bool cut_k = by_k && s.k_bin < kBins;
    // where top-k's bin and top-p's bins begin and end, a bound a warp
    if (warp < 8) {
      const int b = warp == 0 ? s.k_bin : warp == 1 ? s.k_bin - 1 : (warp & 1) == 0 ? s.p_last[warp / 2 - 1] : s.p_first[warp / 2 - 1] - 1;
      const uint32_t q = b >= kBins ? floor : b < 0 ? top + 1 : x.search([&](float v) { return x.bin_of(v) <= b; }, floor, top);
      if (lane == 0) s.bound[warp] = q;
    }
    __syncthreads();
    const uint32_t k_lo = s.bound[0], k_hi = s.bound[1] - 1;
    if (cut_k) {
      if (s.k_whole)
        kept.value = order_value(k_lo);
      else
        x.template refine<false>(kept, k_lo, k_hi, static_cast<uint64_t>(top_k - s.k_before), false);
    }
    by_p = by_p && least <= x.up_to(s.bound[3] - 1);  // else min-p keeps less, whatever top-p does
    // Listed are the logits of all bins that the border may lie in, or, where they are
    // too many, of those that it should lie in.  It is seen whether it does: what is kept
    // above them is less than the share, and with what is listed no less.
    const bool sure = s.n_last[0] - s.n_first[0] <= kList;
    const int likely = s.n_last[1] - s.n_first[1] <= kList ? 1 : 2;
    bool list = sure || (s.n_last[likely] - s.n_first[likely] <= kList && least <= x.up_to(s.bound[2 * likely + 3] - 1));
    while (by_p) {
      const int which = list && !sure ? 2 * likely + 2 : 2;
      const uint32_t lo = max(s.bound[which], x.key(kept.value)), hi = s.bound[which + 1] - 1;
      const float f_lo = order_value(lo), f_hi = x.up_to(hi);
      const int shift = x.shift_of(lo, hi);
      const Prefix before = kept;
      uint64_t all = 0;
      if (!list) {
        x.clear();
      } else {
        if (tid == 0) s.listed = 0;  // of top-k's, too long a list
        __syncthreads();
      }
      Hist& h = s.hist[x.level & 1];
      const float cut = kept.cut();
      // about the bins: none further from the middle lies within
      const float mid = 0.5f * f_lo + 0.5f * f_hi, half = (0.5f * f_hi - 0.5f * f_lo) + 4.76837158203125e-7f * (fabsf(f_lo) + fabsf(f_hi));
      const bool ties = kept.index != INT_MAX;  // at top-k's border: in no sum above, being the last
      const uint64_t last = ties ? x.weight(kept.value) : 0;
      x.sweep_wide([&](int i, const float(&v)[W]) {
        if (!(R::largest(v) >= kept.value)) return;
        if (ties) all += x.ties(kept, i, v) * last;
        x.template weigh<true>(v, cut, f_hi, all, sum);
        float away = fabsf(v[0] - mid);
#pragma unroll
        for (int j = 1; j < W; ++j) away = fminf(away, fabsf(v[j] - mid));
        if (!(away <= half)) return;
#pragma unroll
        for (int j = 0; j < W; ++j) {
          if (!(v[j] >= f_lo && v[j] <= f_hi) || !kept.has(v[j], i + R::at(j))) continue;
          if (list)
            x.push(v[j], i + R::at(j));
          else
            x.template add<true>(h, (hi - x.key(v[j])) >> shift, v[j]);
        }
      });
      const uint64_t above = warp_sum(sum);
      all = warp_sum(all);
      if (lane == 0) s.part[warp] = above, s.rest[warp] = all;
      x.sync();
      if (list) {
        if (rank == 0) {
          typename R::Items items;
          int n[kMaxCtas];
          const bool fits = x.listed(n) <= kList;
          x.take(items, n);
          const uint64_t share = sample_share(top_p, x.cluster_sum(s.rest)), over = x.cluster_sum(s.part);
          uint64_t within;
          x.block_scan((items.w[0] + items.w[1]) + (items.w[2] + items.w[3]), s.scan, within);
          const bool there = fits && share > over && share - over <= within;
          x.template list_cut<true>(items, kept, lo, hi, share > over ? share - over : 1);
          if (least > kept.value) kept = Prefix{least, INT_MAX};
          // what is kept of the list goes to the sums of the warps that have it
          if (tid < kMaxCtas * kWarps) s.chunk[tid] = tid < C * kWarps ? ld_cluster(&s.part[tid % kWarps], tid / kWarps) : 0;
          __syncthreads();
#pragma unroll
          for (int q = 0; q < kItems; ++q) {
            if (items.i[q] < 0 || !kept.has(items.x[q], items.i[q])) continue;
            const int g = (items.i[q] + head) / G::N, of = g / per;
            add64(&s.chunk[of * kWarps + (g - of * per) / per_warp], items.w[q]);
          }
          __syncthreads();
          uint64_t v[4], left;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = s.chunk[4 * lane + j];
          const uint64_t total = warp_sum((v[0] + v[1]) + (v[2] + v[3]));
          left = sample_point(u, total) + 1;
          const int owner = x.owner_of(v, left);
          if (tid == 0) s.owner = there ? owner : -1, s.want = left, s.total = total, s.value = kept.value, s.last = kept.index;
        }
        x.sync();
        const int owner = ld_cluster(&s.owner, 0);
        if (owner < 0) {  // it does not
          list = false;
          sum = 0;
          kept = before;
          continue;
        }
        kept = Prefix{ld_cluster(&s.value, 0), ld_cluster(&s.last, 0)};
        x.draw(kept, owner, ld_cluster(&s.want, 0), ld_cluster(&s.total, 0));
        x.sync();
        return;
      }
      const uint64_t share = sample_share(top_p, x.cluster_sum(s.rest)), over = x.cluster_sum(s.part);
      x.template refine<true>(kept, lo, hi, share > over ? share - over : 1, true);
      if (least > kept.value) kept = Prefix{least, INT_MAX};
      x.sweep([&](int i, float v) {
        if (v <= f_hi && kept.has(v, i)) sum += x.weight(v);
      });
      break;
    }
  }
  if (!by_p) {
    if (least > kept.value) kept = Prefix{least, INT_MAX};
    const float cut = kept.cut();
    const uint64_t last = kept.index != INT_MAX ? x.weight(kept.value) : 0;
    uint64_t none = 0;
    x.sweep_wide([&](int i, const float(&v)[W]) {
      x.template weigh<false>(v, cut, 0.f, sum, none);
      if (last != 0) sum += x.ties(kept, i, v) * last;
    });
  }

  // what every warp's run weighs, and where u points
  sum = warp_sum(sum);
  if (lane == 0) s.count[warp] = sum;
  x.sync();
  uint64_t v[4];
  x.load4(s.count, v);
  const uint64_t total = warp_sum((v[0] + v[1]) + (v[2] + v[3]));
  uint64_t left = sample_point(u, total) + 1;
  const int owner = x.owner_of(v, left);
  x.draw(kept, owner, left, total);
  x.sync();
}

using Kernel = void (*)(SampleParams);
template <int PER_SM>
Kernel sample_kernel_of(int dtype, bool resident) {
  switch (dtype) {
    case EBD_LOGITS_F32:
      return resident ? sample_kernel<EBD_LOGITS_F32, true, PER_SM> : sample_kernel<EBD_LOGITS_F32, false, PER_SM>;
    case EBD_LOGITS_BF16:
      return resident ? sample_kernel<EBD_LOGITS_BF16, true, PER_SM> : sample_kernel<EBD_LOGITS_BF16, false, PER_SM>;
    default: return resident ? sample_kernel<EBD_LOGITS_F16, true, PER_SM> : sample_kernel<EBD_LOGITS_F16, false, PER_SM>;
  }
}
Kernel sample_kernel_of(int dtype, bool resident, bool alone) {
  return alone ? sample_kernel_of<1>(dtype, resident) : sample_kernel_of<2>(dtype, resident);
}

}  // namespace

cudaError_t launch_sample(SampleParams p, cudaStream_t st) {
  struct Table {
    SampleEntry v[kSampleTable];
    Table() {
      for (int j = 0; j < kSampleTable; ++j) v[j] = sample_entry(j);
    }
  };
  static const Table table;
  std::memcpy(p.table, table.v, sizeof(p.table));
  // CTAs per row (a cluster).  Few rows: as many as run at once, one CTA on an SM (so
  // many clusters of 8, 6, .. CTAs find room in the GPU's groups of SMs), with registers
  // to spare and two loads in turn.  Rows of 152064 floats, us with 2 / 3 / 4 / 5 / 6 / 8
  // CTAs, at a temperature: 14 rows 27 / 20 / 18 / 16 / 16 / 15, 20 rows 27 / 20 / 19 / 17
  // / 16 / 28, 28 rows 27 / 21 / 19 / 18 / 29 / 30, 36 rows 27 / 21 / 19 / 31 / 31 / 42, 44
  // rows 27 / 21 / 34 / 32 / 31 / 44.  Many rows: two CTAs on an SM; a cluster's barriers
  // and its launch cost more than they bring, but for long rows, or where they even out how
  // many CTAs an SM has: 512 rows of 152064 at a temperature 188 / 168 / 188 / 198 us with
  // 1 / 2 / 3 / 4 CTAs, of mixed settings 241 / 195 / 203 / 220, 80 rows 109 / 76 / 66 / 62,
  // 200 rows 164 / 114 / 101 / 104; 512 rows of 57000 at a temperature 72 / 77 with 1 / 2, by
  // top-k and top-p 101 / 90 / 98 / 117.
  struct { int rows, ctas; } const fits[] = {{14, 8}, {20, 6}, {24, 5}, {36, 4}, {44, 3}, {76, 2}};
  int alone = 0;
  for (const auto& f : fits)
    if (alone == 0 && p.rows <= f.rows) alone = f.ctas;
  const bool light = p.top_k == nullptr && p.top_p == nullptr;
  p.ctas = alone != 0 ? alone : p.rows <= 100 ? 3 : p.rows <= 128 || p.vocab >= (light ? 100000 : 50000) ? 2 : 1;
  const int most = (p.vocab + 11999) / 12000;  // a CTA wants some logits: one row of 16000 9.2 / 8.5 / 8.0 / 8.7 us with 1 / 2 / 4 / 8
  if (p.ctas > most) p.ctas = most;
  // a slice of a row in shared memory, where it leaves room for two CTAs on an SM
  const long long bytes = p.vocab * (p.dtype == EBD_LOGITS_F32 ? 4ll : 2ll) + 32;  // both ends rounded out
  const long long slice = ((bytes / 16 + p.ctas - 1) / p.ctas + 1) * 16;
  p.resident = slice <= kSliceBytes;
  const Kernel kernel = sample_kernel_of(p.dtype, p.resident != 0, alone != 0);
  if (p.resident) {  // here, so that a process loads the kernels that it calls alone: all took 17 ms
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSliceBytes);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(p.rows) * p.ctas, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = p.resident ? static_cast<size_t>(slice) : 0;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(p.ctas);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace ebd
