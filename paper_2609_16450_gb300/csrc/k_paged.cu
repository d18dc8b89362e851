// Rows of the paged K/V cache: written into pages, quantised on the way where
// the cache holds 8 bits, and read back.
//
// An e4m3 cache holds row x of D values (one position, one head, K or V) as
// codes round_e4m3(x / 2^k) with the exponent byte k + 127, where 2^k is the
// least power of two, k >= -127, with max |x| <= 448 * 2^k.  With m = 1.f * 2^E
// the largest |x|, k = E - 8, or E - 7 where 1.f > 1.75 (448 = 1.75 * 2^8): it
// is read off the bits of m.  A power of two makes x / 2^k and code * 2^k exact,
// and code * 2^k a bf16 value, so that reading back rounds nothing and the
// attention may use the codes as bf16 operands; a free scale would win no
// precision, e4m3 being a floating-point format.  At k = 120, the most there
// is, codes stop at 240: 256 * 2^120 would be infinite in bf16.  A row with a
// value that is not finite is NaN as a whole (exponent byte 255, codes 0x7F), so
// that the attention learns of it from the scale, not from every code.
//
// Both kernels move bytes.  A block is a row, or a part of one: 256 threads by U
// pieces of 16 bytes of bf16, U = 4 where there are blocks enough for all SMs, so
// that what a row's lookup costs (three loads, one after another) is shared by
// more bytes, and 1 where there are not, so that a window of 32 rows is spread
// over them.  A write loads its rows while it looks its page up.
#include <cuda_fp8.h>

#include "paged.h"

namespace ebd {

namespace {

// Sequence, page and place in it of row r: false where the row has none.
__device__ __forceinline__ bool row_slot(const PagedRowsParams& p, int r, long long& page, int& off) {
  const int pos = p.row_pos[r];
  // the row's sequence: as many as end at or before it
  int b = 0;
  for (int i = threadIdx.x; i - static_cast<int>(threadIdx.x) < p.B; i += blockDim.x)
    b += __syncthreads_count(i < p.B && p.cu_rows[i + 1] <= r);
  if (b >= p.B) return false;
  const int i = pos >> p.page_log2;
  if (pos < 0 || i >= p.max_pages) return false;
  const int pg = p.page_table[static_cast<long long>(b) * p.max_pages + i];
  if (pg < 0 || pg >= p.n_pages) return false;
  page = pg;
  off = pos & ((1 << p.page_log2) - 1);
  return true;
}

// A piece of a row: 8 values of a head's K or V.  Its places within a row and
// within a page fit 32 bits (the host sees to it): both kernels are bound by
// what they issue as much as by what they move.
template <int D>
struct Piece {
  bool in, is_v;
  int j;  // of K's (V's) pieces of the row
  __device__ __forceinline__ Piece(const PagedRowsParams& p, int it) {
    const int per = p.Hkv * (D / 8);  // pieces of K, and of V
    in = it < 2 * per;
    is_v = it >= per;
    j = is_v ? it - per : it;
  }
  __device__ __forceinline__ __nv_bfloat16* row(const PagedRowsParams& p, long long at) const {
    return (is_v ? p.v : p.k) + at + j * 8;
  }
  // element that it lies at in its page, and byte of the page's scales
  __device__ __forceinline__ int at(const PagedRowsParams& p, int off) const {
    return scale_at(p, off) * D + j % (D / 8) * 8;
  }
  __device__ __forceinline__ int scale_at(const PagedRowsParams& p, int off) const {
    return ((j / (D / 8)) << p.page_log2) + off;
  }
};
// The page in the pools and in the scales.
struct Page {
  uint8_t *k, *v, *ks, *vs;
  __device__ __forceinline__ Page(const PagedRowsParams& p, long long page) {
    k = p.k_pool + page * p.page_stride;
    v = p.v_pool + page * p.page_stride;
    const long long s = (page * p.Hkv) << p.page_log2;
    ks = p.k_scale + s;
    vs = p.v_scale + s;
  }
};

template <int D, bool E4M3, int U>
__global__ void __launch_bounds__(256) paged_write_kernel(const PagedRowsParams p) {
  constexpr int LPR = D / 8;  // lanes per row of a head, 8 values each
  const int r = blockIdx.x, it0 = blockIdx.y * U * blockDim.x + threadIdx.x;
  const long long src = r * p.kv_stride;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const bool skip = p.skip != nullptr && p.skip[r] != 0;
  if (U > 1 && skip) return;  // a row's bytes count, not its latency
  uint4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Piece<D> c(p, it0 + u * blockDim.x);
    if (c.in) x[u] = __ldcs(reinterpret_cast<const uint4*>(c.row(p, src)));
  }
  long long page;
  int off;
  if (!row_slot(p, r, page, off) || skip) return;
  const Page pg(p, page);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Piece<D> c(p, it0 + u * blockDim.x);
    if (!c.in) break;
    uint8_t* pool = c.is_v ? pg.v : pg.k;
    if constexpr (!E4M3) {
      *reinterpret_cast<uint4*>(pool + 2 * static_cast<long long>(c.at(p, off))) = x[u];
    } else {
      const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      // bits of the largest |value|; past infinity's for NaN
      uint32_t two = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu),
                              __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
      // pieces of K and of V are multiples of LPR, and the block's threads of 32: a row's lanes are in it together
      const uint32_t lanes = (LPR == 16 ? 0xFFFFu : 0xFFu) << ((threadIdx.x & 31) & ~(LPR - 1));
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) two = __vmaxu2(two, __shfl_xor_sync(lanes, two, o));
      const uint32_t amax = max(two & 0xFFFFu, two >> 16);
      const bool finite = amax < 0x7F80u;
      const int e = finite ? max(0, static_cast<int>(amax >> 7) - 8 + ((amax & 0x7Fu) > 0x60u ? 1 : 0)) : 255;
      const float inv = __uint_as_float(static_cast<uint32_t>(254 - min(e, 247)) << 23);  // 2^(127 - e)
      float y[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[2 * i] = __uint_as_float(w[i] << 16) * inv;
        y[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u) * inv;
      }
      if (e == 247) {  // below, no code is past 448
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(y[i], -240.f), 240.f);
      }
      uint32_t code[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        code[i] = __nv_cvt_float2_to_fp8x2(make_float2(y[4 * i], y[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
                  __nv_cvt_float2_to_fp8x2(make_float2(y[4 * i + 2], y[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
      if (!finite) code[0] = code[1] = 0x7F7F7F7Fu;
      *reinterpret_cast<uint2*>(pool + c.at(p, off)) = make_uint2(code[0], code[1]);
      if (c.j % LPR == 0) (c.is_v ? pg.vs : pg.ks)[c.scale_at(p, off)] = static_cast<uint8_t>(e);
    }
  }
}

template <int D, bool E4M3, int U>
__global__ void __launch_bounds__(256) paged_read_kernel(const PagedRowsParams p) {
  const int r = blockIdx.x, it0 = blockIdx.y * U * blockDim.x + threadIdx.x;
  const long long dst = r * p.kv_stride;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  long long page = 0;
  int off = 0;
  const bool held = row_slot(p, r, page, off);
  const Page pg(p, page);
  uint4 x[U];
  uint32_t e[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Piece<D> c(p, it0 + u * blockDim.x);
    x[u] = make_uint4(0u, 0u, 0u, 0u);
    e[u] = 0;
    if (!c.in || !held) continue;
    const uint8_t* pool = c.is_v ? pg.v : pg.k;
    if constexpr (!E4M3) {
      x[u] = __ldcs(reinterpret_cast<const uint4*>(pool + 2 * static_cast<long long>(c.at(p, off))));
    } else {
      const uint2 code = __ldcs(reinterpret_cast<const uint2*>(pool + c.at(p, off)));
      x[u].x = code.x;
      x[u].y = code.y;
      e[u] = (c.is_v ? pg.vs : pg.ks)[c.scale_at(p, off)];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Piece<D> c(p, it0 + u * blockDim.x);
    if (!c.in) break;
    if constexpr (E4M3) {
      const float scale = __uint_as_float(max(e[u] << 23, 1u << 22));  // 2^(e - 127)
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t two = (i < 2 ? x[u].x : x[u].y) >> (16 * (i & 1));
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);  // exact
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
      x[u] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    *reinterpret_cast<uint4*>(c.row(p, dst)) = x[u];
  }
}

// By dtype and head width; many pieces per thread where blocks abound.
template <class K>
cudaError_t launch_rows(const PagedRowsParams& p, int sms, cudaStream_t st, const K& kernel) {
  const int pieces = 2 * p.Hkv * (p.D / 8);
  const int threads = pieces >= 256 ? 256 : (pieces + 31) / 32 * 32;
  const bool many = p.R * static_cast<long long>(pieces) >= 4LL * 1024 * sms;
  const int each = threads * (many ? 4 : 1);
  return paged_launch(kernel(many), dim3(p.R, (pieces + each - 1) / each, 1), threads, 0, st, p);
}

}  // namespace

cudaError_t launch_paged_write(const PagedRowsParams& p, int sms, cudaStream_t st) {
  return launch_rows(p, sms, st, [&](bool many) {
    if (p.D == 64)
      return p.e4m3 ? (many ? paged_write_kernel<64, true, 4> : paged_write_kernel<64, true, 1>)
                    : (many ? paged_write_kernel<64, false, 4> : paged_write_kernel<64, false, 1>);
    return p.e4m3 ? (many ? paged_write_kernel<128, true, 4> : paged_write_kernel<128, true, 1>)
                  : (many ? paged_write_kernel<128, false, 4> : paged_write_kernel<128, false, 1>);
  });
}

cudaError_t launch_paged_read(const PagedRowsParams& p, int sms, cudaStream_t st) {
  return launch_rows(p, sms, st, [&](bool many) {
    if (p.D == 64)
      return p.e4m3 ? (many ? paged_read_kernel<64, true, 4> : paged_read_kernel<64, true, 1>)
                    : (many ? paged_read_kernel<64, false, 4> : paged_read_kernel<64, false, 1>);
    return p.e4m3 ? (many ? paged_read_kernel<128, true, 4> : paged_read_kernel<128, true, 1>)
                  : (many ? paged_read_kernel<128, false, 4> : paged_read_kernel<128, false, 1>);
  });
}

}  // namespace ebd
