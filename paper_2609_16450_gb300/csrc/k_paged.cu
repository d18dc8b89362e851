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
// Both kernels move bytes, and are soon bound by what they issue instead (a piece
// of 16 bytes per thread and turn, K and V apart, took 130 instructions and 70 %
// of the issue slots).  A block is a row, or a part of one; a thread has J places
// of 8 values in it and moves both K's and V's, whose offsets, checks, lookup and
// search for the largest are one then: J = 2 where there are blocks enough for all
// SMs, 1 where there are not, so that a window of 32 rows is spread over them.  A
// write loads its rows while it looks its page up.  4096 rows of 32 128-wide heads
// in 8 bits, on one set of buffers: written in 16.1 us (20.4 with K and V apart;
// J = 1 17.5, 4 19.6), read in 13.9 (17.4; 15.0, 15.7); on several in turn 18.8 and
// 18.4, 5.4 TB/s.
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

// A place of 8 values in a row, of K and of V.  Offsets within a page fit 32 bits
// (the host sees to it).
template <int D>
struct Place {
  bool in;
  int j;
  __device__ __forceinline__ Place(const PagedRowsParams& p, int j_) : in(j_ < p.Hkv * (D / 8)), j(j_) {}
  // byte of the page's scales, and element that it lies at in its page
  __device__ __forceinline__ int scale_at(const PagedRowsParams& p, int off) const {
    return ((j / (D / 8)) << p.page_log2) + off;
  }
  __device__ __forceinline__ int at(const PagedRowsParams& p, int off) const {
    return scale_at(p, off) * D + j % (D / 8) * 8;
  }
};

// e4m3 codes of 8 bf16 values, by their row's exponent byte
__device__ __forceinline__ uint2 codes(const uint4& x, int e) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - min(e, 247)) << 23);  // 2^(127 - e)
  float y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(w[i] << 16) * inv;
    y[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u) * inv;
  }
  if (e >= 247) {  // below, no code is past 448
    if (e == 255) return make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(y[i], -240.f), 240.f);
  }
  uint32_t c[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    c[i] = __nv_cvt_float2_to_fp8x2(make_float2(y[4 * i], y[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
           __nv_cvt_float2_to_fp8x2(make_float2(y[4 * i + 2], y[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
  return make_uint2(c[0], c[1]);
}
// bits of the largest |value| of 8; past infinity's for NaN
__device__ __forceinline__ uint32_t largest(const uint4& x) {
  const uint32_t two = __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
  return max(two & 0xFFFFu, two >> 16);
}
// the exponent byte of a row, by the bits of its largest |value|
__device__ __forceinline__ int exponent(uint32_t amax) {
  return amax < 0x7F80u ? max(0, static_cast<int>(amax >> 7) - 8 + ((amax & 0x7Fu) > 0x60u ? 1 : 0)) : 255;
}

template <int D, bool E4M3, int J>
__global__ void __launch_bounds__(256) paged_write_kernel(const PagedRowsParams p) {
  constexpr int LPR = D / 8;  // lanes per row of a head, 8 values each
  const int r = blockIdx.x, j0 = blockIdx.y * J * blockDim.x + threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const bool skip = p.skip != nullptr && p.skip[r] != 0;
  if (J > 1 && skip) return;  // a row's bytes count, not its latency
  const __nv_bfloat16 *k = p.k + r * p.kv_stride, *v = p.v + r * p.kv_stride;
  uint4 x[J][2];
#pragma unroll
  for (int u = 0; u < J; ++u) {
    const Place<D> c(p, j0 + u * blockDim.x);
    x[u][0] = x[u][1] = make_uint4(0u, 0u, 0u, 0u);
    if (!c.in) continue;
    x[u][0] = __ldcs(reinterpret_cast<const uint4*>(k + c.j * 8));
    x[u][1] = __ldcs(reinterpret_cast<const uint4*>(v + c.j * 8));
  }
  long long page;
  int off;
  if (!row_slot(p, r, page, off) || skip) return;
  uint8_t *kp = p.k_pool + page * p.page_stride, *vp = p.v_pool + page * p.page_stride;
  const long long sp = (page * p.Hkv) << p.page_log2;
#pragma unroll
  for (int u = 0; u < J; ++u) {
    const Place<D> c(p, j0 + u * blockDim.x);
    const int at = c.at(p, off);
    if constexpr (!E4M3) {
      if (!c.in) break;
      *reinterpret_cast<uint4*>(kp + 2 * static_cast<long long>(at)) = x[u][0];
      *reinterpret_cast<uint4*>(vp + 2 * static_cast<long long>(at)) = x[u][1];
    } else {
      // K's and V's largest together; places past the row's end are whole rows of lanes
      uint32_t top = largest(x[u][0]) | largest(x[u][1]) << 16;
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (!c.in) continue;
      const int ek = exponent(top & 0xFFFFu), ev = exponent(top >> 16);
      *reinterpret_cast<uint2*>(kp + at) = codes(x[u][0], ek);
      *reinterpret_cast<uint2*>(vp + at) = codes(x[u][1], ev);
      if (c.j % LPR == 0) {
        p.k_scale[sp + c.scale_at(p, off)] = static_cast<uint8_t>(ek);
        p.v_scale[sp + c.scale_at(p, off)] = static_cast<uint8_t>(ev);
      }
    }
  }
}

// 8 bf16 values of codes and their row's exponent byte: exact
__device__ __forceinline__ uint4 values(const uint2& c, uint32_t e) {
  const float scale = __uint_as_float(max(e << 23, 1u << 22));  // 2^(e - 127)
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = (i < 2 ? c.x : c.y) >> (16 * (i & 1));
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D, bool E4M3, int J>
__global__ void __launch_bounds__(256) paged_read_kernel(const PagedRowsParams p) {
  const int r = blockIdx.x, j0 = blockIdx.y * J * blockDim.x + threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  long long page = 0;
  int off = 0;
  const bool held = row_slot(p, r, page, off);
  const uint8_t *kp = p.k_pool + page * p.page_stride, *vp = p.v_pool + page * p.page_stride;
  const long long sp = (page * p.Hkv) << p.page_log2;
  uint4 x[J][2];
  uint32_t e[J][2];
#pragma unroll
  for (int u = 0; u < J; ++u) {
    const Place<D> c(p, j0 + u * blockDim.x);
    x[u][0] = x[u][1] = make_uint4(0u, 0u, 0u, 0u);
    e[u][0] = e[u][1] = 0u;
    if (!c.in || !held) continue;
    const int at = c.at(p, off);
    if constexpr (!E4M3) {
      x[u][0] = __ldcs(reinterpret_cast<const uint4*>(kp + 2 * static_cast<long long>(at)));
      x[u][1] = __ldcs(reinterpret_cast<const uint4*>(vp + 2 * static_cast<long long>(at)));
    } else {
      const uint2 a = __ldcs(reinterpret_cast<const uint2*>(kp + at)), b = __ldcs(reinterpret_cast<const uint2*>(vp + at));
      x[u][0].x = a.x;
      x[u][0].y = a.y;
      x[u][1].x = b.x;
      x[u][1].y = b.y;
      e[u][0] = p.k_scale[sp + c.scale_at(p, off)];
      e[u][1] = p.v_scale[sp + c.scale_at(p, off)];
    }
  }
  __nv_bfloat16 *k = p.k + r * p.kv_stride, *v = p.v + r * p.kv_stride;
#pragma unroll
  for (int u = 0; u < J; ++u) {
    const Place<D> c(p, j0 + u * blockDim.x);
    if (!c.in) break;
    if constexpr (E4M3) {
      x[u][0] = values(make_uint2(x[u][0].x, x[u][0].y), e[u][0]);
      x[u][1] = values(make_uint2(x[u][1].x, x[u][1].y), e[u][1]);
    }
    *reinterpret_cast<uint4*>(k + c.j * 8) = x[u][0];
    *reinterpret_cast<uint4*>(v + c.j * 8) = x[u][1];
  }
}

// By dtype and head width; two places per thread where blocks abound.
template <class K>
cudaError_t launch_rows(const PagedRowsParams& p, int sms, cudaStream_t st, const K& kernel) {
  const int places = p.Hkv * (p.D / 8);
  const int threads = places >= 256 ? 256 : (places + 31) / 32 * 32;
  const bool many = p.R * static_cast<long long>(places) >= 2LL * 1024 * sms;
  const int each = threads * (many ? 2 : 1);
  return paged_launch(kernel(many), dim3(p.R, (places + each - 1) / each, 1), threads, 0, st, p);
}

}  // namespace

cudaError_t launch_paged_write(const PagedRowsParams& p, int sms, cudaStream_t st) {
  return launch_rows(p, sms, st, [&](bool many) {
    if (p.D == 64)
      return p.e4m3 ? (many ? paged_write_kernel<64, true, 2> : paged_write_kernel<64, true, 1>)
                    : (many ? paged_write_kernel<64, false, 2> : paged_write_kernel<64, false, 1>);
    return p.e4m3 ? (many ? paged_write_kernel<128, true, 2> : paged_write_kernel<128, true, 1>)
                  : (many ? paged_write_kernel<128, false, 2> : paged_write_kernel<128, false, 1>);
  });
}

cudaError_t launch_paged_read(const PagedRowsParams& p, int sms, cudaStream_t st) {
  return launch_rows(p, sms, st, [&](bool many) {
    if (p.D == 64)
      return p.e4m3 ? (many ? paged_read_kernel<64, true, 2> : paged_read_kernel<64, true, 1>)
                    : (many ? paged_read_kernel<64, false, 2> : paged_read_kernel<64, false, 1>);
    return p.e4m3 ? (many ? paged_read_kernel<128, true, 2> : paged_read_kernel<128, true, 1>)
                  : (many ? paged_read_kernel<128, false, 2> : paged_read_kernel<128, false, 1>);
  });
}

}  // namespace ebd
