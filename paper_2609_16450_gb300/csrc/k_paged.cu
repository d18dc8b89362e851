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
// Both kernels move bytes: a block per row (what a sequence's lookup costs is
// then paid once), 16 bytes of bf16 per thread and turn.
#include <cuda_fp8.h>

#include "paged.h"

namespace ebd {

namespace {

// Sequence, page and place in it of row r: false where the row has none.
__device__ __forceinline__ bool row_slot(const PagedRowsParams& p, int r, long long& page, int& off) {
  // the row's sequence: as many as end at or before it
  int b = 0;
  for (int i = threadIdx.x; i - static_cast<int>(threadIdx.x) < p.B; i += blockDim.x)
    b += __syncthreads_count(i < p.B && p.cu_rows[i + 1] <= r);
  if (b >= p.B) return false;
  const int pos = p.row_pos[r];
  const int i = pos >> p.page_log2;
  if (pos < 0 || i >= p.max_pages) return false;
  const int pg = p.page_table[static_cast<long long>(b) * p.max_pages + i];
  if (pg < 0 || pg >= p.n_pages) return false;
  page = pg;
  off = pos & ((1 << p.page_log2) - 1);
  return true;
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(256) paged_write_kernel(const PagedRowsParams p) {
  constexpr int LPR = D / 8;  // lanes per row of a head, 8 values each
  const int r = blockIdx.x;
  long long page;
  int off;
  if (p.skip != nullptr && p.skip[r] != 0) return;
  if (!row_slot(p, r, page, off)) return;
  const int per = p.Hkv * LPR;  // 16-byte pieces of K, and of V
  for (int it = threadIdx.x; it < 2 * per; it += blockDim.x) {
    const bool is_v = it >= per;
    const int j = is_v ? it - per : it;
    const int head = j / LPR, l = j % LPR;
    const uint4 x = *reinterpret_cast<const uint4*>((is_v ? p.v : p.k) + r * p.kv_stride + head * D + l * 8);
    const long long slot = (static_cast<long long>(head) << p.page_log2) + off;
    uint8_t* pool = (is_v ? p.v_pool : p.k_pool) + page * p.page_stride;
    if constexpr (!E4M3) {
      *reinterpret_cast<uint4*>(pool + (slot * D + l * 8) * 2) = x;
    } else {
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
      uint32_t amax = 0;  // bits of the largest |value|; past infinity's for NaN
#pragma unroll
      for (int i = 0; i < 4; ++i) amax = max(amax, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
      // per is a multiple of LPR and the loop's stride of 32: a row's lanes are in it together
      const uint32_t lanes = (LPR == 16 ? 0xFFFFu : 0xFFu) << ((threadIdx.x & 31) & ~(LPR - 1));
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(lanes, amax, o));
      const bool finite = amax < 0x7F80u;
      const int e = finite ? max(0, static_cast<int>(amax >> 7) - 8 + ((amax & 0x7Fu) > 0x60u ? 1 : 0)) : 255;
      const float inv = __uint_as_float(static_cast<uint32_t>(254 - min(e, 247)) << 23);  // 2^(127 - e)
      const float top = e == 247 ? 240.f : 448.f;
      uint32_t code[2] = {0u, 0u};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float lo = __uint_as_float(w[i] << 16) * inv, hi = __uint_as_float(w[i] & 0xFFFF0000u) * inv;
        const float2 y = make_float2(fminf(fmaxf(lo, -top), top), fminf(fmaxf(hi, -top), top));
        const uint32_t c = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
        code[i >> 1] |= c << (16 * (i & 1));
      }
      if (!finite) code[0] = code[1] = 0x7F7F7F7Fu;
      *reinterpret_cast<uint2*>(pool + slot * D + l * 8) = make_uint2(code[0], code[1]);
      if (l == 0) {
        const long long at = ((page * p.Hkv + head) << p.page_log2) + off;
        (is_v ? p.v_scale : p.k_scale)[at] = static_cast<uint8_t>(e);
      }
    }
  }
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(256) paged_read_kernel(const PagedRowsParams p) {
  constexpr int LPR = D / 8;
  const int r = blockIdx.x;
  long long page = 0;
  int off = 0;
  const bool held = row_slot(p, r, page, off);
  const int per = p.Hkv * LPR;
  for (int it = threadIdx.x; it < 2 * per; it += blockDim.x) {
    const bool is_v = it >= per;
    const int j = is_v ? it - per : it;
    const int head = j / LPR, l = j % LPR;
    const long long slot = (static_cast<long long>(head) << p.page_log2) + off;
    const uint8_t* pool = (is_v ? p.v_pool : p.k_pool) + page * p.page_stride;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (held) {
      if constexpr (!E4M3) {
        x = *reinterpret_cast<const uint4*>(pool + (slot * D + l * 8) * 2);
      } else {
        const uint2 c = *reinterpret_cast<const uint2*>(pool + slot * D + l * 8);
        const long long at = ((page * p.Hkv + head) << p.page_log2) + off;
        const uint32_t e = (is_v ? p.v_scale : p.k_scale)[at];
        const float scale = __uint_as_float(e > 0 ? e << 23 : 1u << 22);  // 2^(e - 127)
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t two = (i < 2 ? c.x : c.y) >> (16 * (i & 1));
          const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
          const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);  // exact
          w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        x = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    *reinterpret_cast<uint4*>((is_v ? p.v : p.k) + r * p.kv_stride + head * D + l * 8) = x;
  }
}

int block_threads(const PagedRowsParams& p) {
  const int n = 2 * p.Hkv * (p.D / 8);
  return n >= 256 ? 256 : (n + 31) / 32 * 32;
}

}  // namespace

cudaError_t launch_paged_write(const PagedRowsParams& p, cudaStream_t st) {
  if (p.R <= 0) return cudaSuccess;
  const auto k = p.D == 64 ? (p.e4m3 ? paged_write_kernel<64, true> : paged_write_kernel<64, false>)
                           : (p.e4m3 ? paged_write_kernel<128, true> : paged_write_kernel<128, false>);
  k<<<p.R, block_threads(p), 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_paged_read(const PagedRowsParams& p, cudaStream_t st) {
  if (p.R <= 0) return cudaSuccess;
  const auto k = p.D == 64 ? (p.e4m3 ? paged_read_kernel<64, true> : paged_read_kernel<64, false>)
                           : (p.e4m3 ? paged_read_kernel<128, true> : paged_read_kernel<128, false>);
  k<<<p.R, block_threads(p), 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace ebd
