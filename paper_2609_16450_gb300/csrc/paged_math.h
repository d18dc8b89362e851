// Arithmetic of the paged attention's softmax that its loops and ranges rest
// on, for the kernels and, compiled by a host compiler, for tests.
#pragma once
#include <cmath>

#ifdef __CUDACC__
#define EBD_HD __host__ __device__ __forceinline__
#else
#define EBD_HD inline
#endif

namespace ebd {

// A row's probabilities are 2^(y - ref), y its scores in log2 units, rounded to
// 32 bits before the reference is taken off (not in one fused operation, but for a
// power of two): what is left of y against a reference near it is then exact,
// however large y is.
//
// The tcgen05 kernel does a half step of 64 keys again, after moving the
// reference, where the largest y - ref, `top`, is past 24.  A row without a
// reference yet (started = false, ref = 0) takes its first one so, exactly.  From
// 2^24 on, where nothing is left of the probabilities so far and ref + top may
// miss y by any number of units, a row begins anew.  So one move is enough, or two.
constexpr float kPagedFar = 24.f, kPagedAnew = 16777216.f;
constexpr int kPagedMoves = 3;  // of a half step, at most

EBD_HD bool paged_far(float top, bool started) { return started ? top > kPagedFar : top > -INFINITY; }
// Moves ref; returns the log2 of what probabilities so far lose by it: a whole
// number, so that they scale exactly.
EBD_HD float paged_move(float top, float& ref, bool& started) {
  if (started && top >= kPagedAnew) {
    ref = 0.f;
    started = false;
    return INFINITY;
  }
  const float up = started ? ceilf(top) : top, lost = started ? up : 0.f;
  ref += up;
  started = true;
  return lost;
}

// The mma.sync kernel's 8-bit caches' P is f16, and holds probabilities times their
// values' scales.  What is taken off a row's scores is its largest product of both,
// `top` in log2 units, less kPagedUp, so that this product becomes 2^kPagedUp.  Past
// 2^22 (steps of 0.5), where 32 bits soon do not resolve offsets from a score any
// more, `top` is the largest score itself: no product is past 2^8 then, the
// rounding of the difference in it, and such keys' probabilities are 1 at least.
constexpr float kPagedUp = 7.f, kPagedCoarse = 4194304.f;
EBD_HD bool paged_coarse(float top) { return fabsf(top) >= kPagedCoarse && top > -INFINITY; }
EBD_HD float paged_product_ref(float m, float top) { return fmaxf(m, top - kPagedUp); }

}  // namespace ebd
