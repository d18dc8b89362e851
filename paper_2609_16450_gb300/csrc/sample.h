// Launch parameters of the sampler (k_sample.cu).
#pragma once
#include <cuda_runtime.h>
#include <cstdint>

#include "sample_math.h"

namespace ebd {

struct SampleParams {
  const void* logits;
  long long stride;          // elements from row to row
  int rows, vocab, dtype;    // EBD_LOGITS_*
  const float *u, *temperature, *top_p, *min_p;
  const int* top_k;
  int* token;
  float* prob;
  int* status;
  int ctas;                  // CTAs (a cluster) per row
  int resident;              // a CTA's slice of the row stays in its shared memory
  uint64_t limit_ns;
  SampleEntry table[kSampleTable];
};

cudaError_t launch_sample(SampleParams p, cudaStream_t st);

}  // namespace ebd
