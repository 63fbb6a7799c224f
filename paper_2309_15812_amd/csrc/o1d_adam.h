// Host-side interface of the AdamW step over many tensors.
#pragma once

#include "o1d_rows.h"

namespace o1d {
namespace rows {

constexpr int kAdamGroup = 128;  // values of an 8-bit state that share a scale; parts of the states start at multiples of it

struct AdamTensor {
  void* p;
  const void* g;
  long long n, at;  // values, and where their part of the states starts
};

struct AdamState {
  void *m, *v;            // float32, or e4m3 (of v the root)
  float *ms, *vs;         // 8 bits: a scale for each 128 values
  float* master;          // (or NULL) the parameters in float32
  int* step;              // {steps taken, 0}
  int bits;
};

struct AdamHyper {
  float lr, beta1, beta2, eps, decay;
  double beta1_64, beta2_64;
  float rest1, rest2, keep;  // 1 - beta1, 1 - beta2, 1 - lr decay
  const float* lr_at;     // (or NULL) device value of the learning rate
  const float* norm;      // (or NULL) the gradients' norm, to be limited to max_norm
  float max_norm;
  bool follow;            // with masters: parameters that were written since are read
};

// The count of steps that a call finds in device memory, where no check of the host's sees it: one that no
// call has left is read as the nearest that one may have.
__host__ __device__ inline int steps_taken(int found) { return found < 0 ? 0 : (found < 0x7ffffffe ? found : 0x7ffffffe); }
// b^t for t >= 0, by squaring: at most 31 times whatever t is.
__host__ __device__ inline double power(double b, int t) {
  double r = 1.;
  for (uint32_t k = (uint32_t)t; k; k >>= 1, b *= b)
    if (k & 1) r *= b;
  return r;
}

constexpr int kAdamMost = 112;  // tensors of a launch (what its arguments hold)
// Tensors 0 .. count - 1 of a call; the call's last launch counts the step.
hipError_t launch_adam(Dtype pdt, Dtype gdt, const AdamTensor* t, int count, const AdamState& s, const AdamHyper& h,
                       hipStream_t stream);

constexpr int kNormBlocks = 256;  // partial sums (float64) of a call
// norm = sqrt(sum of squares over all gradients); part: kNormBlocks doubles; arrived: a device integer that is 0
hipError_t launch_grad_norm(Dtype gdt, const AdamTensor* t, int count, double* part, int* arrived, float* norm,
                            hipStream_t stream);

}  // namespace rows
}  // namespace o1d
