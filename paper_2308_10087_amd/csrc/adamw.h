// The AdamW step (adamw.hip) as the training loop calls it.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

#include "../../include/gnntrain.h"

struct AdamwRates {
  float lr, beta1, beta2, eps;
};
// why a list is refused; empty: it is not
std::string adamw_check(const gnntrain_adamw_tensor *t, int n, int bits, const float *grad_scale);
// a hipError_t; the list has been checked
int launch_adamw(const gnntrain_adamw_tensor *t, int n, int bits, const AdamwRates &r, const float *grad_scale, int64_t step, uint64_t seed, hipStream_t s);
