// dropout.hip -- dropout of a list of values, on its own or added to a residual
// (snls_dropout).
#include "philox.h"

namespace snls {

__global__ void __launch_bounds__(256) dropout_kernel(const float* x, const float* residual, Drop d, long long n,
                                                      float* out) {
  const Philox gen(d);
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
    float v = x[i];
    if (d.rng) v = dropped(v, gen.word(i), d);
    out[i] = residual ? residual[i] + v : v;
  }
}

snls_status launch_dropout(const float* x, const float* residual, const Drop& drop, long long n, float* out,
                           hipStream_t s) {
  const long long groups = (n + 255) / 256;
  hipLaunchKernelGGL(dropout_kernel, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0, s, x, residual,
                     drop, n, out);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
