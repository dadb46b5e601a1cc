// dropout.hip -- dropout of a list of values, on its own or added to a residual
// (snls_dropout).
//
// 8 bytes a value, 12 with a residual, and 20 products of 32 by 32 bits per four
// values for the mask: vector instructions are issued in 0.45 of the time (0.29 with
// a residual), and bandwidth bounds it (31 million values 44.9 us, 5.6 TB/s; 25
// million with a residual 52.9, 5.7).  A lane takes four consecutive values, the
// words of one block.
#include "lanes.h"
#include "philox.h"

namespace snls {

__global__ void __launch_bounds__(256) dropout_kernel(const float* x, const float* residual, Drop d, long long n,
                                                      float* out) {
  const Philox gen(d);
  for (long long i = (blockIdx.x * 256LL + threadIdx.x) * 4; i < n; i += gridDim.x * 1024LL) {
    const int cnt = (int)min(4LL, n - i);
    float v[4], r[4] = {};
    load_run<4>(x + i, cnt, v);
    if (residual) load_run<4>(residual + i, cnt, r);
    if (d.rng) {
      unsigned w[4];
      gen.run<4>(i, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = dropped(v[j], w[j], d);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = residual ? r[j] + v[j] : v[j];
    store_run<4>(out + i, cnt, v);
  }
}

snls_status launch_dropout(const float* x, const float* residual, const Drop& drop, long long n, float* out,
                           hipStream_t s) {
  const long long groups = (n + 1023) / 1024;
  hipLaunchKernelGGL(dropout_kernel, dim3((unsigned)(groups < 65536 ? groups : 65536)), dim3(256), 0, s, x, residual,
                     drop, n, out);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
