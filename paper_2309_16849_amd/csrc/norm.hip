// norm.hip -- layer norm over the channels of every pixel, of a residual sum
// with dropout, and its gradients (snls_norm, snls_norm_backward).
#include "philox.h"

namespace snls {

// A thread per pixel.
__global__ void __launch_bounds__(256) norm_kernel(const float* x, const float* branch, Drop d,
                                                   const float* __restrict__ gamma, const float* __restrict__ beta,
                                                   long long frames, int C, long long P, float eps, float* total,
                                                   float* y, float* stats) {
  const Philox gen(d);
  const long long px = frames * P;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < px; i += gridDim.x * 256LL) {
    const long long f = i / P, at = f * C * P + (i - f * P);
    float sum = 0.f;
    for (int c = 0; c < C; ++c) {
      const long long e = at + c * P;
      float v = x[e];
      if (branch) {
        float b = branch[e];
        if (d.rng) b = dropped(b, gen.word(e), d);
        v += b;
        total[e] = v;
      }
      sum += v;
    }
    const float* from = branch ? total : x;
    const float mean = sum / C;
    float sq = 0.f;
    for (int c = 0; c < C; ++c) {
      const float t = from[at + c * P] - mean;
      sq = fmaf(t, t, sq);
    }
    const float rstd = 1.f / sqrtf(sq / C + eps);
    for (int c = 0; c < C; ++c) {
      const float t = (from[at + c * P] - mean) * rstd;
      y[at + c * P] = fmaf(t, gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
    }
    if (stats) stats[i] = mean, stats[px + i] = rstd;
  }
}

// A thread per pixel: gradients of the input and the branch.
__global__ void __launch_bounds__(256) norm_grad_kernel(const float* grad_y, const float* grad_total,
                                                        const float* __restrict__ total,
                                                        const float* __restrict__ stats,
                                                        const float* __restrict__ gamma, Drop d, long long frames,
                                                        int C, long long P, float* grad_x, float* grad_branch) {
  const Philox gen(d);
  const long long px = frames * P;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < px; i += gridDim.x * 256LL) {
    const long long f = i / P, at = f * C * P + (i - f * P);
    const float mean = stats[i], rstd = stats[px + i];
    float sg = 0.f, sgx = 0.f;
    for (int c = 0; c < C; ++c) {
      const float g = grad_y[at + c * P] * (gamma ? gamma[c] : 1.f), xh = (total[at + c * P] - mean) * rstd;
      sg += g;
      sgx = fmaf(g, xh, sgx);
    }
    sg /= C, sgx /= C;
    for (int c = 0; c < C; ++c) {
      const long long e = at + c * P;
      const float g = grad_y[e] * (gamma ? gamma[c] : 1.f), xh = (total[e] - mean) * rstd;
      float r = rstd * (g - sg - xh * sgx);
      if (grad_total) r += grad_total[e];
      if (grad_branch) grad_branch[e] = d.rng ? dropped(r, gen.word(e), d) : r;
      grad_x[e] = r;
    }
  }
}

// Partial sums of a channel over a slice of the pixels, in 64 bits.
__global__ void __launch_bounds__(256) norm_weights_kernel(const float* __restrict__ grad_y,
                                                           const float* __restrict__ total,
                                                           const float* __restrict__ stats, long long frames, int C,
                                                           long long P, double* __restrict__ part) {
  __shared__ double sums[2][256];
  const int c = blockIdx.x;
  const long long px = frames * P;
  double sg = 0.0, sb = 0.0;
  for (long long i = blockIdx.y * 256LL + threadIdx.x; i < px; i += gridDim.y * 256LL) {
    const long long f = i / P, e = (f * C + c) * P + (i - f * P);
    const float g = grad_y[e];
    sg += (double)(g * ((total[e] - stats[i]) * stats[px + i]));
    sb += (double)g;
  }
  sums[0][threadIdx.x] = sg, sums[1][threadIdx.x] = sb;
  __syncthreads();
  for (int half = 128; half > 0; half /= 2) {
    if (threadIdx.x < half) {
      sums[0][threadIdx.x] += sums[0][threadIdx.x + half];
      sums[1][threadIdx.x] += sums[1][threadIdx.x + half];
    }
    __syncthreads();
  }
  if (threadIdx.x < 2) part[((long long)blockIdx.y * 2 + threadIdx.x) * C + c] = sums[threadIdx.x][0];
}

__global__ void __launch_bounds__(256) norm_weights_sum_kernel(const double* __restrict__ part, int slices, int C,
                                                               float* __restrict__ grad_gamma,
                                                               float* __restrict__ grad_beta) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= 2 * C) return;
  double s = 0.0;
  for (int k = 0; k < slices; ++k) s += part[(long long)k * 2 * C + i];
  (i < C ? grad_gamma : grad_beta)[i < C ? i : i - C] = (float)s;
}

constexpr int kSlices = 64;

size_t norm_backward_ws_bytes(const snls_norm_params& np) { return (size_t)kSlices * 2 * np.C * sizeof(double); }

static unsigned pixel_groups(const snls_norm_params& np) {
  const long long groups = (np.frames * np.pixels + 255) / 256;
  return (unsigned)(groups < 16384 ? groups : 16384);
}

snls_status launch_norm(const float* x, const float* branch, const Drop& drop, const float* gamma, const float* beta,
                        const snls_norm_params& np, float* total, float* y, float* stats, hipStream_t s) {
  hipLaunchKernelGGL(norm_kernel, dim3(pixel_groups(np)), dim3(256), 0, s, x, branch, drop, gamma, beta, np.frames,
                     np.C, np.pixels, np.eps, total, y, stats);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

// The sums over the pixels come first: grad_x may be grad_y.
snls_status launch_norm_backward(const float* grad_y, const float* grad_total, const float* total, const float* stats,
                                 const float* gamma, const Drop& drop, const snls_norm_params& np, float* grad_x,
                                 float* grad_branch, float* grad_gamma, float* grad_beta, double* ws, hipStream_t s) {
  if (grad_gamma) {
    hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)np.C, kSlices), dim3(256), 0, s, grad_y, total, stats,
                       np.frames, np.C, np.pixels, ws);
    hipLaunchKernelGGL(norm_weights_sum_kernel, dim3((unsigned)((2 * np.C + 255) / 256)), dim3(256), 0, s, ws, kSlices,
                       np.C, grad_gamma, grad_beta);
  }
  if (np.frames > 0)
    hipLaunchKernelGGL(norm_grad_kernel, dim3(pixel_groups(np)), dim3(256), 0, s, grad_y, grad_total, total, stats,
                       gamma, drop, np.frames, np.C, np.pixels, grad_x, grad_branch);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
