// norm.hip -- layer norm over the channels of every pixel, of a residual sum
// with dropout, and its gradients (snls_norm, snls_norm_backward).
#include <algorithm>

#include "lanes.h"
#include "philox.h"

namespace snls {

// What a call's kernels share.
struct NormGeo {
  long long frames, P;
  long long tiles, per_frame;  // runs of 64 * V pixels, of a frame
  int C, n;                    // n: channels a wave takes
  float eps;
};

// Frames: a workgroup of W waves takes 64 * V consecutive pixels, V a lane, and
// every wave up to R channels of them; the values stay in registers from their
// only read on, and the sums over the channels are joined in LDS: first the
// mean, then the squares of the differences from it.
template <int V, int R>
__global__ void __launch_bounds__(1024) norm_tile_kernel(const float* x, const float* branch, Drop d,
                                                         const float* __restrict__ gamma,
                                                         const float* __restrict__ beta, NormGeo g, float* total,
                                                         float* y, float* stats) {
  extern __shared__ float part[];  // sums, then squares: a row a wave
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Philox gen(d);
  // (a row of sums is written again only behind a barrier that follows its last read)
  for (long long tile = blockIdx.x; tile < g.tiles; tile += gridDim.x) {
    const long long f = tile / g.per_frame, p = (tile - f * g.per_frame) * (64 * V) + lane * V;
    const int cnt = (int)max(0LL, min((long long)V, g.P - p));
    const int c0 = wv * g.n, n = min(g.n, g.C - c0);
    const long long at = (f * g.C + c0) * g.P + (cnt > 0 ? p : 0);
    float s[R][V];
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n) load_run<V>(x + at + c * g.P, cnt, s[c]);
    if (branch) {
#pragma unroll
      for (int c = 0; c < R; ++c)
        if (c < n) {
          float b[V];
          load_run<V>(branch + at + c * g.P, cnt, b);
          if (d.rng) {
            unsigned w[V];
            gen.run<V>(at + c * g.P, w);
#pragma unroll
            for (int j = 0; j < V; ++j) b[j] = dropped(b[j], w[j], d);
          }
#pragma unroll
          for (int j = 0; j < V; ++j) s[c][j] += b[j];
          store_run<V>(total + at + c * g.P, cnt, s[c]);
        }
    }
    // the sum over all channels of what every wave has of its own
    auto joined = [&](float* own, float* rows) {
      if (waves == 1) return;
#pragma unroll
      for (int j = 0; j < V; ++j) rows[(wv * V + j) * 64 + lane] = own[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) own[j] = 0.f;
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int j = 0; j < V; ++j) own[j] += rows[(w * V + j) * 64 + lane];
    };
    float mean[V] = {}, sq[V] = {};
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n)
#pragma unroll
        for (int j = 0; j < V; ++j) mean[j] += s[c][j];
    joined(mean, part);
#pragma unroll
    for (int j = 0; j < V; ++j) mean[j] /= g.C;
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          s[c][j] -= mean[j];
          sq[j] = fmaf(s[c][j], s[c][j], sq[j]);
        }
    joined(sq, part + waves * V * 64);
    float rstd[V];
#pragma unroll
    for (int j = 0; j < V; ++j) rstd[j] = 1.f / sqrtf(sq[j] / g.C + g.eps);
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n) {
        const float ga = gamma ? gamma[c0 + c] : 1.f, be = beta ? beta[c0 + c] : 0.f;
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = fmaf(s[c][j] * rstd[j], ga, be);
        store_run<V>(y + at + c * g.P, cnt, o);
      }
    if (stats && wv == 0) {
      store_run<V>(stats + f * g.P + (cnt > 0 ? p : 0), cnt, mean);
      store_run<V>(stats + (g.frames + f) * g.P + (cnt > 0 ? p : 0), cnt, rstd);
    }
  }
}

// Sum over the G lanes of a group.
template <int G>
SNLS_DEV float group_sum(float v) {
#pragma unroll
  for (int m = G / 2; m > 0; m /= 2) v += __shfl_xor(v, m);
  return v;
}

// Tokens: G lanes take one, four consecutive channels a lane and N times that
// many; one read.
template <int G, int N>
__global__ void __launch_bounds__(256) norm_token_kernel(const float* x, const float* branch, Drop d,
                                                         const float* __restrict__ gamma,
                                                         const float* __restrict__ beta, NormGeo g, float* total,
                                                         float* y, float* stats) {
  const int l = threadIdx.x & (G - 1);
  const Philox gen(d);
  for (long long row = blockIdx.x * (256LL / G) + threadIdx.x / G; row < g.frames; row += gridDim.x * (256LL / G)) {
    const long long at = row * g.C;
    float s[N][4], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = (k * G + l) * 4, cnt = max(0, min(4, g.C - c));
      load_run<4>(x + at + (cnt > 0 ? c : 0), cnt, s[k]);
      if (branch && cnt > 0) {
        float b[4];
        load_run<4>(branch + at + c, cnt, b);
        if (d.rng) {
          unsigned w[4];
          gen.run<4>(at + c, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) b[j] = dropped(b[j], w[j], d);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s[k][j] += b[j];
        store_run<4>(total + at + c, cnt, s[k]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += s[k][j];
    }
    const float mean = group_sum<G>(sum) / g.C;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int cnt = g.C - (k * G + l) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[k][j] = j < cnt ? s[k][j] - mean : 0.f;
        sq = fmaf(s[k][j], s[k][j], sq);
      }
    }
    const float rstd = 1.f / sqrtf(group_sum<G>(sq) / g.C + g.eps);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = (k * G + l) * 4, cnt = min(4, g.C - c);
      if (cnt <= 0) continue;
      float ga[4] = {1.f, 1.f, 1.f, 1.f}, be[4] = {};
      if (gamma) load_run<4>(gamma + c, cnt, ga);
      if (beta) load_run<4>(beta + c, cnt, be);
#pragma unroll
      for (int j = 0; j < 4; ++j) s[k][j] = fmaf(s[k][j] * rstd, ga[j], be[j]);
      store_run<4>(y + at + c, cnt, s[k]);
    }
    if (stats && l == 0) stats[row] = mean, stats[g.frames + row] = rstd;
  }
}

// More channels than registers hold: a thread per pixel (or token) that reads
// them again.
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
        if (d.rng) {
          unsigned w;
          gen.run<1>(e, &w);
          b = dropped(b, w, d);
        }
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
      if (grad_branch) {
        unsigned w = 0;
        if (d.rng) gen.run<1>(e, &w);
        grad_branch[e] = d.rng ? dropped(r, w, d) : r;
      }
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

constexpr long long kMostGroups = 1 << 21;  // a launch holds less than 2^32 threads

// Waves of a tile of V pixels a lane, R channels a wave at most.
static int tile_waves(int C, int R) { return (C + R - 1) / R; }

snls_status launch_norm(const float* x, const float* branch, const Drop& drop, const float* gamma, const float* beta,
                        const snls_norm_params& np, float* total, float* y, float* stats, hipStream_t s) {
  NormGeo g = {np.frames, np.pixels, 0, 0, np.C, 0, np.eps};
  if (np.pixels == 1 && np.C <= 2048) {
    const int per = np.C <= 128 ? 16 : 4;
    const long long groups = (np.frames + per - 1) / per;
    const dim3 grid((unsigned)std::min(groups, kMostGroups));
    if (np.C <= 64)
      hipLaunchKernelGGL((norm_token_kernel<16, 1>), grid, dim3(256), 0, s, x, branch, drop, gamma, beta, g, total, y, stats);
    else if (np.C <= 128)
      hipLaunchKernelGGL((norm_token_kernel<16, 2>), grid, dim3(256), 0, s, x, branch, drop, gamma, beta, g, total, y, stats);
    else if (np.C <= 256)
      hipLaunchKernelGGL((norm_token_kernel<64, 1>), grid, dim3(256), 0, s, x, branch, drop, gamma, beta, g, total, y, stats);
    else if (np.C <= 1024)
      hipLaunchKernelGGL((norm_token_kernel<64, 4>), grid, dim3(256), 0, s, x, branch, drop, gamma, beta, g, total, y, stats);
    else
      hipLaunchKernelGGL((norm_token_kernel<64, 8>), grid, dim3(256), 0, s, x, branch, drop, gamma, beta, g, total, y, stats);
  } else if (np.pixels > 1 && np.C <= 512) {
    const bool wide = np.C <= 256 && np.frames * ((np.pixels + 255) / 256) >= 1024;
    const int V = wide ? 4 : 1, waves = wide ? tile_waves(np.C, 16) : std::min(16, tile_waves(np.C, 4));
    g.n = (np.C + waves - 1) / waves;
    g.per_frame = (np.pixels + 64 * V - 1) / (64 * V), g.tiles = g.per_frame * np.frames;
    const dim3 grid((unsigned)std::min(g.tiles, kMostGroups)), block(64 * waves);
    const size_t lds = waves > 1 ? 2 * waves * V * 64 * sizeof(float) : 0;
    if (wide)
      hipLaunchKernelGGL((norm_tile_kernel<4, 16>), grid, block, lds, s, x, branch, drop, gamma, beta, g, total, y, stats);
    else if (np.C <= 256)
      hipLaunchKernelGGL((norm_tile_kernel<1, 16>), grid, block, lds, s, x, branch, drop, gamma, beta, g, total, y, stats);
    else
      hipLaunchKernelGGL((norm_tile_kernel<1, 32>), grid, block, lds, s, x, branch, drop, gamma, beta, g, total, y, stats);
  } else {
    hipLaunchKernelGGL(norm_kernel, dim3(pixel_groups(np)), dim3(256), 0, s, x, branch, drop, gamma, beta, np.frames,
                       np.C, np.pixels, np.eps, total, y, stats);
  }
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
