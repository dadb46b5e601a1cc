// bias.hip -- learned bias of the neighbours' relative position: added to the
// scores (snls_bias), and the gradient of its table (snls_bias_backward).
//
// A neighbour's entry is table[hd, step, bucket(dh), bucket(dw)].  Both
// directions read 16 or 20 bytes a neighbour and write 4 or (almost) nothing,
// so memory bandwidth bounds them.
#include "position_bias.h"

namespace snls {

// Scores of one image (one head of one query frame: nH * nW * k of them lie
// together, with one frame index and one table) per group of workgroups.
struct BiasRows {
  long long per_image;  // scores of an image
  int T, HD;
};

static BiasRows bias_rows(const Geo& g) {
  return {(long long)g.nH * g.nW * (g.k > 0 ? g.k : g.ncand), g.T, g.HD};
}

// Flat bucket of a neighbour of query frame t, or -1 when it contributes
// nothing to the aggregation.
SNLS_DEV int neighbour_bucket(float frame, float dh, float dw, int t, int T, const Bias& b) {
  const bool ok = frame >= 0.f && frame < (float)T && frame == floorf(frame) && fabsf(dh) < kFarDisp &&
                  fabsf(dw) < kFarDisp;
  if (!ok) return -1;
  return (bias_step_bucket((int)frame - t, b) * b.nb + bias_bucket(dh, b)) * b.nb + bias_bucket(dw, b);
}

__global__ void __launch_bounds__(256) bias_kernel(const float* dists, const float* __restrict__ inds,
                                                   const float* __restrict__ table, BiasRows r, Bias b, float sign,
                                                   unsigned chunks, float* out) {
  extern __shared__ float tab[];
  const long long img = blockIdx.x / chunks;
  const unsigned chunk = blockIdx.x % chunks;
  const int t = (int)(img % r.T), hd = (int)(img / r.T % r.HD);
  for (int i = threadIdx.x; i < b.buckets; i += 256) tab[i] = sign * table[(long long)hd * b.buckets + i];
  __syncthreads();
  const long long base = img * r.per_image;
  for (long long i = (long long)chunk * 256 + threadIdx.x; i < r.per_image; i += (long long)chunks * 256) {
    const long long n = base + i;
    const float d = dists[n];
    const int at = neighbour_bucket(inds[3 * n], inds[3 * n + 1], inds[3 * n + 2], t, r.T, b);
    out[n] = isfinite(d) && at >= 0 ? d + tab[at] : d;
  }
}

// One wave per slice of a head's scores.  The table of partial sums lies in
// LDS, `cols` copies of every entry; lane i adds to copy i % cols, cols lanes
// at a time, so that no two lanes of one step meet and the order of every
// entry's additions is fixed.
__global__ void __launch_bounds__(64) bias_grad_kernel(const float* __restrict__ grad, const float* __restrict__ dists,
                                                       const float* __restrict__ inds, BiasRows r, Bias b, int B,
                                                       float sign, int cols, int slices, float* __restrict__ part) {
  extern __shared__ float acc[];
  const int lane = threadIdx.x;
  const int hd = blockIdx.x / slices, slice = blockIdx.x % slices;
  for (int i = lane; i < b.buckets * cols; i += 64) acc[i] = 0.f;
  wave_lds_sync();
  const long long total = (long long)B * r.T * r.per_image;  // of this head
  const long long per = ((total + slices - 1) / slices + 63) / 64 * 64;
  const long long u1 = min(total, (slice + 1) * per);
  const int mycol = lane & (cols - 1), turn = lane / cols;
  for (long long u0 = slice * per; u0 < u1; u0 += 64) {
    const long long u = u0 + lane;
    int at = -1;
    float gv = 0.f;
    if (u < u1) {
      const long long bt = u / r.per_image, i = u - bt * r.per_image;
      const int t = (int)(bt % r.T);
      const long long n = ((bt / r.T * r.HD + hd) * r.T + t) * r.per_image + i;
      gv = sign * grad[n];
      if (isfinite(dists[n])) at = neighbour_bucket(inds[3 * n], inds[3 * n + 1], inds[3 * n + 2], t, r.T, b);
    }
    for (int k = 0; k < 64 / cols; ++k) {
      if (turn == k && at >= 0) acc[at * cols + mycol] += gv;
      wave_lds_sync();
    }
  }
  for (int i = lane; i < b.buckets; i += 64) {
    float s = 0.f;
    for (int c = 0; c < cols; ++c) s += acc[i * cols + c];
    part[(long long)blockIdx.x * b.buckets + i] = s;
  }
}

// grad_table[hd][i] = sum of the head's slices, in 64 bits.
__global__ void __launch_bounds__(256) bias_grad_sum_kernel(const float* __restrict__ part, int buckets, int slices,
                                                            float* __restrict__ grad_table) {
  const int hd = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  if (i >= buckets) return;
  double s = 0.0;
  for (int k = 0; k < slices; ++k) s += part[((long long)hd * slices + k) * buckets + i];
  grad_table[(long long)hd * buckets + i] = (float)s;
}

constexpr int kBiasSlices = 1280;  // one wave each: 5 on every CU

static int bias_slices(const Geo& g) {
  const long long total = (long long)g.B * g.T * bias_rows(g).per_image;
  const long long want = (total + 255) / 256;
  const long long most = kBiasSlices / g.HD > 1 ? kBiasSlices / g.HD : 1;
  return (int)(want < most ? want : most);
}

size_t bias_backward_ws_bytes(const Geo& g) {
  return (size_t)g.HD * bias_slices(g) * SNLS_BIAS_MAX_BUCKETS * sizeof(float);
}

snls_status launch_bias(const float* dists, const float* inds, const float* table, const Geo& g, const Bias& bias,
                        float* out, hipStream_t s) {
  const BiasRows r = bias_rows(g);
  const long long images = (long long)g.B * g.HD * g.T;
  long long chunks = (r.per_image + 1023) / 1024;
  const long long most = images < 8192 ? 8192 / images : 1;
  if (chunks > most) chunks = most;
  if (images * chunks > 0x7fffffffLL) return SNLS_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(bias_kernel, dim3((unsigned)(images * chunks)), dim3(256), bias.buckets * sizeof(float), s, dists,
                     inds, table, r, bias, g.dist == SNLS_DIST_PROD ? 1.f : -1.f, (unsigned)chunks, out);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

snls_status launch_bias_backward(const float* grad, const float* dists, const float* inds, const Geo& g,
                                 const Bias& bias, float* grad_table, float* ws, hipStream_t s) {
  const int slices = bias_slices(g);
  int cols = 16;
  while (cols > 1 && bias.buckets * cols > 8192) cols /= 2;  // at most 32 KB
  hipLaunchKernelGGL(bias_grad_kernel, dim3((unsigned)(g.HD * slices)), dim3(64),
                     (size_t)bias.buckets * cols * sizeof(float), s, grad, dists, inds, bias_rows(g), bias, g.B,
                     g.dist == SNLS_DIST_PROD ? 1.f : -1.f, cols, slices, ws);
  hipLaunchKernelGGL(bias_grad_sum_kernel, dim3((unsigned)((bias.buckets + 255) / 256), (unsigned)g.HD), dim3(256), 0,
                     s, ws, bias.buckets, slices, grad_table);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
