// rotate.hip -- rotary positions over time, rows and columns (snls_rotate,
// snls_rotate_points).
#include "snls_internal.h"

namespace snls {

// cos and sin of pos * turns turns.  The angle is formed and reduced to the
// nearest quarter turn in 64 bits, so that what is rounded to fp32 is at most
// an eighth of a turn: 2.3e-8 radians, however far the position.
SNLS_DEV void phase(double pos, double turns, float* c, float* s) {
  const double r = pos * turns * 4.0;
  const double q = rint(r);
  float sn, cs;
  sincospif(0.5f * (float)(r - q), &sn, &cs);
  const int k = (int)(q - 4.0 * floor(q * 0.25));
  const float a = (k & 1) ? sn : cs, b = (k & 1) ? cs : sn;
  *c = (k == 1 || k == 2) ? -a : a;
  *s = k >= 2 ? -b : b;
}

// Axis, channels within the head and index of pair p.
struct Pair {
  int axis, first, second;
};
SNLS_DEV Pair pair_of(int p, const Rotary& r) {
  int axis = 0, at = 0;
  if (p >= r.pairs[0]) p -= r.pairs[0], at += 2 * r.pairs[0], axis = 1;
  if (axis == 1 && p >= r.pairs[1]) p -= r.pairs[1], at += 2 * r.pairs[1], axis = 2;
  const int n = axis == 0 ? r.pairs[0] : axis == 1 ? r.pairs[1] : r.pairs[2];
  return r.interleaved ? Pair{axis, at + 2 * p, at + 2 * p + 1} : Pair{axis, at + p, at + n + p};
}

// A thread per pixel of a pair's two planes; behind the pairs, per pixel of the
// planes that are copied.
__global__ void __launch_bounds__(256) rotate_kernel(const float* x, const int64_t* __restrict__ times, Rotary r,
                                                     long long groups, float* out) {
  const int units = r.total + (r.Ch - 2 * r.total);
  const long long HW = (long long)r.H * r.W;
  const long long work = (long long)r.B * r.T * r.HD * units * groups;
  for (long long g = blockIdx.x; g < work; g += gridDim.x) {
    const long long i = g % groups * 256 + threadIdx.x;
    if (i >= HW) continue;
    const long long u = g / groups;
    const int p = (int)(u % units);
    const long long head = u / units;
    const float* src = x + head * r.Ch * HW + i;
    float* dst = out + head * r.Ch * HW + i;
    if (p >= r.total) {
      const long long c = r.total + p;
      dst[c * HW] = src[c * HW];
      continue;
    }
    const Pair pr = pair_of(p, r);
    const long long bt = head / r.HD;
    const double pos = pr.axis == 0   ? (times ? (double)times[bt] : (double)(bt % r.T))
                       : pr.axis == 1 ? (double)r.row0 + (double)(i / r.W)
                                      : (double)r.col0 + (double)(i % r.W);
    float c, s;
    phase(pos, r.turns[p], &c, &s);
    const float a = src[pr.first * HW], b = src[pr.second * HW];
    dst[pr.first * HW] = fmaf(a, c, -(b * s));
    dst[pr.second * HW] = fmaf(a, s, b * c);
  }
}

// A thread per pair, or channel behind the pairs, of a token's head.
__global__ void __launch_bounds__(256) rotate_points_kernel(const float* q, const int32_t* __restrict__ points,
                                                            long long n, const int64_t* __restrict__ times, Rotary r,
                                                            float* out) {
  const int units = r.total + (r.Ch - 2 * r.total), per = r.HD * units;
  for (long long w = blockIdx.x * 256LL + threadIdx.x; w < n * per; w += gridDim.x * 256LL) {
    const long long token = w / per;
    const int rest = (int)(w - token * per), hd = rest / units, p = rest - hd * units;
    const int b = points[3 * token], h = points[3 * token + 1], x = points[3 * token + 2];
    const bool in = b >= 0 && b < r.B && h >= 0 && h < r.H && x >= 0 && x < r.W;
    const float* src = q + token * r.C + hd * r.Ch;
    float* dst = out + token * r.C + hd * r.Ch;
    if (p >= r.total) {
      const int c = r.total + p;
      dst[c] = in ? src[c] : 0.f;
      continue;
    }
    const Pair pr = pair_of(p, r);
    if (!in) {
      dst[pr.first] = dst[pr.second] = 0.f;
      continue;
    }
    const double pos = pr.axis == 0   ? (times ? (double)times[b] : 0.0)
                       : pr.axis == 1 ? (double)r.row0 + (double)h
                                      : (double)r.col0 + (double)x;
    float c, s;
    phase(pos, r.turns[p], &c, &s);
    const float a = src[pr.first], e = src[pr.second];
    dst[pr.first] = fmaf(a, c, -(e * s));
    dst[pr.second] = fmaf(a, s, e * c);
  }
}

snls_status launch_rotate(const float* q, const float* k, const int64_t* times, const Rotary& r, float* q_out,
                          float* k_out, hipStream_t s) {
  const long long groups = ((long long)r.H * r.W + 255) / 256;
  const long long work = (long long)r.B * r.T * r.HD * (r.Ch - r.total) * groups;
  const dim3 grid((unsigned)(work < (1 << 20) ? work : (1 << 20)));
  hipLaunchKernelGGL(rotate_kernel, grid, dim3(256), 0, s, q, times, r, groups, q_out);
  if (k) hipLaunchKernelGGL(rotate_kernel, grid, dim3(256), 0, s, k, times, r, groups, k_out);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

snls_status launch_rotate_points(const float* q, const int32_t* points, long long n, const int64_t* times,
                                 const Rotary& r, float* out, hipStream_t s) {
  const long long groups = (n * r.HD * (r.Ch - r.total) + 255) / 256;
  hipLaunchKernelGGL(rotate_points_kernel, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(256), 0, s, q,
                     points, n, times, r, out);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
