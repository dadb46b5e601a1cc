// project.hip -- projections in 8-bit integers: tokens quantised on the way, a
// scale per token and per output channel (snls_project, snls_project_pack).
#include "snls_internal.h"

namespace snls {

// Magnitudes as bits: ordered like the numbers, infinities and NaN above all.
SNLS_DEV unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr unsigned kInfBits = 0x7f800000u;

// Scale of the codes of values up to the magnitude `most` (NaN where that is
// not finite) and their rounding.  A code is the whole number nearest to the
// exact quotient x / s, ties to even: the product with the rounded reciprocal
// is off by at most 127 * 2^-23, so the number it rounds to is off by at most
// one, and x - code * s, which a fused multiply-add gives exactly where it
// counts, says in which direction.
struct Quant {
  float s, inv, half;
  SNLS_DEV explicit Quant(unsigned most) {
    s = most < kInfBits ? fmaxf(__uint_as_float(most), 0x1p-100f) / 127.f : NAN;
    inv = 1.f / s, half = 0.5f * s;
  }
  SNLS_DEV int code(float x) const {
    float c = rintf(x * inv);
    const float r = fmaf(-c, s, x), m = fabsf(r);
    const bool odd = (int)c & 1;
    if (m > half || (m == half && odd)) c += copysignf(1.f, r);
    return (int)c;
  }
};

// 64 pixels (or tokens) a workgroup: a thread quantises one into LDS and sums
// its products.
__global__ void __launch_bounds__(64) project_kernel(const float* __restrict__ x, const int8_t* __restrict__ w,
                                                     const float* __restrict__ scales, const float* __restrict__ bias,
                                                     snls_project_params p, float* __restrict__ out) {
  extern __shared__ int8_t codes[];
  const long long P = p.pixels, px = p.frames * P;
  const int per = p.cout / p.parts;
  for (long long i0 = blockIdx.x * 64LL; i0 < px; i0 += gridDim.x * 64LL) {
    const long long i = i0 + threadIdx.x;
    if (i >= px) continue;
    const long long f = i / P, at = f * p.cin * P + (i - f * P);
    unsigned most = 0;
    for (int c = 0; c < p.cin; ++c) most = max(most, magnitude(x[at + c * P]));
    const Quant q(most);
    const bool ok = most < kInfBits;
    for (int c = 0; c < p.cin; ++c) codes[c * 64 + threadIdx.x] = ok ? (int8_t)q.code(x[at + c * P]) : 0;
    for (int o = 0; o < p.cout; ++o) {
      int acc = 0;
      for (int c = 0; c < p.cin; ++c) acc += (int)codes[c * 64 + threadIdx.x] * (int)w[(long long)o * p.cin + c];
      const int part = o / per;
      const long long to = (((long long)part * p.frames + f) * per + (o - part * per)) * P + (i - f * P);
      out[to] = fmaf((float)acc * q.s, scales[o], bias ? bias[o] : 0.f);
    }
  }
}

// A wave per output channel.
__global__ void __launch_bounds__(64) project_pack_kernel(const float* __restrict__ w, int cin,
                                                          int8_t* __restrict__ codes, float* __restrict__ scales) {
  const long long at = (long long)blockIdx.x * cin;
  unsigned most = 0;
  for (int c = threadIdx.x; c < cin; c += 64) most = max(most, magnitude(w[at + c]));
  for (int m = 32; m > 0; m /= 2) most = max(most, (unsigned)__shfl_xor((int)most, m));
  const Quant q(most);
  const bool ok = most < kInfBits;
  for (int c = threadIdx.x; c < cin; c += 64) codes[at + c] = ok ? (int8_t)q.code(w[at + c]) : 0;
  if (threadIdx.x == 0) scales[blockIdx.x] = q.s;
}

snls_status launch_project_pack(const float* w, int cin, int cout, int8_t* codes, float* scales, hipStream_t s) {
  hipLaunchKernelGGL(project_pack_kernel, dim3((unsigned)cout), dim3(64), 0, s, w, cin, codes, scales);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

snls_status launch_project(const float* x, const int8_t* codes, const float* scales, const float* bias,
                           const snls_project_params& pp, float* out, hipStream_t s) {
  const long long groups = (pp.frames * pp.pixels + 63) / 64;
  hipLaunchKernelGGL(project_kernel, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(64), 64 * pp.cin, s, x,
                     codes, scales, bias, pp, out);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
