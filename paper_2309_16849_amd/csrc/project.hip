// project.hip -- projections in 8-bit integers: tokens quantised on the way, a
// scale per token and per output channel (snls_project, snls_project_pack).
#include "snls_internal.h"

namespace snls {

// Magnitudes as bits: ordered like the numbers, infinities and NaN above all.
SNLS_DEV unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr unsigned kInfBits = 0x7f800000u;

// Scale of the codes of values up to the magnitude `most` (NaN where that is
// not finite) and their rounding: a code is the whole number nearest to the
// exact quotient x / s, ties to even.  The sum of x * inv and 1.5 * 2^23, in one
// rounding, has the nearest whole number to that product in its last bits; inv
// is a rounded reciprocal, so it is the quotient's too unless the quotient lies
// within 127 * 2^-24 of a half.  The remainder x - code * s, exact where it
// counts, tells: beyond 0.49999 s, one value in 50,000, the code is settled by
// comparing it with half a step.
struct Quant {
  float s, inv, near, half;
  SNLS_DEV explicit Quant(unsigned most) {
    s = most < kInfBits ? fmaxf(__uint_as_float(most), 0x1p-100f) / 127.f : NAN;
    inv = 1.f / s, near = 0.49999f * s, half = 0.5f * s;
  }
  static constexpr float kMagic = 12582912.f;
  SNLS_DEV float settle(float f, float x) const {
    const float r = fmaf(-(f - kMagic), s, x), m = fabsf(r);
    return m > half || (m == half && (__float_as_uint(f) & 1)) ? f + copysignf(1.f, r) : f;
  }
  SNLS_DEV int code(float x) const {  // of one value
    return (int)(settle(fmaf(x, inv, kMagic), x) - kMagic);
  }
  // Codes of 16 values, four a register.
  template <class Codes>
  SNLS_DEV void codes16(const float* x, Codes& out) const {
    float f[16], far = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      f[j] = fmaf(x[j], inv, kMagic);
      far = fmaxf(far, fabsf(fmaf(-(f[j] - kMagic), s, x[j])));
    }
    if (far > near)
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] = settle(f[j], x[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned a = __builtin_amdgcn_perm(__float_as_uint(f[4 * j + 1]), __float_as_uint(f[4 * j]), 0x0c0c0400u);
      const unsigned b = __builtin_amdgcn_perm(__float_as_uint(f[4 * j + 3]), __float_as_uint(f[4 * j + 2]), 0x04000c0cu);
      out[j] = (int)(a | b);
    }
  }
};

typedef int Int4 __attribute__((ext_vector_type(4)));
typedef int Int16 __attribute__((ext_vector_type(16)));

// A call's sizes on the device.  span: tiles of 32 output channels a workgroup
// takes; hold: of these, how many lie in LDS at a time.
struct ProjectGeo {
  long long px, P, groups;  // pixels in all, of a frame; groups of 128 of them
  long long F;              // frames
  int cin, cout, per;       // per: output channels of a part
  int span, hold;
};

// What the epilogue needs of an output channel: where its plane starts (a
// token's: its place in the row), scale and bias.
struct OutChannel {
  long long at;
  float scale, bias;
};

// 16 consecutive weights of a channel as a lane of the matrix instruction takes
// them; 0 behind the last channel of either side.
SNLS_DEV Int4 weights16(const int8_t* __restrict__ w, int o, int c, const ProjectGeo& g) {
  Int4 v = {0, 0, 0, 0};
  if (o >= g.cout || c >= g.cin) return v;
  const int8_t* from = w + (long long)o * g.cin + c;
  if (c + 16 <= g.cin && !((uintptr_t)from & 15)) return *reinterpret_cast<const Int4*>(from);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const unsigned b = c + i < g.cin ? (unsigned)(uint8_t)from[i] : 0u;
    v[i / 4] = (int)((unsigned)v[i / 4] | b << (8 * (i % 4)));
  }
  return v;
}

// The product on the matrix cores, 32 x 32 outputs an instruction over 32
// channels: the weights' tile is one operand, the codes of 32 pixels the other.
// Both give a lane 16 consecutive channels of one row (lane mod 32; the upper
// lanes have the upper 16), so a lane loads its pixel's channels, finds the
// largest with its partner and packs the codes where the instruction wants them:
// they never leave the registers.  The weights lie in LDS in the order of the
// lanes.  NK: steps of 32 channels.  TOK: a list of tokens (pixels == 1), whose
// rows and columns change places so that stores run along the output channels.
// Up to KEEP steps, the values stay in registers between the maximum and the
// codes; beyond, they are read again.
template <int NK, bool TOK>
__global__ void __launch_bounds__(256) project_kernel(const float* __restrict__ x, const int8_t* __restrict__ w,
                                                      const float* __restrict__ scales,
                                                      const float* __restrict__ bias, ProjectGeo g,
                                                      float* __restrict__ out) {
  extern __shared__ char lds[];
  constexpr bool KEEP = NK <= 8;
  Int4* const wt = reinterpret_cast<Int4*>(lds);
  OutChannel* const chan = reinterpret_cast<OutChannel*>(lds + g.hold * NK * 1024);
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5, wv = threadIdx.x >> 6;
  const int tiles = (g.cout + 31) / 32, t0 = blockIdx.y * g.span, t1 = min(t0 + g.span, tiles);
  const bool once = t1 - t0 <= g.hold;

  // tiles [from, to) into LDS
  auto stage = [&](int from, int to) {
    const int n = (to - from) * NK * 64;
    for (int i = threadIdx.x; i < n; i += 256) {
      const int l = i & 63, ks = (i >> 6) % NK, t = from + (i >> 6) / NK;
      wt[i] = weights16(w, t * 32 + (l & 31), ks * 32 + (l >> 5) * 16, g);
    }
    for (int i = threadIdx.x; i < (to - from) * 32; i += 256) {
      const int o = from * 32 + i;
      if (o < g.cout) {
        const int part = o / g.per;
        chan[i] = TOK ? OutChannel{(long long)part * g.F * g.per + (o - part * g.per), scales[o], bias ? bias[o] : 0.f}
                      : OutChannel{(o + part * (g.F - 1) * g.per) * g.P, scales[o], bias ? bias[o] : 0.f};
      }
    }
  };

  bool staged = false;
  for (long long grp = blockIdx.x; grp < g.groups; grp += gridDim.x) {
    const long long i0 = grp * 128 + wv * 32;
    const bool any = i0 < g.px;  // of this wave
    const bool mine = i0 + col < g.px;
    const long long f0 = TOK || !any ? i0 : i0 / g.P;
    const unsigned rel = TOK || !any ? 0 : (unsigned)(i0 - f0 * g.P) + (mine ? col : 0);
    const long long f = TOK ? i0 + (mine ? col : 0) : f0 + rel / (unsigned)g.P;
    const long long p = TOK ? 0 : rel % (unsigned)g.P;
    const long long step = TOK ? 1 : g.P;
    const float* const first = x + f * g.cin * g.P + p;  // channel 0 of this lane's pixel
    int upper = half * 16;
    asm volatile("" : "+v"(upper));  // (else every guard below is held in registers across the groups)
    // this lane's 16 channels of step ks
    auto load16 = [&](int ks, float* v) {
      const int c = ks * 32 + upper;
      if (ks * 32 + 32 <= g.cin) {
        const float* from = first + c * step;
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = from[j * step];
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float u = first[min(c + j, g.cin - 1) * step];
          v[j] = c + j < g.cin ? u : 0.f;
        }
      }
    };
    float v[KEEP ? NK * 16 : 64];
    if (KEEP && any)
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) load16(ks, v + ks * 16);
    // (the weights' way to LDS goes by while the values come in)
    const bool now = once && !staged;
    if (now) stage(t0, t1);
    Int4 codes[NK];
    float ts = 0.f;
    if (any) {
      unsigned most = 0;
      if constexpr (KEEP) {
#pragma unroll
        for (int j = 0; j < NK * 16; ++j) most = max(most, magnitude(v[j]));
      } else {
#pragma unroll 1
        for (int ks = 0; ks < NK; ks += 4) {
#pragma unroll
          for (int b = 0; b < 4; ++b) load16(ks + b, v + b * 16);
#pragma unroll
          for (int j = 0; j < 64; ++j) most = max(most, magnitude(v[j]));
        }
      }
      most = max(most, (unsigned)__shfl_xor((int)most, 32));
      const bool ok = most < kInfBits;
      const Quant q(most);
      ts = q.s;
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        if constexpr (!KEEP)
          if (ks % 4 == 0) {
            __builtin_amdgcn_sched_barrier(0);  // four steps' values at a time: all at once do not fit
#pragma unroll
            for (int b = 0; b < 4; ++b) load16(ks + b, v + b * 16);
          }
        q.codes16(v + (KEEP ? ks : ks % 4) * 16, codes[ks]);
        if (!ok) codes[ks] = Int4{0, 0, 0, 0};
      }
    }
    if (now) __syncthreads();
    staged = true;
    for (int from = t0; from < t1; from += g.hold) {
      const int to = min(from + g.hold, t1);
      if (!once) {
        __syncthreads();
        stage(from, to);
        __syncthreads();
      }
      if (!any) continue;
      for (int t = from; t < to; ++t) {
        Int16 acc = {};
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
          const Int4 a = wt[((t - from) * NK + ks) * 64 + lane];
          acc = TOK ? __builtin_amdgcn_mfma_i32_32x32x32_i8(codes[ks], a, acc, 0, 0, 0)
                    : __builtin_amdgcn_mfma_i32_32x32x32_i8(a, codes[ks], acc, 0, 0, 0);
        }
        // register r: row 8 * (r / 4) + 4 * half + r % 4, column lane mod 32
        if constexpr (TOK) {
          const OutChannel ch = chan[(t - from) * 32 + col];
          float* const to_row = out + ch.at + (i0 + 4 * half) * g.per;
          const int rows = t * 32 + col < g.cout ? (int)min(32LL, g.px - i0) - 4 * half : 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r / 4) + r % 4;
            const float s = __shfl(ts, row + 4 * half);
            if (row < rows)
              __builtin_nontemporal_store(fmaf((float)acc[r] * s, ch.scale, ch.bias), to_row + (long long)row * g.per);
          }
        } else {
          float* const to_px = out + f * g.per * g.P + p;
          const OutChannel* const ch = chan + (t - from) * 32 + 4 * half;
          const int rows = mine ? g.cout - t * 32 - 4 * half : 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r / 4) + r % 4;
            const OutChannel c = ch[row];
            if (row < rows) __builtin_nontemporal_store(fmaf((float)acc[r] * ts, c.scale, c.bias), to_px + c.at);
          }
        }
      }
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

template <int NK>
static void run_project(const float* x, const int8_t* codes, const float* scales, const float* bias,
                        const ProjectGeo& g, bool tokens, dim3 grid, float* out, hipStream_t s) {
  const size_t lds = (size_t)g.hold * (NK * 1024 + 32 * sizeof(OutChannel));
  if (tokens)
    hipLaunchKernelGGL((project_kernel<NK, true>), grid, dim3(256), lds, s, x, codes, scales, bias, g, out);
  else
    hipLaunchKernelGGL((project_kernel<NK, false>), grid, dim3(256), lds, s, x, codes, scales, bias, g, out);
}

snls_status launch_project(const float* x, const int8_t* codes, const float* scales, const float* bias,
                           const snls_project_params& pp, float* out, hipStream_t s) {
  const int steps = (pp.cin + 31) / 32;
  const int nk = steps <= 4 ? steps : steps <= 6 ? 6 : steps <= 8 ? 8 : steps <= 12 ? 12 : steps <= 16 ? 16 : 32;
  ProjectGeo g;
  g.px = pp.frames * pp.pixels, g.P = pp.pixels, g.F = pp.frames;
  g.groups = (g.px + 127) / 128;
  g.cin = pp.cin, g.cout = pp.cout, g.per = pp.cout / pp.parts;
  const int tiles = (pp.cout + 31) / 32;
  // few pixels: the output channels are shared out too, until the chip has two workgroups a CU
  const long long want = (512 + g.groups - 1) / g.groups;
  const int split = (int)(want < tiles ? want : tiles);
  g.span = (tiles + split - 1) / split;
  const int fit = 60 / nk;  // 60 KB of weights
  g.hold = g.span < fit ? g.span : fit;
  const dim3 grid((unsigned)(g.groups < 1280 ? g.groups : 1280), (unsigned)((tiles + g.span - 1) / g.span));
  const bool tokens = pp.pixels == 1;
  switch (nk) {
    case 1: run_project<1>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    case 2: run_project<2>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    case 3: run_project<3>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    case 4: run_project<4>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    case 6: run_project<6>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    case 8: run_project<8>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    case 12: run_project<12>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    case 16: run_project<16>(x, codes, scales, bias, g, tokens, grid, out, s); break;
    default: run_project<32>(x, codes, scales, bias, g, tokens, grid, out, s); break;
  }
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
