// project.hip -- projections in 8-bit integers: tokens quantised on the way, a
// scale per token and per output channel (snls_project, snls_project_pack).
#include <algorithm>
#include <type_traits>

#include "lanes.h"

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
      unsigned u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(f[4 * j + i]);
      out[j] = (int)(__builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u) | __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu));
    }
  }
};

typedef int Int4 __attribute__((ext_vector_type(4)));
typedef int Int16 __attribute__((ext_vector_type(16)));

// A call's sizes on the device.  A group is 128 pixels of one frame (or 128
// tokens), so that a wave's loads and stores have one base and 32-bit offsets.
struct ProjectGeo {
  long long P, groups, per_frame;  // pixels of a frame; groups in all, of a frame
  long long F;                     // frames
  int cin, cout, per;              // per: output channels of a part
  int run;                         // runs of 32 pixels a workgroup takes (project_run_kernel)
  int span, hold, buffers;         // tiles of 32 output channels a workgroup takes, that lie in LDS at a time, in one
                                   // buffer (all of them) or two
  bool aligned;                    // rows of weights at 16 bytes
};

// Forms of a call.  Whole: every plane of the output starts a cache line, which
// a wave's stores fill.  Odd: they do not.  Tokens: a list of them (pixels == 1).
enum class Form { Whole, Odd, Tokens };

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
// lanes.  NK: steps of 32 channels.  A list of tokens has rows and columns in each
// other's place, so that stores run along the output channels.
// 4 bytes an input and an output channel a pixel: up to some hundred channels
// bandwidth bounds it (24 -> 48 at 9x396x392 73 us, 5.5 TB/s), beyond the values'
// second read and the weights' way into LDS (512 -> 512 at 2x128x128 60 us, 284
// TOP/s).  Up to KEEP steps, the values stay in registers between the maximum and
// the codes; beyond, they are read again, four steps at a time.
template <int NK, Form FORM>
__global__ void __launch_bounds__(256, 2) project_kernel(const float* __restrict__ x, const int8_t* __restrict__ w,
                                                         const float* __restrict__ scales,
                                                         const float* __restrict__ bias, ProjectGeo g,
                                                         float* __restrict__ out) {
  extern __shared__ char lds[];
  constexpr bool KEEP = NK <= 6, TOK = FORM == Form::Tokens;
  constexpr int STEPS = KEEP ? NK : 4;  // whose values are held at a time
  Int4* const wt = reinterpret_cast<Int4*>(lds);
  // a tile's scales, its biases, and where its channels' planes start in a frame 0
  float* const sb = reinterpret_cast<float*>(lds + g.buffers * g.hold * NK * 1024);
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = (g.cout + 31) / 32, t0 = blockIdx.y * g.span, t1 = min(t0 + g.span, tiles);
  const bool once = t1 - t0 <= g.hold;

  // Tiles [from, to) into buffer b; aligned rows without a detour over registers
  // (past the last row and channel others are read: those sums are not stored,
  // and those codes are 0).
  auto stage = [&](int from, int to, int b) {
    Int4* const wb = wt + b * g.hold * NK * 64;
    float* const tb = sb + b * g.hold * 128;
    if (g.aligned) {
      for (int n = wv; n < (to - from) * NK; n += 4) {
        const int o = min((from + n / NK) * 32 + col, g.cout - 1), c = min(n % NK * 32 + half * 16, g.cin - 16);
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void*)(w + (long long)o * g.cin + c),
            (__attribute__((address_space(3))) void*)(wb + n * 64), 16, 0, 0);
      }
    } else {
      for (int i = threadIdx.x; i < (to - from) * NK * 64; i += 256) {
        const int l = i & 63, ks = (i >> 6) % NK, t = from + (i >> 6) / NK;
        wb[i] = weights16(w, t * 32 + (l & 31), ks * 32 + (l >> 5) * 16, g);
      }
    }
    for (int i = threadIdx.x; i < (to - from) * 32; i += 256) {
      const int o = min(from * 32 + i, g.cout - 1);
      float* const to = tb + (i >> 5) * 128 + (i & 31);
      to[0] = scales[o], to[32] = bias ? bias[o] : 0.f;
      const long long part = o / g.per;
      reinterpret_cast<long long*>(tb + (i >> 5) * 128 + 64)[i & 31] = (part * (g.F - 1) * g.per + o) * (TOK ? 1 : g.P);
    }
  };
  // what this wave has on the way to LDS is there, and then everyone's
  auto all_staged = [] {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  bool staged = false;
  const Walk way = walk<FORM == Form::Odd>(g.groups);
  for (long long grp = way.first; grp < way.end; grp += way.step) {
    const long long f = TOK ? 0 : grp / g.per_frame;
    const long long p0 = (TOK ? grp : grp - f * g.per_frame) * 128 + wv * 32;  // this wave's first pixel or token
    const int have = (int)max(0LL, min(32LL, (TOK ? g.F : g.P) - p0));         // of its 32
    const bool any = have > 0;
    const int mine = min(col, have - 1);
    const float* const base = TOK ? x + p0 * g.cin : x + f * g.cin * g.P + p0;
    long long step = TOK ? 1 : g.P;  // from channel to channel
    unsigned at = (TOK ? mine * g.cin + half * 16 : (unsigned)(half * 16 * g.P) + mine) * 4u;
    int upper = half * 16;
    // (else every channel's offset and guard is held in registers across the groups)
    asm volatile("" : "+v"(upper), "+v"(at));
    if constexpr (!TOK) asm volatile("" : "+s"(step));
    // this lane's 16 channels of step ks
    auto load16 = [&](int ks, float* v) {
      if (ks * 32 + 32 <= g.cin) {
        const float* from = base + ks * 32 * step;
        if constexpr (TOK) {
#pragma unroll
          for (int j = 0; j < 16; j += 4)
            load_run<4>(reinterpret_cast<const float*>(reinterpret_cast<const char*>(from + j) + at), 4, v + j);
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j, from += step) v[j] = load_at(from, at);
        }
      } else {
        const float* from = base + ks * 32 * step;
        const int left = g.cin - ks * 32 - upper;
#pragma unroll
        for (int j = 0; j < 16; ++j, from += step) {
          v[j] = 0.f;
          if (j < left) v[j] = load_at(from, at);
        }
      }
    };
    float v[STEPS * 16];
    if (KEEP && any)
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) load16(ks, v + ks * 16);
    // (the weights' way to LDS goes by while the values come in)
    const bool now = once && !staged;
    if (now) stage(t0, t1, 0);
    Int4 codes[NK];
    float ts = 0.f;
    if (any) {
      unsigned most = 0;
      if constexpr (KEEP) {
#pragma unroll
        for (int j = 0; j < NK * 16; ++j) most = max(most, magnitude(v[j]));
      } else {
#pragma unroll 1
        for (int ks = 0; ks < NK; ks += STEPS) {
#pragma unroll
          for (int b = 0; b < STEPS; ++b) load16(ks + b, v + b * 16);
#pragma unroll
          for (int j = 0; j < STEPS * 16; ++j) most = max(most, magnitude(v[j]));
        }
      }
      most = max(most, (unsigned)__shfl_xor((int)most, 32));
      const bool ok = most < kInfBits;
      const Quant q(most);
      ts = q.s;
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        if constexpr (!KEEP)
          if (ks % STEPS == 0) {
            __builtin_amdgcn_sched_barrier(0);  // so many values at a time: all at once do not fit
#pragma unroll
            for (int b = 0; b < STEPS; ++b) load16(ks + b, v + b * 16);
          }
        q.codes16(v + ks % STEPS * 16, codes[ks]);
        if (!ok) codes[ks] = Int4{0, 0, 0, 0};
      }
    }
    if (now) all_staged();
    staged = true;
    int b = 0;
    if (!once) {
      __syncthreads();  // (the last group's tiles are read)
      stage(t0, min(t0 + g.hold, t1), 0);
      all_staged();
    }
    for (int from = t0; from < t1; from += g.hold, b ^= 1) {
      const int to = min(from + g.hold, t1);
      // the next tiles come in while these are used
      if (to < t1) stage(to, min(to + g.hold, t1), b ^ 1);
      for (int t = from; t < (any ? to : from); ++t) {
        const Int4* const wb = wt + (b * g.hold + t - from) * NK * 64;
        const float* const tb = sb + (b * g.hold + t - from) * 128;
        Int16 acc = {};
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
          const Int4 a = wb[ks * 64 + lane];
          acc = TOK ? __builtin_amdgcn_mfma_i32_32x32x32_i8(codes[ks], a, acc, 0, 0, 0)
                    : __builtin_amdgcn_mfma_i32_32x32x32_i8(a, codes[ks], acc, 0, 0, 0);
        }
        // register r: row 8 * (r / 4) + 4 * half + r % 4, column lane mod 32
        const int o0 = t * 32, left = g.cout - o0;
        const long long* const planes = reinterpret_cast<const long long*>(tb + 64);
        if constexpr (TOK) {
          const float sc = tb[col], be = tb[32 + col];
          float* const to_row = out + planes[col] + (p0 + 4 * half) * g.per;
          const int rows = col < left ? have - 4 * half : 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r / 4) + r % 4;
            const float s = __shfl(ts, row + 4 * half);
            if (row < rows)
              to_row[(long long)row * g.per] = fmaf((float)acc[r] * s, sc, be);
          }
        } else if (const int part = o0 / g.per; left >= 32 && have == 32 && o0 + 32 <= (part + 1) * g.per) {
          // the whole tile, in one part
          float* to_px = out + (((long long)part * g.F + f) * g.per + (o0 - part * g.per)) * step + p0;
          const unsigned lane_at = ((unsigned)(4 * half * g.P) + col) * 4u;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            float sc[4], be[4];
            load_run<4>(tb + 8 * n + 4 * half, 4, sc);
            load_run<4>(tb + 32 + 8 * n + 4 * half, 4, be);
#pragma unroll
            for (int r = 0; r < 4; ++r, to_px += step)
              store_at<FORM == Form::Whole>(to_px, lane_at, fmaf((float)acc[4 * n + r] * ts, sc[r], be[r]));
            to_px += 4 * step;
          }
        } else if (col < have) {
          float* const to_px = out + f * g.per * g.P + p0 + col;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r / 4) + 4 * half + r % 4;
            if (row < left)
              to_px[planes[row]] = fmaf((float)acc[r] * ts, tb[row], tb[32 + row]);
          }
        }
      }
      if (to < t1) all_staged();
    }
  }
}

// More channels: the four waves share a group's channels, S steps each, so that
// every value is loaded once and at once, and join the largest magnitudes and then
// the codes in LDS; each takes every fourth tile of the weights, whose rows it
// reads by itself (aligned ones), with no barrier on the way.  A group is 32 * PT
// pixels or tokens.
template <int S, int PT, Form FORM>
__global__ void __launch_bounds__(256, 2) project_wide_kernel(const float* __restrict__ x,
                                                              const int8_t* __restrict__ w,
                                                              const float* __restrict__ scales,
                                                              const float* __restrict__ bias, ProjectGeo g,
                                                              float* __restrict__ out) {
  constexpr int NK = 4 * S;
  constexpr bool TOK = FORM == Form::Tokens;
  extern __shared__ char lds[];
  Int4* const shared = reinterpret_cast<Int4*>(lds);                        // codes, in the order of the lanes
  unsigned* const top = reinterpret_cast<unsigned*>(lds + PT * NK * 1024);  // rows of magnitudes, by waves
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = (g.cout + 31) / 32, t0 = blockIdx.y * g.span, t1 = min(t0 + g.span, tiles);
  const Walk way = walk<FORM == Form::Odd>(g.groups);
  for (long long grp = way.first; grp < way.end; grp += way.step) {
    const long long f = TOK ? 0 : grp / g.per_frame;
    const long long p0 = (TOK ? grp : grp - f * g.per_frame) * (32 * PT);
    const int have = (int)min(32LL * PT, (TOK ? g.F : g.P) - p0);
    const float* const base = TOK ? x + p0 * g.cin : x + f * g.cin * g.P + p0;
    long long step = TOK ? 1 : g.P;  // from channel to channel
    if constexpr (!TOK) asm volatile("" : "+s"(step));
    float v[PT][S][16];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = (wv * S + s) * 32, left = g.cin - c - half * 16;
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) {
        const int mine = min(pt * 32 + col, have - 1);  // (a lane without a pixel reads another's)
        const unsigned at = (TOK ? mine * g.cin + half * 16 : (unsigned)(half * 16 * g.P) + mine) * 4u;
        const float* from = base + c * step;
        if (c + 32 <= g.cin) {
          if constexpr (TOK) {
#pragma unroll
            for (int j = 0; j < 16; j += 4)
              load_run<4>(reinterpret_cast<const float*>(reinterpret_cast<const char*>(from + j) + at), 4, v[pt][s] + j);
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j, from += step) v[pt][s][j] = load_at(from, at);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j, from += step) {
            v[pt][s][j] = 0.f;
            if (j < left) v[pt][s][j] = load_at(from, at);
          }
        }
      }
    }
    unsigned most[PT] = {};
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < 16; ++j) most[pt] = max(most[pt], magnitude(v[pt][s][j]));
      most[pt] = max(most[pt], (unsigned)__shfl_xor((int)most[pt], 32));
      top[(wv * PT + pt) * 32 + col] = most[pt];
    }
    __syncthreads();
    float ts[PT];
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
#pragma unroll
      for (int k = 0; k < 4; ++k) most[pt] = max(most[pt], top[(k * PT + pt) * 32 + col]);
      const bool ok = most[pt] < kInfBits;
      const Quant q(most[pt]);
      ts[pt] = q.s;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        Int4 c;
        q.codes16(v[pt][s], c);
        if (!ok) c = Int4{0, 0, 0, 0};
        shared[(pt * NK + wv * S + s) * 64 + lane] = c;
      }
    }
    __syncthreads();
    for (int t = t0 + wv; t < t1; t += 4) {
      const int o0 = t * 32, left = g.cout - o0;
      Int16 acc[PT] = {};
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        // (a row or a channel past the last is another's: not stored, times 0)
        const Int4 a = *reinterpret_cast<const Int4*>(
            w + (long long)min(o0 + col, g.cout - 1) * g.cin + min(ks * 32 + half * 16, g.cin - 16));
#pragma unroll
        for (int pt = 0; pt < PT; ++pt) {
          const Int4 b = shared[(pt * NK + ks) * 64 + lane];
          acc[pt] = TOK ? __builtin_amdgcn_mfma_i32_32x32x32_i8(b, a, acc[pt], 0, 0, 0)
                        : __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc[pt], 0, 0, 0);
        }
      }
      // register r: row 8 * (r / 4) + 4 * half + r % 4, column lane mod 32
      if constexpr (TOK) {
        const int o = min(o0 + col, g.cout - 1), part = o / g.per;
        const float sc = scales[o], be = bias ? bias[o] : 0.f;
        float* const to_row = out + ((long long)part * g.F + p0 + 4 * half) * g.per + (o - part * g.per);
        const int rows = col < left ? have - 4 * half : 0;
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r / 4) + r % 4;
            const float s = __shfl(ts[pt], row + 4 * half);
            if (pt * 32 + row < rows) to_row[(long long)(pt * 32 + row) * g.per] = fmaf((float)acc[pt][r] * s, sc, be);
          }
      } else {
        const int part = o0 / g.per;
        const bool whole = left >= 32 && have == 32 * PT && o0 + 32 <= (part + 1) * g.per;
        float* to_px = out + (((long long)part * g.F + f) * g.per + (o0 - part * g.per)) * step + p0;
        const unsigned lane_at = ((unsigned)(4 * half * g.P) + col) * 4u;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
#pragma unroll
          for (int r = 0; r < 4; ++r, to_px += step) {
            const int o = min(o0 + 8 * n + 4 * half + r, g.cout - 1);
            const float sc = scales[o], be = bias ? bias[o] : 0.f;
            const int in = o / g.per;  // the part this channel is in
#pragma unroll
            for (int pt = 0; pt < PT; ++pt) {
              const float u = fmaf((float)acc[pt][4 * n + r] * ts[pt], sc, be);
              if (whole)
                store_at<FORM == Form::Whole>(to_px + pt * 32, lane_at, u);
              else if (8 * n + 4 * half + r < left && pt * 32 + col < have)
                out[(((long long)in * g.F + f) * g.per + (o - in * g.per)) * step + p0 + pt * 32 + col] = u;
            }
          }
          to_px += 4 * step;
        }
      }
    }
    __syncthreads();  // (the codes are read)
  }
}

// Frames of up to 192 channels whose tiles of 32 output channels lie in one part,
// with aligned rows of weights: a workgroup takes a run of pixels, its waves
// quantise 32 of them at a time into LDS and then share out the products, so that a
// plane's pixels are stored one after the other.  Planes that do not start a cache
// line (Odd): the lanes of a row of products exchange places with those of the
// next 32 pixels, so that every store fills a line all the same; a run's last line
// takes pixels of the next run, whose first 32 are quantised here too.  Bandwidth
// bounds it: 64 -> 192 at 480x854 84 us, 5.0 TB/s, at 470x854 92; 192 -> 576 at
// 5x152x152 72 us, 4.9 TB/s.
template <int NK, Form FORM>
__global__ void __launch_bounds__(256, NK <= 4 ? 4 : 3)
    project_run_kernel(const float* __restrict__ x, const int8_t* __restrict__ w, const float* __restrict__ scales,
                       const float* __restrict__ bias, ProjectGeo g, float* __restrict__ out) {
  extern __shared__ char lds[];
  constexpr bool ODD = FORM == Form::Odd;
  const int slots = g.run + ODD;
  Int4* const shared = reinterpret_cast<Int4*>(lds);                      // codes, in the order of the lanes
  float* const token = reinterpret_cast<float*>(lds + slots * NK * 1024);  // scales of the pixels
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = (g.cout + 31) / 32, t0 = blockIdx.y * g.span, t1 = min(t0 + g.span, tiles);
  const Walk way = walk<ODD>(g.groups);
  for (long long grp = way.first; grp < way.end; grp += way.step) {
    const long long f = grp / g.per_frame, p0 = (grp - f * g.per_frame) * (32 * g.run);
    const int have = (int)min(32LL * slots, g.P - p0), all = (have + 31) / 32, used = min(all, g.run);
    long long step = g.P;  // from channel to channel
    int upper = half * 16;
    for (int pt = wv; pt < all; pt += 4) {
      // (else every channel's offset and guard is held in registers across the loop; so below)
      asm volatile("" : "+s"(step), "+v"(upper));
      const int mine = min(col, have - pt * 32 - 1);
      const float* const base = x + f * g.cin * g.P + p0 + pt * 32;
      const unsigned at = ((unsigned)(half * 16 * g.P) + mine) * 4u;
      float v[NK * 16];
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        const float* from = base + ks * 32 * step;
        const int left = g.cin - ks * 32 - upper;
        if (ks * 32 + 32 <= g.cin) {
#pragma unroll
          for (int j = 0; j < 16; ++j, from += step) v[ks * 16 + j] = load_at(from, at);
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j, from += step) {
            v[ks * 16 + j] = 0.f;
            if (j < left) v[ks * 16 + j] = load_at(from, at);
          }
        }
      }
      unsigned most = 0;
#pragma unroll
      for (int j = 0; j < NK * 16; ++j) most = max(most, magnitude(v[j]));
      most = max(most, (unsigned)__shfl_xor((int)most, 32));
      const bool ok = most < kInfBits;
      const Quant q(most);
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        Int4 c;
        q.codes16(v + ks * 16, c);
        if (!ok) c = Int4{0, 0, 0, 0};
        shared[(pt * NK + ks) * 64 + lane] = c;
      }
      token[pt * 32 + col] = q.s;
    }
    __syncthreads();
    const int before = ODD && p0 == 0;  // a frame's first line starts before its first pixel
    const int lines = used + before, units = (t1 - t0) * lines, last = units * (wv + 1) / 4;
    for (int u = units * wv / 4; u < last;) {
      const int t = u / lines, o0 = (t0 + t) * 32, left = g.cout - o0, part = o0 / g.per;
      const int end = min(last, (t + 1) * lines) - t * lines - before;
      int pt = u - t * lines - before;
      u = (t + 1) * lines;
      Int4 a[NK];
#pragma unroll
      for (int ks = 0; ks < NK; ++ks)  // (a row or a channel past the last is another's: not stored, times 0)
        a[ks] = *reinterpret_cast<const Int4*>(w + (long long)min(o0 + col, g.cout - 1) * g.cin +
                                               min(ks * 32 + upper, g.cin - 16));
      // register r of a product: row 8 * (r / 4) + 4 * half + r % 4, column lane mod 32
      float sc[16], be[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int o = min(o0 + 8 * (r / 4) + (upper >> 2) + r % 4, g.cout - 1);
        sc[r] = scales[o], be[r] = bias ? bias[o] : 0.f;
      }
      auto product = [&](int n, float* to) {
        Int16 acc = {};
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
          acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[ks], shared[(n * NK + ks) * 64 + lane], acc, 0, 0, 0);
        const float ts = token[n * 32 + col];
#pragma unroll
        for (int r = 0; r < 16; ++r) to[r] = fmaf((float)acc[r] * ts, sc[r], be[r]);
      };
      const long long plane = ((long long)part * g.F + f) * g.per + (o0 - part * g.per);
      float* const to = out + plane * step + p0;
      if constexpr (ODD) {
        float cur[16] = {}, next[16];
        if (pt >= 0) product(pt, cur);
        const unsigned pixels = (unsigned)g.P, first = (unsigned)((uintptr_t)out / 4) + (unsigned)plane * pixels;
        for (; pt < end; ++pt) {
          product(min(pt + 1, all - 1), next);
          asm volatile("" : "+s"(step), "+v"(upper));
          float* to_px = to + pt * 32;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
#pragma unroll
            for (int r = 0; r < 4; ++r, to_px += step) {
              const int row = 8 * n + (upper >> 2) + r;
              const int skip = -(int)(first + row * pixels) & 31;  // pixels before the line starts
              const float give = col < skip ? next[4 * n + r] : cur[4 * n + r];
              const float v = __int_as_float(__builtin_amdgcn_ds_bpermute(
                  (((col + skip) & 31) + 2 * upper) * 4, __float_as_int(give)));
              const int px = pt * 32 + col + skip;
              const unsigned lane_at = ((upper >> 2) * pixels + col + skip) * 4u;
              if (row < left && px >= 0 && px < have) store_at<true>(to_px, lane_at, v);
              cur[4 * n + r] = next[4 * n + r];
            }
            to_px += 4 * step;
          }
        }
      } else {
        auto lines_of = [&](auto count) {
          constexpr int L = decltype(count)::value;
          float v[L][16];
#pragma unroll
          for (int b = 0; b < L; ++b) product(pt + b, v[b]);
          asm volatile("" : "+s"(step), "+v"(upper));
          float* to_px = to + pt * 32;
          const unsigned lane_at = ((upper >> 2) * (unsigned)g.P + col) * 4u;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
#pragma unroll
            for (int r = 0; r < 4; ++r, to_px += step)
              if (left >= 32 || 8 * n + (upper >> 2) + r < left)
#pragma unroll
                for (int b = 0; b < L; ++b) store_at<true>(to_px + b * 32, lane_at, v[b][4 * n + r]);
            to_px += 4 * step;
          }
          pt += L;
        };
        while (pt + 2 <= end) lines_of(std::integral_constant<int, 2>());
        if (pt < end) lines_of(std::integral_constant<int, 1>());
      }
    }
    __syncthreads();  // (the codes are read)
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
                        const ProjectGeo& g, Form form, dim3 grid, float* out, hipStream_t s) {
  const size_t lds = (size_t)g.buffers * g.hold * (NK * 1024 + 128 * sizeof(float));
  const auto kernel = form == Form::Tokens ? project_kernel<NK, Form::Tokens>
                      : form == Form::Odd  ? project_kernel<NK, Form::Odd>
                                           : project_kernel<NK, Form::Whole>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), lds, s, x, codes, scales, bias, g, out);
}

snls_status launch_project(const float* x, const int8_t* codes, const float* scales, const float* bias,
                           const snls_project_params& pp, float* out, hipStream_t s) {
  const int steps = (pp.cin + 31) / 32;
  const int nk = steps <= 4 ? steps : steps <= 6 ? 6 : steps <= 8 ? 8 : steps <= 12 ? 12 : steps <= 16 ? 16 : 32;
  ProjectGeo g;
  const bool tokens = pp.pixels == 1;
  g.P = pp.pixels, g.F = pp.frames;
  g.per_frame = ((tokens ? g.F : g.P) + 127) / 128, g.groups = tokens ? g.per_frame : g.per_frame * g.F;
  g.cin = pp.cin, g.cout = pp.cout, g.per = pp.cout / pp.parts;
  const int tiles = (pp.cout + 31) / 32;
  // few pixels: the output channels are shared out too, until the chip has two workgroups a CU
  // (64x64 pixels 192 -> 576 12.9 us, 23.1 without; 2,039 tokens 12.6 and 28.0)
  const long long want = std::max(1LL, 512 / g.groups);
  const int split = (int)(want < tiles ? want : tiles);
  g.span = (tiles + split - 1) / split;
  g.aligned = pp.cin % 16 == 0 && !(reinterpret_cast<uintptr_t>(codes) & 15);
  const bool whole = pp.pixels % 32 == 0 && !(reinterpret_cast<uintptr_t>(out) & 127);
  const Form form = tokens ? Form::Tokens : whole ? Form::Whole : Form::Odd;
  // the waves share the channels: lists of tokens above 192 of them (3,000 of 384
  // channels to 384: 15.5 us, 28 with a wave a token's channels), frames above 512
  // (1,024 -> 1,024 at 2x64x64: 53 us and 84; 384 -> 384 at 5x96x96 54 and 48)
  if (g.aligned && (tokens ? nk >= 8 : nk == 32)) {
    const int PT = nk <= 12 ? 2 : 1;
    const long long full = nk == 8 || nk == 16 ? 768 : 512;  // by registers, 3 or 2 a CU
    g.per_frame = ((tokens ? g.F : g.P) + 32 * PT - 1) / (32 * PT);
    g.groups = tokens ? g.per_frame : g.per_frame * g.F;
    const long long share = std::max(1LL, std::min((long long)(tiles + 3) / 4, full / g.groups));
    g.span = (int)((tiles + share - 1) / share);
    const dim3 grid((unsigned)std::min(g.groups, 1LL << 20), (unsigned)((tiles + g.span - 1) / g.span));
    const auto kernel = nk == 8    ? project_wide_kernel<2, 2, Form::Tokens>
                        : nk == 12 ? project_wide_kernel<3, 2, Form::Tokens>
                        : nk == 16 ? project_wide_kernel<4, 1, Form::Tokens>
                        : tokens   ? project_wide_kernel<8, 1, Form::Tokens>
                        : whole    ? project_wide_kernel<8, 1, Form::Whole>
                                   : project_wide_kernel<8, 1, Form::Odd>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), PT * (nk * 1024 + 512), s, x, codes, scales, bias, g, out);
    return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
  }
  // Runs of pixels, against 128 pixels a workgroup: planes that start a line, 64 ->
  // 192 at 480x854 84 us and 90, 192 -> 576 at 5x152x152 72 and 77, but 16 -> 384 at
  // 304x622 63 and 61; planes that do not, 470x854 92 and 123, 32 -> 64 at 9x397x391
  // 117 and 173, but 16 -> 384 at 305x620 74 and 66, and nothing won or less where
  // the 256 MB of cache hold all: 271x483 32 and 25, 96 -> 96 at 435x437 39 and 37.
  // The border of 268 MB of output is a coarse one: below it runs are the faster from
  // about 190,000 odd pixels on on inputs that no cache holds (64 -> 192 at 305x622 45
  // and 56, 438x795 83 and 110; 32 -> 64 at 700x1003 60 and 75; 96 -> 96 at 600x667 77
  // and 80, 192 -> 192 at 300x601 82 and 75).
  if (!tokens && nk <= 6 && g.aligned && (pp.parts == 1 || g.per % 32 == 0) && pp.cout <= 8 * pp.cin &&
      (whole || g.F * g.P * g.cout > 1LL << 26)) {
    // as many workgroups as the chip holds at once, by registers, take the frames in
    // as few turns as LDS allows, of the same length
    const int by_regs = nk <= 4 ? 4 : 3, slot = nk * 1024 + 128, odd = form == Form::Odd;
    const long long all = (g.P + 31) / 32 * g.F, held = 256LL * by_regs;
    const int most = 160 * 1024 / by_regs / slot - odd;
    const long long turns = (all + held * most - 1) / (held * most);
    g.run = (int)((all + held * turns - 1) / (held * turns));
    g.per_frame = (g.P + 32 * g.run - 1) / (32 * g.run), g.groups = g.per_frame * g.F;
    const long long share = std::max(1LL, std::min((long long)tiles, 512 / g.groups));
    g.span = (int)((tiles + share - 1) / share);
    const dim3 grid((unsigned)std::min(g.groups, held), (unsigned)((tiles + g.span - 1) / g.span));
#define SNLS_RUN(K) (odd ? project_run_kernel<K, Form::Odd> : project_run_kernel<K, Form::Whole>)
    const auto kernel = nk == 1   ? SNLS_RUN(1)
                        : nk == 2 ? SNLS_RUN(2)
                        : nk == 3 ? SNLS_RUN(3)
                        : nk == 4 ? SNLS_RUN(4)
                                  : SNLS_RUN(6);
#undef SNLS_RUN
    hipLaunchKernelGGL(kernel, grid, dim3(256), (g.run + odd) * slot, s, x, codes, scales, bias, g, out);
    return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
  }
  // 60 KB of weights and what goes with them at once, or two buffers of 32 KB, of
  // one tile at least (33 KB with 1,024 channels)
  const int tile = nk * 1024 + 512;
  g.buffers = g.span * tile <= 60 * 1024 ? 1 : 2;
  g.hold = g.buffers == 1 ? g.span : std::max(1, 32 * 1024 / tile);
  // as many workgroups as the chip holds at once, by registers and by LDS (48 -> 96
  // channels at 4x271x483 73 us, 89 with 5 a CU, where 4 fit)
  const int by_regs = nk <= 2 ? 4 : nk == 3 ? 3 : 2, by_lds = 160 * 1024 / (g.buffers * g.hold * tile);
  const dim3 grid((unsigned)std::min(g.groups, 256LL * std::min(by_regs, by_lds)),
                  (unsigned)((tiles + g.span - 1) / g.span));
  switch (nk) {
    case 1: run_project<1>(x, codes, scales, bias, g, form, grid, out, s); break;
    case 2: run_project<2>(x, codes, scales, bias, g, form, grid, out, s); break;
    case 3: run_project<3>(x, codes, scales, bias, g, form, grid, out, s); break;
    case 4: run_project<4>(x, codes, scales, bias, g, form, grid, out, s); break;
    case 6: run_project<6>(x, codes, scales, bias, g, form, grid, out, s); break;
    case 8: run_project<8>(x, codes, scales, bias, g, form, grid, out, s); break;
    case 12: run_project<12>(x, codes, scales, bias, g, form, grid, out, s); break;
    case 16: run_project<16>(x, codes, scales, bias, g, form, grid, out, s); break;
    default: run_project<32>(x, codes, scales, bias, g, form, grid, out, s); break;
  }
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
