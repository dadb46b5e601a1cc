// norm.hip -- layer norm over the channels of every pixel, of a residual sum
// with dropout, and its gradients (snls_norm, snls_norm_backward).
#include <algorithm>

#include "lanes.h"
#include "philox.h"
#include "row16.h"

namespace snls {

// What a call's kernels share.
struct NormGeo {
  long long frames, P;
  long long tiles, per_frame;  // runs of pixels, of a frame
  int C, n;                    // n: channels a wave takes
  float eps;
};

// Frames: a workgroup of W waves takes 64 * V consecutive pixels, V a lane, and
// every wave up to R channels of them; the values stay in registers from their
// only read on, and the sums over the channels are joined in LDS: first the
// mean, then the squares of the differences from it.  16 bytes an element of a
// residual sum, 8 without: bandwidth bounds it.  V = 2 keeps more waves on the
// chip than V = 4 does (5x64x480x854: 201 and 243 us) and needs half the
// instructions of V = 1 (633 us); 8 channels a wave where 16 waves are enough.
// Measured: the residual sum with dropout 400 us, 5.3 TB/s.  Where planes do not
// start a cache line (WHOLE false), neighbouring tiles lie on one XCD
// (4x64x270x483: 126 us, 147 in the order of the tiles; at 5x64x480x854 that
// order is the faster, 399 and 426).
template <int R, bool WHOLE>
__global__ void __launch_bounds__(1024) norm_tile_kernel(const float* x, const float* branch, Drop d,
                                                         const float* __restrict__ gamma,
                                                         const float* __restrict__ beta, NormGeo g, float* total,
                                                         float* y, float* stats) {
  constexpr int V = 2;
  extern __shared__ float part[];  // sums, then squares: a row a wave
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Philox gen(d);
  // (a row of sums is written again only behind a barrier that follows its last read)
  const Walk way = walk<!WHOLE>(g.tiles);
  for (long long tile = way.first; tile < way.end; tile += way.step) {
    const long long f = tile / g.per_frame, p = (tile - f * g.per_frame) * (64 * V) + lane * V;
    const int cnt = (int)max(0LL, min((long long)V, g.P - p));
    const int c0 = wv * g.n, n = min(g.n, g.C - c0);
    const long long at = (f * g.C + c0) * g.P + (cnt > 0 ? p : 0);
    float s[R][V];
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n) load_run<V>(x + at + c * g.P, cnt, s[c]);
    if (branch) {
      const bool shared = !(g.P & 3);  // two lanes, one block in every plane
#pragma unroll
      for (int c2 = 0; c2 < R; c2 += 2) {
        unsigned w[2][V];
        if (d.rng && shared && c2 < n) share_blocks(gen.block((at + (c2 + (lane & 1)) * g.P) >> 2), lane & 1, w);
#pragma unroll
        for (int c = c2; c < c2 + 2; ++c)
          if (c < n) {
            float b[V];
            load_run<V>(branch + at + c * g.P, cnt, b);
            if (d.rng) {
              if (!shared) gen.run<V>(at + c * g.P, w[c - c2]);
#pragma unroll
              for (int j = 0; j < V; ++j) b[j] = dropped(b[j], w[c - c2][j], d);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) s[c][j] += b[j];
            put_run<WHOLE, V>(total + at + c * g.P, cnt, s[c]);
          }
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
        put_run<WHOLE, V>(y + at + c * g.P, cnt, o);
      }
    if (stats && wv == 0) {
      store_run<V>(stats + f * g.P + (cnt > 0 ? p : 0), cnt, mean);
      store_run<V>(stats + (g.frames + f) * g.P + (cnt > 0 ? p : 0), cnt, rstd);
    }
  }
}

// v of lane ^ M, M below 16.
template <int M>
SNLS_DEV double partner_value(double v, int lane) {
  return __longlong_as_double((long long)grp_xor64<M>((unsigned long long)__double_as_longlong(v), lane & 15));
}

// One step of the sum of a list over the lanes: a lane with bit M set goes on
// with b, the others with a, each plus what its partner (lane ^ M) has of it.
template <int M>
SNLS_DEV double halve(double a, double b, int lane) {
  if constexpr (M >= 16) {
    // the rows of a whose lanes have the bit change places with those of b whose
    // lanes have not
    const auto swap = [](unsigned ua, unsigned ub) {
      return M == 32 ? __builtin_amdgcn_permlane32_swap(ua, ub, false, false)
                     : __builtin_amdgcn_permlane16_swap(ua, ub, false, false);
    };
    const auto lo = swap((unsigned)__double2loint(a), (unsigned)__double2loint(b));
    const auto hi = swap((unsigned)__double2hiint(a), (unsigned)__double2hiint(b));
    return __hiloint2double((int)hi[0], (int)lo[0]) + __hiloint2double((int)hi[1], (int)lo[1]);
  } else {
    const bool up = lane & M;
    const double give = up ? a : b, keep = up ? b : a;
    return keep + partner_value<M>(give, lane);
  }
}

// Sums over 2 M lanes of LEN values each (a power of two up to 2 M): lane l of
// them returns that of value l / (2 M / LEN).
template <int LEN, int M>
SNLS_DEV double list_sum(double* v, int lane) {
  if constexpr (M == 0) {
    return v[0];
  } else if constexpr (LEN > 1) {
#pragma unroll
    for (int i = 0; i < LEN / 2; ++i) v[i] = halve<M>(v[i], v[i + LEN / 2], lane);
    return list_sum<LEN / 2, M / 2>(v, lane);
  } else {
    v[0] += partner_value<M>(v[0], lane);
    return list_sum<1, M / 2>(v, lane);
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
// many; one read.  16 lanes up to 128 channels: 64 would stand idle there (100,000
// tokens of 48 channels 13.1 us with 16, 32.7 with 64; the gradients 21.6 and 50.0).
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
// them again.  One lane adds up all of them, up to 65,535, so in 64 bits
// (4x600x96x96 558 us, 546 with sums in 32).  Not tuned: a thread's loads wait for
// each other, and for tokens the lanes' loads are C floats apart (64 tokens of 4,096
// channels 1.6 ms, 4,000 2.4 ms; the gradients 1.8 and 3.4 ms).
__global__ void __launch_bounds__(256) norm_kernel(const float* x, const float* branch, Drop d,
                                                   const float* __restrict__ gamma, const float* __restrict__ beta,
                                                   long long frames, int C, long long P, float eps, float* total,
                                                   float* y, float* stats) {
  const Philox gen(d);
  const long long px = frames * P;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < px; i += gridDim.x * 256LL) {
    const long long f = i / P, at = f * C * P + (i - f * P);
    double sum = 0.0;
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
      sum += (double)v;
    }
    const float* from = branch ? total : x;
    const float mean = (float)(sum / C);
    double sq = 0.0;
    for (int c = 0; c < C; ++c) {
      const double t = (double)(from[at + c * P] - mean);
      sq = fma(t, t, sq);
    }
    const float rstd = 1.f / sqrtf((float)(sq / C) + eps);
    for (int c = 0; c < C; ++c) {
      const float t = (from[at + c * P] - mean) * rstd;
      y[at + c * P] = fmaf(t, gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
    }
    if (stats) stats[i] = mean, stats[px + i] = rstd;
  }
}

// Gradients of frames: tiles, waves and channels as in the forward pass.  Both
// the scaled gradients and the normalised values stay in registers, one join of
// two sums a tile.  A workgroup walks every gridDim.x-th tile, at most 64 of them,
// and a lane adds up the terms of the weights' gradients of its and its partner's
// pixels (lane ^ 32), the lower lanes gamma's, the upper lanes beta's; at the end a
// wave's lanes are left with one sum each, and a workgroup writes one row of
// partial sums.  Products and sums of these terms are in 64 bits from the start:
// the vector units have the time (16x64x256x256 163.4 us, 162.5 with sums in 32;
// 4x48x271x483 66.2 and 66.1).
template <int R, bool WHOLE>
__global__ void __launch_bounds__(1024) norm_grad_tile_kernel(const float* grad_y, const float* grad_total,
                                                              const float* __restrict__ total,
                                                              const float* __restrict__ stats,
                                                              const float* __restrict__ gamma, Drop d, NormGeo g,
                                                              float* grad_x, float* grad_branch,
                                                              double* __restrict__ sums) {
  constexpr int V = 4;
  extern __shared__ float part[];  // two tables of two rows a wave, taken in turn
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Philox gen(d);
  const int c0 = wv * g.n, n = min(g.n, g.C - c0);
  double over[R] = {};  // this lane's sums over the tiles
  int turn = 0;
  const Walk way = walk<!WHOLE>(g.tiles);
  for (long long tile = way.first; tile < way.end; tile += way.step) {
    const long long f = tile / g.per_frame, p = (tile - f * g.per_frame) * (64 * V) + lane * V;
    const int cnt = (int)max(0LL, min((long long)V, g.P - p));
    const long long px = f * g.P + (cnt > 0 ? p : 0), at = (f * g.C + c0) * g.P + (cnt > 0 ? p : 0);
    float mean[V], rstd[V], gy[R][V], xh[R][V], sum[2][V] = {};
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n) {
        load_run<V>(grad_y + at + c * g.P, cnt, gy[c]);
        load_run<V>(total + at + c * g.P, cnt, xh[c]);
      }
    load_run<V>(stats + px, cnt, mean);
    load_run<V>(stats + g.frames * g.P + px, cnt, rstd);
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n) {
        const float ga = gamma ? gamma[c0 + c] : 1.f;
        double tg = 0.0, tb = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          xh[c][j] = (xh[c][j] - mean[j]) * rstd[j];
          tg = fma((double)gy[c][j], (double)xh[c][j], tg);
          tb += (double)gy[c][j];
          gy[c][j] *= ga;
          sum[0][j] += gy[c][j];
          sum[1][j] = fmaf(gy[c][j], xh[c][j], sum[1][j]);
        }
        over[c] += halve<32>(tg, tb, lane);
      }
    if (waves > 1) {
      float* const rows = part + turn * 2 * waves * V * 64;
      turn ^= 1;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        rows[(wv * V + j) * 64 + lane] = sum[0][j];
        rows[((waves + wv) * V + j) * 64 + lane] = sum[1][j];
        sum[0][j] = sum[1][j] = 0.f;
      }
      __syncthreads();
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          sum[0][j] += rows[(w * V + j) * 64 + lane];
          sum[1][j] += rows[((waves + w) * V + j) * 64 + lane];
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sum[0][j] /= g.C, sum[1][j] /= g.C;
#pragma unroll
    for (int c = 0; c < R; ++c)
      if (c < n) {
        const long long e = at + c * g.P;
        float r[V], t[V];
        if (grad_total) load_run<V>(grad_total + e, cnt, t);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          r[j] = rstd[j] * (gy[c][j] - sum[0][j] - xh[c][j] * sum[1][j]);
          if (grad_total) r[j] += t[j];
        }
        put_run<WHOLE, V>(grad_x + e, cnt, r);
        if (grad_branch) {
          if (d.rng) {
            unsigned w[V];
            gen.run<V>(e, w);
#pragma unroll
            for (int j = 0; j < V; ++j) r[j] = dropped(r[j], w[j], d);
          }
          put_run<WHOLE, V>(grad_branch + e, cnt, r);
        }
      }
  }
  if (!sums) return;
  const double acc = list_sum<R, 16>(over, lane);  // this lane's of the R sums of its half
  const int c = (lane & 31) / (32 / R);
  if (lane % (32 / R) == 0 && c < n) sums[((long long)blockIdx.x * 2 + lane / 32) * g.C + c0 + c] = acc;
}

// Gradients of frames of many channels: one pixel a lane, L = 64 pixels a tile up
// to 256 channels, 32 and two channels side by side in a wave up to 512, so that
// 64 registers hold a wave's tile and two workgroups of 8 waves fit a CU, one
// loading while the other stores (5x256x128x128 without dropout 59 us, with one
// workgroup of 16 waves 75; 5x384x96x96 60 and 77).  The terms of the weights'
// gradients are multiplied and summed over the pixels in 64 bits; those figures
// were taken with 32, against which 64 cost 2 us (59.8 -> 62.0, 62.0 -> 64.2).
template <int L, int R, bool WHOLE>
__global__ void __launch_bounds__(512, 4) norm_grad_wide_kernel(const float* grad_y, const float* grad_total,
                                                                const float* __restrict__ total,
                                                                const float* __restrict__ stats,
                                                                const float* __restrict__ gamma, Drop d, NormGeo g,
                                                                float* grad_x, float* grad_branch,
                                                                double* __restrict__ sums) {
  constexpr int SIDE = 64 / L;     // channels a step; R steps a wave
  extern __shared__ float part[];  // two tables of two rows a wave, taken in turn, and gamma
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6, l = lane & (L - 1), side = lane / L;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Philox gen(d);
  const int c0 = wv * g.n * SIDE, n = min(g.n, (g.C - c0 + SIDE - 1) / SIDE);
  const int own = min(n, (g.C - c0 - side + SIDE - 1) / SIDE);  // this lane's steps: n, or one less
  float* const scale = part + 4 * waves * 64;
  for (int c = threadIdx.x; c < waves * g.n * SIDE; c += blockDim.x) scale[c] = gamma && c < g.C ? gamma[c] : 1.f;
  __syncthreads();
  double acc[R / 8] = {};
  int turn = 0;
  const Walk way = walk<!WHOLE>(g.tiles);
  for (long long tile = way.first; tile < way.end; tile += way.step) {
    const long long f = tile / g.per_frame, p = (tile - f * g.per_frame) * L;
    const bool in = l < g.P - p;
    const unsigned here = in ? l : 0;
    const long long at = (f * g.C + c0) * g.P + p;  // the wave's first element
    // a lane without a pixel, or without a channel in the last step, reads another's
    unsigned off = (here + side * (unsigned)g.P) * 4u;
    auto place = [&](int k) { return SIDE > 1 && k == n - 1 && own < n ? here * 4u : off; };
    long long step = SIDE * g.P;
    asm volatile("" : "+s"(step), "+v"(off));  // (else every step's offset is held in registers across the tiles)
    float gy[R], xh[R];
    {
      const float *a = grad_y + at, *b = total + at;
#pragma unroll
      for (int k = 0; k < R; ++k, a += step, b += step)
        if (k < n) gy[k] = load_at(a, place(k)), xh[k] = load_at(b, place(k));
    }
    const float mean = load_at(stats + f * g.P + p, here * 4u);
    const float rstd = load_at(stats + (g.frames + f) * g.P + p, here * 4u);
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int k0 = 0; k0 < R; k0 += 8)
      if (k0 < n) {
        double over[8] = {};  // the lower half's lanes gamma's terms, the upper half's beta's
#pragma unroll
        for (int k = k0; k < k0 + 8; ++k)
          if (k < n) {
            const bool ok = in && k < own;
            gy[k] = ok ? gy[k] : 0.f;
            xh[k] = ok ? (xh[k] - mean) * rstd : 0.f;
            if (sums) over[k - k0] = halve<L / 2>((double)gy[k] * (double)xh[k], (double)gy[k], lane);
            gy[k] *= scale[c0 + k * SIDE + side];
            s0 += gy[k];
            s1 = fmaf(gy[k], xh[k], s1);
          }
        if (sums) acc[k0 / 8] += list_sum<8, L / 4>(over, lane);
      }
    if (L == 32) s0 += __shfl_xor(s0, 32), s1 += __shfl_xor(s1, 32);
    float* const rows = part + turn * 2 * waves * 64;
    turn ^= 1;
    rows[wv * 64 + lane] = s0, rows[(waves + wv) * 64 + lane] = s1;
    __syncthreads();
    s0 = s1 = 0.f;
    for (int w = 0; w < waves; ++w) s0 += rows[w * 64 + lane], s1 += rows[(waves + w) * 64 + lane];
    s0 /= g.C, s1 /= g.C;
    const bool shared = !(g.P & 3);  // four lanes, one block in every plane
    long long e = at;
#pragma unroll
    for (int k0 = 0; k0 < R; k0 += 4)
      if (k0 < n) {
        float t[4];
        if (grad_total) {
          const float* a = grad_total + e;
#pragma unroll
          for (int k = 0; k < 4; ++k, a += step)
            if (k0 + k < n) t[k] = load_at(a, place(k0 + k));
        }
        unsigned w[4];
        if (d.rng && shared) share_blocks(gen.block((e + off / 4 + (lane & 3) * step) >> 2), (int)(l & 3), w);
#pragma unroll
        for (int k = 0; k < 4; ++k, e += step)
          if (k0 + k < n) {
            float r = rstd * (gy[k0 + k] - s0 - xh[k0 + k] * s1);
            if (grad_total) r += t[k];
            if (d.rng && !shared) gen.run<1>(e + off / 4, w + k);
            if (in && k0 + k < own) {
              store_at<WHOLE>(grad_x + e, off, r);
              if (grad_branch) store_at<WHOLE>(grad_branch + e, off, d.rng ? dropped(r, w[k], d) : r);
            }
          }
      }
  }
  if (!sums) return;
  const int which = l / (L / 2), step = l % (L / 2) / (L / 16);  // of the 2 sums of 8 steps
#pragma unroll
  for (int k0 = 0; k0 < R; k0 += 8) {
    const int k = k0 + step;
    if (l % (L / 16) == 0 && k < own)
      sums[((long long)blockIdx.x * 2 + which) * g.C + c0 + k * SIDE + side] = acc[k0 / 8];
  }
}

// Gradients of tokens: G lanes a token, as in the forward pass; a workgroup
// walks rows and keeps its channels' sums in 64 bits, joined over its groups at the
// end.
template <int G, int N>
__global__ void __launch_bounds__(256) norm_grad_token_kernel(const float* grad_y, const float* grad_total,
                                                              const float* __restrict__ total,
                                                              const float* __restrict__ stats,
                                                              const float* __restrict__ gamma, Drop d, NormGeo g,
                                                              float* grad_x, float* grad_branch,
                                                              double* __restrict__ sums) {
  __shared__ double rows[256 / G][G * N * 4];
  const int l = threadIdx.x & (G - 1), group = threadIdx.x / G;
  const Philox gen(d);
  double acc[2][N][4] = {};
  float ga[N][4];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int c = (k * G + l) * 4, cnt = max(0, min(4, g.C - c));
#pragma unroll
    for (int j = 0; j < 4; ++j) ga[k][j] = 1.f;
    if (gamma && cnt > 0) load_run<4>(gamma + c, cnt, ga[k]);
  }
  for (long long row = blockIdx.x * (256LL / G) + group; row < g.frames; row += gridDim.x * (256LL / G)) {
    const long long at = row * g.C;
    const float mean = stats[row], rstd = stats[g.frames + row];
    float gy[N][4], xh[N][4], s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = (k * G + l) * 4, cnt = max(0, min(4, g.C - c));
      load_run<4>(grad_y + at + (cnt > 0 ? c : 0), cnt, gy[k]);
      load_run<4>(total + at + (cnt > 0 ? c : 0), cnt, xh[k]);
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = (k * G + l) * 4 + j < g.C;
        xh[k][j] = in ? (xh[k][j] - mean) * rstd : 0.f;
        acc[0][k][j] = fma((double)gy[k][j], (double)xh[k][j], acc[0][k][j]);
        acc[1][k][j] += (double)gy[k][j];
        gy[k][j] *= ga[k][j];
        s0 += gy[k][j];
        s1 = fmaf(gy[k][j], xh[k][j], s1);
      }
    s0 = group_sum<G>(s0) / g.C, s1 = group_sum<G>(s1) / g.C;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = (k * G + l) * 4, cnt = min(4, g.C - c);
      if (cnt <= 0) continue;
      float r[4], t[4] = {};
      if (grad_total) load_run<4>(grad_total + at + c, cnt, t);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        r[j] = rstd * (gy[k][j] - s0 - xh[k][j] * s1);
        if (grad_total) r[j] += t[j];
      }
      store_run<4>(grad_x + at + c, cnt, r);
      if (grad_branch) {
        if (d.rng) {
          unsigned w[4];
          gen.run<4>(at + c, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) r[j] = dropped(r[j], w[j], d);
        }
        store_run<4>(grad_branch + at + c, cnt, r);
      }
    }
  }
  if (!sums) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which) __syncthreads();  // (the first sums are read)
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) rows[group][(k * G + l) * 4 + j] = acc[which][k][j];
    __syncthreads();
    for (int c = threadIdx.x; c < g.C; c += 256) {
      double s = 0.0;
      for (int k = 0; k < 256 / G; ++k) s += rows[k][c];
      sums[((long long)blockIdx.x * 2 + which) * g.C + c] = s;
    }
  }
}

// More channels than registers hold: a thread per pixel, gradients of the input and
// the branch; sums over the channels in 64 bits, as above.
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
    double over = 0.0, over_x = 0.0;
    for (int c = 0; c < C; ++c) {
      const float g = grad_y[at + c * P] * (gamma ? gamma[c] : 1.f), xh = (total[at + c * P] - mean) * rstd;
      over += (double)g;
      over_x = fma((double)g, (double)xh, over_x);
    }
    const float sg = (float)(over / C), sgx = (float)(over_x / C);
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
    sg += (double)g * (double)((total[e] - stats[i]) * stats[px + i]);
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

// The 2 C sums of all slices: 8 entries a workgroup, 128 lanes in turn over the
// slices of each.
constexpr int kEntries = 8;
__global__ void __launch_bounds__(1024) norm_weights_sum_kernel(const double* __restrict__ part, int slices, int C,
                                                                float* __restrict__ grad_gamma,
                                                                float* __restrict__ grad_beta) {
  __shared__ double sums[1024];
  const int i = blockIdx.x * kEntries + (threadIdx.x % kEntries), group = threadIdx.x / kEntries;
  double s = 0.0;
  if (i < 2 * C)
    for (int k = group; k < slices; k += 1024 / kEntries) s += part[(long long)k * 2 * C + i];
  sums[threadIdx.x] = s;
  __syncthreads();
  for (int half = 512 / kEntries; half > 0; half /= 2) {
    if (group < half) sums[threadIdx.x] += sums[threadIdx.x + half * kEntries];
    __syncthreads();
  }
  if (group == 0 && i < 2 * C) (i < C ? grad_gamma : grad_beta)[i < C ? i : i - C] = (float)sums[threadIdx.x];
}

constexpr long long kMostGroups = 1 << 21;  // a launch holds less than 2^32 threads

// Whether planes start a cache line (as torch's allocations do).
static bool whole_lines(const snls_norm_params& np) { return np.pixels % 32 == 0; }

// Waves that share a tile's channels, n each, if 16 are enough.
static int tile_waves(int C, int n) { return std::min(16, (C + n - 1) / n); }

// How the gradients of a call are cut.  slices: rows of partial sums.
struct GradCut {
  enum { Tokens, Tiles, Pixels } form;
  bool wide;       // more than 128 channels
  int run, waves;  // pixels a tile, waves
  long long units;  // tiles, or groups of tokens
  long long slices;
};

static GradCut grad_cut(const snls_norm_params& np) {
  GradCut c = {};
  if (np.pixels == 1 && np.C <= 1024) {
    c.form = GradCut::Tokens;
    const int per = np.C <= 128 ? 16 : 4;
    c.units = (np.frames + per - 1) / per;
  } else if (np.pixels > 1 && np.C <= 512) {
    c.form = GradCut::Tiles;
    c.wide = np.C > 128;
    c.run = !c.wide ? 256 : np.C <= 256 ? 64 : 32;
    c.waves = !c.wide ? tile_waves(np.C, 8) : 8;
    c.units = np.frames * ((np.pixels + c.run - 1) / c.run);
  } else {
    c.form = GradCut::Pixels;
    c.slices = 64;
    return c;
  }
  // the chip is full with 512, with workgroups of up to 4 waves with 1,024
  // (4x16x271x483: 29.7 us, 36.3 with 512; 48 channels, 6 waves: 87 with 512, 103
  // with 1,024); 64 units a workgroup at most, but for lists that no launch of so
  // many workgroups holds
  const long long full = c.form == GradCut::Tiles && c.waves <= 4 ? 1024 : 512;
  c.slices = std::min(std::max(std::min(c.units, full), (c.units + 63) / 64), 1LL << 20);
  return c;
}

size_t norm_backward_ws_bytes(const snls_norm_params& np) {
  return (size_t)std::max(grad_cut(np).slices, 1LL) * 2 * np.C * sizeof(double);
}

static unsigned pixel_groups(const snls_norm_params& np) {
  const long long groups = (np.frames * np.pixels + 255) / 256;
  return (unsigned)(groups < 16384 ? groups : 16384);
}

snls_status launch_norm(const float* x, const float* branch, const Drop& drop, const float* gamma, const float* beta,
                        const snls_norm_params& np, float* total, float* y, float* stats, hipStream_t s) {
  NormGeo g = {np.frames, np.pixels, 0, 0, np.C, 0, np.eps};
  if (np.pixels == 1 && np.C <= 2048) {
    const int per = np.C <= 128 ? 16 : 4;
    const long long groups = (np.frames + per - 1) / per;
    const dim3 grid((unsigned)std::min(groups, kMostGroups));
    const auto kernel = np.C <= 64     ? norm_token_kernel<16, 1>
                        : np.C <= 128  ? norm_token_kernel<16, 2>
                        : np.C <= 256  ? norm_token_kernel<64, 1>
                        : np.C <= 1024 ? norm_token_kernel<64, 4>
                                       : norm_token_kernel<64, 8>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, x, branch, drop, gamma, beta, g, total, y, stats);
  } else if (np.pixels > 1 && np.C <= 512) {
    const int waves = tile_waves(np.C, 8);
    g.n = (np.C + waves - 1) / waves;
    g.per_frame = (np.pixels + 127) / 128, g.tiles = g.per_frame * np.frames;
    const dim3 grid((unsigned)std::min(g.tiles, kMostGroups)), block(64 * waves);
    const size_t lds = waves > 1 ? 2 * waves * 128 * sizeof(float) : 0;
    const bool whole = whole_lines(np);
#define SNLS_TILES(R) (whole ? norm_tile_kernel<R, true> : norm_tile_kernel<R, false>)
    const auto kernel = g.n <= 8    ? SNLS_TILES(8)
                        : g.n <= 16 ? SNLS_TILES(16)
                        : g.n <= 24 ? SNLS_TILES(24)
                                    : SNLS_TILES(32);
#undef SNLS_TILES
    hipLaunchKernelGGL(kernel, grid, block, lds, s, x, branch, drop, gamma, beta, g, total, y, stats);
  } else {
    hipLaunchKernelGGL(norm_kernel, dim3(pixel_groups(np)), dim3(256), 0, s, x, branch, drop, gamma, beta, np.frames,
                       np.C, np.pixels, np.eps, total, y, stats);
  }
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

snls_status launch_norm_backward(const float* grad_y, const float* grad_total, const float* total, const float* stats,
                                 const float* gamma, const Drop& drop, const snls_norm_params& np, float* grad_x,
                                 float* grad_branch, float* grad_gamma, float* grad_beta, double* ws, hipStream_t s) {
  const GradCut cut = grad_cut(np);
  double* const sums = grad_gamma ? ws : nullptr;
  NormGeo g = {np.frames, np.pixels, cut.units, 0, np.C, 0, np.eps};
  const dim3 grid((unsigned)cut.slices);
  if (np.frames > 0 && cut.form == GradCut::Tiles) {
    const int side = cut.wide && cut.run == 32 ? 2 : 1;
    g.n = (np.C + side * cut.waves - 1) / (side * cut.waves);
    g.per_frame = cut.units / np.frames;
    const dim3 block(64 * cut.waves);
    // two tables of two rows a wave, one pixel or four a lane; many channels: gamma
    const size_t lds = cut.waves > 1 ? 4 * cut.waves * (cut.wide ? 1 : 4) * 256 + (cut.wide ? 512 * 4 : 0) : 0;
    const bool whole = whole_lines(np);
#define SNLS_WIDE(L, R) (whole ? norm_grad_wide_kernel<L, R, true> : norm_grad_wide_kernel<L, R, false>)
    const auto kernel = !cut.wide     ? (whole ? norm_grad_tile_kernel<8, true> : norm_grad_tile_kernel<8, false>)
                        : np.C <= 256 ? SNLS_WIDE(64, 32)
                        : np.C <= 384 ? SNLS_WIDE(32, 24)
                                      : SNLS_WIDE(32, 32);
#undef SNLS_WIDE
    hipLaunchKernelGGL(kernel, grid, block, lds, s, grad_y, grad_total, total, stats, gamma, drop, g, grad_x,
                       grad_branch, sums);
  } else if (np.frames > 0 && cut.form == GradCut::Tokens) {
    const auto kernel = np.C <= 64    ? norm_grad_token_kernel<16, 1>
                        : np.C <= 128 ? norm_grad_token_kernel<16, 2>
                        : np.C <= 256 ? norm_grad_token_kernel<64, 1>
                                      : norm_grad_token_kernel<64, 4>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, grad_y, grad_total, total, stats, gamma, drop, g, grad_x,
                       grad_branch, sums);
  } else {
    // the sums over the pixels come first: grad_x may be grad_y
    if (sums && np.frames > 0)
      hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)np.C, (unsigned)cut.slices), dim3(256), 0, s, grad_y,
                         total, stats, np.frames, np.C, np.pixels, ws);
    if (np.frames > 0)
      hipLaunchKernelGGL(norm_grad_kernel, dim3(pixel_groups(np)), dim3(256), 0, s, grad_y, grad_total, total, stats,
                         gamma, drop, np.frames, np.C, np.pixels, grad_x, grad_branch);
  }
  if (sums)
    hipLaunchKernelGGL(norm_weights_sum_kernel, dim3((unsigned)((2 * np.C + kEntries - 1) / kEntries)), dim3(1024), 0,
                       s, ws, np.frames > 0 ? (int)cut.slices : 0, np.C, grad_gamma, grad_beta);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
