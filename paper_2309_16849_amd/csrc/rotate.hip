// rotate.hip -- rotary positions over time, rows and columns (snls_rotate,
// snls_rotate_points).
#include <algorithm>

#include "lanes.h"

namespace snls {
constexpr int kRows = 2;  // rows a lane takes, all in flight

// cos and sin of pos * turns turns.  The angle is formed and reduced to the
// nearest quarter turn in 64 bits: turns is off by at most 1.25 * 2^-53 of it, pos
// (past 2^53) and the product by 2^-53 each, in all less than 2^-51 of the angle,
// and the reduction is exact.  What is rounded to fp32 is at most an eighth of a
// turn: 2.3e-8 radians more.
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

// How the frames of a call are cut: a workgroup takes `rows` rows of up to 1024
// columns of the two planes of a pair (or of a plane that is copied).
struct RotateGeo {
  long long heads;         // B * T * HD
  int units, quads, cols;  // quads: runs of four columns in a block of columns; cols: such blocks
  int steps;               // rows a workgroup takes at once, a lane a run
  int rows, chunks;        // chunks of rows
};

// 8 bytes a pair read and as many written: bandwidth bounds it.  A lane keeps its
// four columns down kRows rows, all in flight, so that the angles of a column
// pair and of a time pair are formed once, those of a row pair once a row:
// 5x64x480x854 q and k, 889 us with a thread and a phase per pixel, 378 so
// (5.6 TB/s).  Short workgroups keep the loads near each other: with 8 rows a lane
// and 512 lanes the same took 405, 9x32x491x523 243 instead of 205, 720x1280 284
// instead of 271; with one row a lane 396, 251 and 312.
template <bool WHOLE>
__global__ void __launch_bounds__(256) rotate_kernel(const float* q, const float* k,
                                                     const int64_t* __restrict__ times, Rotary r, RotateGeo g,
                                                     float* q_out, float* k_out) {
  const long long HW = (long long)r.H * r.W;
  const int down = threadIdx.x / g.quads, steps = g.steps;
  const int col = ((int)(blockIdx.x % g.cols) * 256 + (int)threadIdx.x - down * g.quads) * 4, cnt = r.W - col;
  const int row0 = (int)(blockIdx.x / g.cols) * g.rows, row1 = min(row0 + g.rows, r.H);
  for (long long h = blockIdx.z; h < (k ? 2 : 1) * g.heads; h += gridDim.z) {
    const bool second = h >= g.heads;
    const long long head = second ? h - g.heads : h, bt = head / r.HD;
    const float* const src = (second ? k : q) + head * r.Ch * HW;
    float* const dst = (second ? k_out : q_out) + head * r.Ch * HW;
    for (int p = blockIdx.y; p < g.units; p += gridDim.y) {
      if (p >= r.total) {
        // (rows are one run of floats here, shared out over the blocks of columns)
        const long long c = (r.total + p) * HW, at = (long long)row0 * r.W, n = (long long)(row1 - row0) * r.W;
        const float* const a = src + (c + at);
        float* const o = dst + (c + at);
        const long long stride = (long long)g.cols * blockDim.x * 4;
        if (src != dst)
          for (long long i = (blockIdx.x % g.cols * blockDim.x + threadIdx.x) * 4LL; i < n; i += kRows * stride) {
            float v[kRows][4];
#pragma unroll
            for (int u = 0; u < kRows; ++u)
              if (i + u * stride < n) load_run<4>(a + i + u * stride, (int)min(4LL, n - i - u * stride), v[u]);
#pragma unroll
            for (int u = 0; u < kRows; ++u)
              if (i + u * stride < n) put_run<WHOLE, 4>(o + i + u * stride, (int)min(4LL, n - i - u * stride), v[u]);
          }
        continue;
      }
      if (down >= steps || cnt <= 0) continue;
      const Pair pr = pair_of(p, r);
      const double turns = r.turns[p];
      float cs[4], sn[4];
      if (pr.axis == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) phase((double)r.col0 + (double)(col + j), turns, cs + j, sn + j);
      } else {
        phase(times ? (double)times[bt] : (double)(bt % r.T), turns, cs, sn);
#pragma unroll
        for (int j = 1; j < 4; ++j) cs[j] = cs[0], sn[j] = sn[0];
      }
      const long long c1 = pr.first * HW + col, c2 = pr.second * HW + col;
      // (turns at most once: straight code for the two rows took 421 us where this takes 378)
      for (int y = row0 + down; y < row1; y += kRows * steps) {
        float a[kRows][4], b[kRows][4];
#pragma unroll
        for (int u = 0; u < kRows; ++u)
          if (y + u * steps < row1) {
            const long long at = (long long)(y + u * steps) * r.W;
            load_run<4>(src + c1 + at, cnt, a[u]);
            load_run<4>(src + c2 + at, cnt, b[u]);
          }
#pragma unroll
        for (int u = 0; u < kRows; ++u)
          if (y + u * steps < row1) {
            const long long at = (long long)(y + u * steps) * r.W;
            if (pr.axis == 1) {
              phase((double)r.row0 + (double)(y + u * steps), turns, cs, sn);
#pragma unroll
              for (int j = 1; j < 4; ++j) cs[j] = cs[0], sn[j] = sn[0];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float t = fmaf(a[u][j], cs[j], -(b[u][j] * sn[j]));
              b[u][j] = fmaf(a[u][j], sn[j], b[u][j] * cs[j]);
              a[u][j] = t;
            }
            put_run<WHOLE, 4>(dst + c1 + at, cnt, a[u]);
            put_run<WHOLE, 4>(dst + c2 + at, cnt, b[u]);
          }
      }
    }
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
  RotateGeo g;
  const int quads = (r.W + 3) / 4;
  g.heads = (long long)r.B * r.T * r.HD;
  g.units = r.Ch - r.total;
  g.quads = std::min(quads, 256);
  g.cols = (quads + 255) / 256;
  // rows at once: what leaves the fewest lanes of whole waves without a run
  // (38 runs a row: 3 rows on 128 lanes)
  g.steps = 1;
  int threads = (g.quads + 63) / 64 * 64;
  for (int n = 2; n * g.quads <= 128; ++n) {
    const int t = (n * g.quads + 63) / 64 * 64;
    if ((double)n * g.quads / t > (double)g.steps * g.quads / threads + 0.01) g.steps = n, threads = t;
  }
  g.rows = g.steps * kRows;
  g.chunks = (r.H + g.rows - 1) / g.rows;
  const dim3 grid((unsigned)((long long)g.chunks * g.cols), (unsigned)std::min(g.units, 1024),
                  (unsigned)std::min(g.heads * (k ? 2 : 1), 1024LL));
  const auto kernel = r.W % 32 == 0 ? rotate_kernel<true> : rotate_kernel<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, q, k, times, r, g, q_out, k_out);
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
