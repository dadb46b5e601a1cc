// bias.hip -- learned bias of the neighbours' relative position: added to the
// scores (snls_bias), and the gradient of its table (snls_bias_backward).
//
// A neighbour's entry is table[hd, step, bucket(dh), bucket(dw)].  Both
// directions read 16 or 20 bytes a neighbour and write 4 or (almost) nothing,
// so memory bandwidth bounds them.  The scores of one image -- one head of one
// query frame, nH * nW * k of them -- lie together and share the query frame
// and the head's table; they are walked in chunks of 256 per wave, four
// consecutive neighbours a lane, in 16-byte reads.
#include "position_bias.h"

namespace snls {

constexpr int kChunk = 256;  // neighbours a wave takes at a time

struct BiasRows {
  long long per_image;  // scores of an image
  long long chunks;     // of an image
  int B, T, HD;
};

static BiasRows bias_rows(const Geo& g) {
  const long long n = (long long)g.nH * g.nW * (g.k > 0 ? g.k : g.ncand);
  return {n, (n + kChunk - 1) / kChunk, g.B, g.T, g.HD};
}

// Four floats at any 4-byte address.
struct __attribute__((packed, aligned(4))) Float4 {
  float x, y, z, w;
};

// A lane's four neighbours: flat buckets, -1 for one that contributes nothing
// to the aggregation.  cnt: how many of them there are (4 but at an image's
// end, where they are read one by one).
struct Quartet {
  float ind[12];
  SNLS_DEV void load(const float* __restrict__ inds, int cnt) {
    if (cnt == 4) {
      const Float4* p = reinterpret_cast<const Float4*>(inds);
      const Float4 a = p[0], b = p[1], c = p[2];
      ind[0] = a.x, ind[1] = a.y, ind[2] = a.z, ind[3] = a.w;
      ind[4] = b.x, ind[5] = b.y, ind[6] = b.z, ind[7] = b.w;
      ind[8] = c.x, ind[9] = c.y, ind[10] = c.z, ind[11] = c.w;
    } else {
#pragma unroll
      for (int i = 0; i < 12; ++i) ind[i] = i < 3 * cnt ? inds[i] : -1.f;
    }
  }
  SNLS_DEV int bucket(int i, int t, int T, const Bias& b) const {
    const float frame = ind[3 * i], dh = ind[3 * i + 1], dw = ind[3 * i + 2];
    const bool ok = frame >= 0.f && frame < (float)T && frame == floorf(frame) && fabsf(dh) < kFarDisp &&
                    fabsf(dw) < kFarDisp;
    const int at = (bias_step_bucket((int)frame - t, b) * b.nb + bias_bucket(dh, b)) * b.nb + bias_bucket(dw, b);
    return ok ? at : -1;
  }
};

SNLS_DEV void load4(const float* p, int cnt, float* to) {
  if (cnt == 4) {
    const Float4 a = *reinterpret_cast<const Float4*>(p);
    to[0] = a.x, to[1] = a.y, to[2] = a.z, to[3] = a.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = i < cnt ? p[i] : 0.f;
  }
}

// A workgroup takes `run` chunks of one image per wave.
__global__ void __launch_bounds__(256) bias_kernel(const float* dists, const float* __restrict__ inds,
                                                   const float* __restrict__ table, BiasRows r, Bias b, float sign,
                                                   int run, unsigned groups, float* out) {
  extern __shared__ float tab[];
  const long long img = blockIdx.x / groups;
  const int t = (int)(img % r.T), hd = (int)(img / r.T % r.HD);
  for (int i = threadIdx.x; i < b.buckets; i += 256) tab[i] = sign * table[(long long)hd * b.buckets + i];
  __syncthreads();
  const long long base = img * r.per_image;
  const long long first = ((long long)(blockIdx.x % groups) * 4 + (threadIdx.x >> 6)) * run;
  for (int c = 0; c < run; ++c) {
    const long long i = (first + c) * kChunk + (threadIdx.x & 63) * 4;
    if (i >= r.per_image) return;
    const int cnt = (int)min(4LL, r.per_image - i);
    const long long n = base + i;
    float d[4];
    Quartet q;
    load4(dists + n, cnt, d);
    q.load(inds + 3 * n, cnt);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = q.bucket(j, t, r.T, b);
      const float x = d[j] + tab[max(at, 0)];
      d[j] = at >= 0 && fabsf(d[j]) < INFINITY ? x : d[j];
    }
    if (cnt == 4) {
      *reinterpret_cast<Float4*>(out + n) = Float4{d[0], d[1], d[2], d[3]};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < cnt) out[n + j] = d[j];
    }
  }
}

// One wave per slice of a head's chunks, with a table of partial sums of its
// own in LDS: 64-bit additions, which LDS performs in hardware (fp32 atomics
// take 180 cycles an instruction on this chip, fp64 10 to 13, a read and a
// write 25), `cols` copies of every entry so that fewer lanes meet.  No other
// wave touches the table, so every entry's additions happen in one order.
// NW waves a workgroup join their tables in LDS, in order, and write one: its
// sums stay in 64 bits to the end, twice the bytes of fp32 ones, which lost
// the last places where the slices cancel and all of a sum whose slices pass
// fp32's range (31 million gradients into 4 tables of 1,183: 149 us a call,
// 157 with a 64-bit table per wave, 150 with an fp32 one).
template <int NW>
__global__ void __launch_bounds__(64 * NW) bias_grad_kernel(const float* __restrict__ grad,
                                                            const float* __restrict__ dists,
                                                            const float* __restrict__ inds, BiasRows r, Bias b,
                                                            float sign, int cols, int groups,
                                                            double* __restrict__ part) {
  extern __shared__ double tables[];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int hd = blockIdx.x / groups, slices = groups * NW, slice = (int)(blockIdx.x % groups) * NW + wv;
  double* const acc = tables + wv * b.buckets * cols;
  for (int i = lane; i < b.buckets * cols; i += 64) acc[i] = 0.0;
  wave_lds_sync();
  const long long total = (long long)r.B * r.T * r.chunks;  // of this head
  const long long c1 = total * (slice + 1) / slices;
  const int col = lane & (cols - 1);
  for (long long c = total * slice / slices; c < c1; ++c) {
    const long long bt = c / r.chunks, i = (c - bt * r.chunks) * kChunk + lane * 4;
    const int t = (int)(bt % r.T), cnt = (int)min(4LL, max(0LL, r.per_image - i));
    const long long n = ((bt / r.T * r.HD + hd) * r.T + t) * r.per_image + i;
    if (cnt > 0) {
      float d[4], gv[4];
      Quartet q;
      load4(grad + n, cnt, gv);
      load4(dists + n, cnt, d);
      q.load(inds + 3 * n, cnt);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = q.bucket(j, t, r.T, b);
        if (at >= 0 && fabsf(d[j]) < INFINITY) unsafeAtomicAdd(acc + at * cols + col, (double)(sign * gv[j]));
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < b.buckets; i += 64 * NW) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < NW; ++w)
      for (int k = 0; k < cols; ++k) s += tables[(w * b.buckets + i) * cols + k];
    part[(long long)blockIdx.x * b.buckets + i] = s;
  }
}

// grad_table[hd][i] = sum of the head's `slices` tables, in 64 bits: `ent`
// entries (a power of two up to 64) of a head a workgroup, its 1024 / ent
// groups of lanes take the tables in turn.
__global__ void __launch_bounds__(1024) bias_grad_sum_kernel(const double* __restrict__ part, int buckets, int slices,
                                                             int ent, float* __restrict__ grad_table) {
  __shared__ double sums[1024];
  const int lane = threadIdx.x & (ent - 1), group = threadIdx.x / ent, groups = 1024 / ent;
  const int per = (buckets + ent - 1) / ent, hd = blockIdx.x / per, i = (int)(blockIdx.x % per) * ent + lane;
  double s = 0.0;
  if (i < buckets) {
    const double* p = part + (long long)hd * slices * buckets + i;
#pragma unroll 8
    for (int k = group; k < slices; k += groups) s += p[(long long)k * buckets];
  }
  sums[threadIdx.x] = s;
  __syncthreads();
  for (int half = groups / 2; half > 0; half /= 2) {
    if (group < half) sums[threadIdx.x] += sums[threadIdx.x + half * ent];
    __syncthreads();
  }
  if (group == 0 && i < buckets) grad_table[(long long)hd * buckets + i] = (float)sums[lane];
}

// Slices of a head: as many waves as lie on the chip at once with their tables
// (16 a CU up to 1,280 entries: 31 million gradients into 4 tables of 1,183
// took 215 us with 8 a CU, 142 with 16, 178 with 24, which do not fit), and
// four chunks a slice at least.  Where 16 tables fit, four waves share a
// workgroup; larger ones keep a workgroup each, whose launches fill LDS.
constexpr int kCUs = 256, kLds = 160 * 1024, kMostWaves = 16;

static long long bias_slices(const Geo& g, int buckets) {
  const BiasRows r = bias_rows(g);
  const long long want = ((long long)g.B * g.T * r.chunks + 3) / 4;
  const int fit = kLds / (buckets * (int)sizeof(double));
  const long long most = kCUs * (fit < kMostWaves ? fit : kMostWaves) / g.HD;
  return want < most ? want : most > 1 ? most : 1;
}

// slices * buckets is largest where the tables fill LDS
size_t bias_backward_ws_bytes(const Geo& g) {
  const size_t heads = (size_t)g.HD * SNLS_BIAS_MAX_BUCKETS, full = (size_t)kCUs * (kLds / sizeof(double));
  const size_t few = heads * bias_slices(g, 1);
  const size_t most = heads > full ? heads : full;
  return (few < most ? few : most) * sizeof(double);
}

snls_status launch_bias(const float* dists, const float* inds, const float* table, const Geo& g, const Bias& bias,
                        float* out, hipStream_t s) {
  const BiasRows r = bias_rows(g);
  const long long images = (long long)g.B * g.HD * g.T;
  // chunks a wave takes: enough workgroups for the chip, few copies of the table
  long long run = images * r.chunks / (4 * 8192);
  run = run < 1 ? 1 : run > 16 ? 16 : run;
  const long long groups = (r.chunks + 4 * run - 1) / (4 * run);
  if (images * groups >= 1LL << 24) return SNLS_ERR_UNSUPPORTED;  // a launch holds less than 2^32 threads
  hipLaunchKernelGGL(bias_kernel, dim3((unsigned)(images * groups)), dim3(256), bias.buckets * sizeof(float), s, dists,
                     inds, table, r, bias, g.dist == SNLS_DIST_PROD ? 1.f : -1.f, (int)run, (unsigned)groups, out);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

snls_status launch_bias_backward(const float* grad, const float* dists, const float* inds, const Geo& g,
                                 const Bias& bias, float* grad_table, double* ws, hipStream_t s) {
  const bool four = bias.buckets * (int)sizeof(double) <= kLds / kMostWaves;
  const int slices = (int)bias_slices(g, bias.buckets), groups = four ? (slices + 3) / 4 : slices;
  // entries a workgroup of the second kernel: few while the table is small and
  // workgroups short (a whole call with 16 / 64, a table a wave: 2 tables of 75
  // 21.0 / 22.4 us, 4 of 1,183 141 / 138)
  const int ent = bias.buckets <= 256 ? 16 : 64, sums = (bias.buckets + ent - 1) / ent * g.HD;  // at most 64 a head
  int cols = 8;  // as many copies as leave room for all the waves
  while (cols > 1 && bias.buckets * cols * (int)sizeof(double) > kLds / kMostWaves) cols /= 2;
  const size_t lds = (size_t)bias.buckets * cols * sizeof(double);
  const float sign = g.dist == SNLS_DIST_PROD ? 1.f : -1.f;
  const dim3 grid((unsigned)(g.HD * groups));
  if (four)
    hipLaunchKernelGGL(bias_grad_kernel<4>, grid, dim3(256), 4 * lds, s, grad, dists, inds, bias_rows(g), bias, sign,
                       cols, groups, ws);
  else
    hipLaunchKernelGGL(bias_grad_kernel<1>, grid, dim3(64), lds, s, grad, dists, inds, bias_rows(g), bias, sign, cols,
                       groups, ws);
  hipLaunchKernelGGL(bias_grad_sum_kernel, dim3((unsigned)sums), dim3(1024), 0, s, ws, bias.buckets, groups, ent,
                     grad_table);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
