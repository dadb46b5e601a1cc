// cache.hip -- past frames held in 8 bits, and attention over their windows
// (snls_cache_store, snls_cache_attend, snls_cache_attend_points).
//
// A token is a pixel and head: its C/HD channels lie together as e4m3 codes,
// padded to whole 16-byte vectors, so one lane's 16-byte load is 16 channels.
// The scale of a block of pixels is a power of two: code * scale is exact in
// fp32, and so is the quotient that is rounded to a code.
//
// All cells of one query's window in one frame share the fraction (ay, ax) of
// the flow, so the (ws+1)^2 whole-pixel taps are scored once each and a cell's
// score is the bilinear sum of four tap scores; in the same way the softmax
// weights of the cells are folded onto the taps before the values are read.
#include "position_bias.h"

namespace snls {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------ store --

// Scale of a block whose largest finite magnitude is amax: the smallest power
// of two with amax <= 448 * scale (448 = 1.75 * 2^8), 1 for a block of zeros.
SNLS_DEV float block_scale(float amax) {
  if (amax == 0.f) return 1.f;
  const unsigned u = __float_as_uint(amax);
  int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);  // biased exponent of the scale
  e = max(e, 1);                                                     // 2^-126
  return __uint_as_float((unsigned)e << 23);
}

// Four values to four codes.  Magnitudes beyond 448 (infinities) are held as
// 448; NaN becomes the code of NaN.
SNLS_DEV unsigned encode4(float a, float b, float c, float d, float inv) {
  auto fit = [&](float x) {
    const float y = x * inv;
    return y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
  };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(fit(a), fit(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(fit(c), fit(d), w, true);
  return (unsigned)w;
}

// One workgroup = 256 pixels of one (video, head): a 16 x 16 block, or four
// 8 x 8 blocks side by side; one thread per pixel, its channels 16 at a time
// (read twice: for the largest magnitude, then for the codes).  blockIdx.y = 0
// stores keys, 1 values.
__global__ void __launch_bounds__(256) cache_store_kernel(const float* __restrict__ k, const float* __restrict__ v,
                                                          const int32_t* __restrict__ slots, CacheGeo c,
                                                          uint8_t* __restrict__ kc, float* __restrict__ ks,
                                                          uint8_t* __restrict__ vc, float* __restrict__ vs,
                                                          int tiles_x, int tiles_y) {
  __shared__ unsigned top[4];
  const int tiles = tiles_x * tiles_y;
  const int bh = (int)(blockIdx.x / (unsigned)tiles), tile = (int)(blockIdx.x % (unsigned)tiles);
  const int b = bh / c.HD, hd = bh % c.HD;
  const int slot = slots[b];
  if (slot < 0 || slot >= c.S) return;  // the whole workgroup
  const float* src = (blockIdx.y ? v : k) + ((long long)b * c.C + (long long)hd * c.Ch) * c.H * c.W;
  const long long img = ((long long)b * c.S + slot) * c.HD + hd;
  uint8_t* codes = (blockIdx.y ? vc : kc) + img * c.H * c.W * c.Cp;
  float* scales = (blockIdx.y ? vs : ks) + img * c.nby * c.nbx;
  const int tw = c.sh == 3 ? 32 : 16, th = 256 / tw;
  const int ly = threadIdx.x / tw, lx = threadIdx.x % tw;
  const int y = tile / tiles_x * th + ly, x = tile % tiles_x * tw + lx;
  const int sub = lx >> c.sh;  // block of this pixel within the workgroup
  const bool in = y < c.H && x < c.W;
  if (threadIdx.x < 4) top[threadIdx.x] = 0u;
  __syncthreads();
  const long long HW = (long long)c.H * c.W;
  const float* px = src + (in ? (long long)y * c.W + x : 0);
  float amax = 0.f;
  if (in)
    for (int ch = 0; ch < c.Ch; ++ch) {
      const float m = fabsf(px[ch * HW]);
      if (m < INFINITY) amax = fmaxf(amax, m);
    }
  atomicMax(&top[sub], __float_as_uint(amax));  // magnitudes order like their bits
  __syncthreads();
  const float scale = block_scale(__uint_as_float(top[sub]));
  if (!in) return;
  const float inv = 1.f / scale;  // exact; at most 2^126
  if ((ly & ((1 << c.sh) - 1)) == 0 && (lx & ((1 << c.sh) - 1)) == 0)
    scales[(y >> c.sh) * c.nbx + (x >> c.sh)] = scale;
  uint4* dst = reinterpret_cast<uint4*>(codes + ((long long)y * c.W + x) * c.Cp);
  for (int j = 0; j < c.nv; ++j) {
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = j * 16 + i < c.Ch ? px[(j * 16 + i) * HW] : 0.f;
    dst[j] = make_uint4(encode4(f[0], f[1], f[2], f[3], inv), encode4(f[4], f[5], f[6], f[7], inv),
                        encode4(f[8], f[9], f[10], f[11], inv), encode4(f[12], f[13], f[14], f[15], inv));
  }
}

snls_status launch_cache_store(const float* k, const float* v, const int32_t* slots, const CacheGeo& c,
                               uint8_t* k_codes, float* k_scales, uint8_t* v_codes, float* v_scales, hipStream_t s) {
  const int tw = c.sh == 3 ? 32 : 16, th = 256 / tw;
  const int tx = (c.W + tw - 1) / tw, ty = (c.H + th - 1) / th;
  // (fewer workgroups than pixels and heads, which fit 31 bits)
  hipLaunchKernelGGL(cache_store_kernel, dim3((unsigned)(c.B * c.HD * tx * ty), 2), dim3(256), 0, s, k, v, slots, c,
                     k_codes, k_scales, v_codes, v_scales, tx, ty);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

// ----------------------------------------------------------------- attend --

struct AttendArgs {
  const float* q;
  const int32_t* points;
  long long n;
  const float* flows;
  const int32_t* ages;
  const uint8_t* kc;
  const float* ks;
  const uint8_t* vc;
  const float* vs;
  const float* table;  // nullptr: no bias
  CacheGeo c;
  Bias bias;
  int ws;
  float scale;
  float* out;
};

// acc += dot of 16 codes with q (or, in spread16, acc[i] += w * code i).
SNLS_DEV float dot16(uint4 t, const float* q) {
  float s = 0.f;
  const unsigned w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    s = fmaf(a.x, q[4 * i], s);
    s = fmaf(a.y, q[4 * i + 1], s);
    s = fmaf(b.x, q[4 * i + 2], s);
    s = fmaf(b.y, q[4 * i + 3], s);
  }
  return s;
}
SNLS_DEV void spread16(uint4 t, float wgt, float* acc) {
  const unsigned w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    acc[4 * i] = fmaf(wgt, a.x, acc[4 * i]);
    acc[4 * i + 1] = fmaf(wgt, a.y, acc[4 * i + 1]);
    acc[4 * i + 2] = fmaf(wgt, b.x, acc[4 * i + 2]);
    acc[4 * i + 3] = fmaf(wgt, b.y, acc[4 * i + 3]);
  }
}

// A cell at whole-pixel position y, plus a fraction or not, has its centre in
// [0, n-1].
SNLS_DEV bool cell_ok(int y, bool frac, int n) { return y >= 0 && (frac ? y < n - 1 : y < n); }

// One query and head, SPLIT waves: wave i takes the slots i, i + SPLIT, ...;
// the waves' maxima, sums and outputs are joined in LDS.  Within a wave G
// lanes hold the channels of a token (16 each), 64 / G tokens are read at a
// time.
template <int G, int SPLIT>
__global__ void __launch_bounds__(64 * SPLIT) attend_wave_kernel(AttendArgs a) {
  constexpr int TP = 64 / G;            // tokens per step
  constexpr int NT = kMaxAttendWs + 1;  // taps per side at most
  constexpr int NC = (kMaxAttendWs * kMaxAttendWs + 63) / 64;
  __shared__ float taps_[SPLIT][NT * NT];
  __shared__ float cells_[SPLIT][(NT + 1) * (NT + 1)];  // softmax weights with a border of zeros
  __shared__ float join_acc[SPLIT][256];
  __shared__ float join_mz[SPLIT][2];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const CacheGeo& c = a.c;
  const long long qi = blockIdx.x / c.HD;
  const int hd = (int)(blockIdx.x % c.HD);
  const int ws = a.ws, nt = ws + 1, r = ws / 2, pitch = ws + 2;
  float* taps = taps_[wv];
  float* cells = cells_[wv];
  int b, h, w;
  const long long HW = (long long)c.H * c.W;
  if (a.points) {
    b = a.points[3 * qi];
    h = a.points[3 * qi + 1];
    w = a.points[3 * qi + 2];
  } else {
    b = (int)(qi / HW);
    const int pix = (int)(qi - b * HW);
    h = pix / c.W;
    w = pix - h * c.W;
  }
  const bool inb = b >= 0 && b < c.B && h >= 0 && h < c.H && w >= 0 && w < c.W;
  const int vec = lane & (G - 1), tok = lane / G;
  const bool vlive = vec < c.nv;
  float q[16], acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int ch = vec * 16 + i;
    q[i] = 0.f;
    acc[i] = 0.f;
    if (inb && ch < c.Ch) {
      const long long at = a.points ? qi * c.C + hd * c.Ch + ch
                                    : ((long long)b * c.C + hd * c.Ch + ch) * HW + (long long)h * c.W + w;
      q[i] = a.q[at];
    }
  }
  for (int i = lane; i < (ws + 2) * (ws + 2); i += 64) cells[i] = 0.f;
  float m = -INFINITY, z = 0.f;  // running maximum (of the wave) and this lane's sum
  if (inb)
    for (int s = wv; s < c.S; s += SPLIT) {
      const int age = a.ages[(long long)b * c.S + s];
      if (age < 0) continue;
      float Fh = 0.f, Fw = 0.f;
      if (a.flows) {
        const long long at = a.points ? (qi * c.S + s) * 2 : (((long long)b * c.S + s) * 2 * HW + (long long)h * c.W + w);
        Fh = a.flows[at];
        Fw = a.flows[at + (a.points ? 1 : HW)];
      }
      if (!(fabsf(Fh) < kFarDisp && fabsf(Fw) < kFarDisp)) continue;
      int nh, nw;
      float ay, ax;
      split_disp(Fh, &nh, &ay);
      split_disp(Fw, &nw, &ax);
      const int y0 = h + nh - r, x0 = w + nw - r;
      const long long img = ((long long)b * c.S + s) * c.HD + hd;
      const uint8_t* kp = a.kc + img * HW * c.Cp;
      const uint8_t* vp = a.vc + img * HW * c.Cp;
      const float* ksp = a.ks + img * c.nby * c.nbx;
      const float* vsp = a.vs + img * c.nby * c.nbx;
      // scores of the whole-pixel taps
      for (int t0 = 0; t0 < nt * nt; t0 += TP) {
        const int t = t0 + tok;
        const int ty = t / nt, y = y0 + ty, x = x0 + t - ty * nt;
        const bool in = t < nt * nt && y >= 0 && y < c.H && x >= 0 && x < c.W;
        float d = 0.f;
        if (in && vlive) {
          d = dot16(*reinterpret_cast<const uint4*>(kp + (unsigned)((y * c.W + x) * c.Cp + vec * 16)), q);
          d *= ksp[(y >> c.sh) * c.nbx + (x >> c.sh)];
        }
#pragma unroll
        for (int o = 1; o < G; o <<= 1) d += __shfl_xor(d, o);
        if (vec == 0 && t < nt * nt) taps[t] = d;
      }
      wave_lds_sync();
      // cells: logits, the new maximum, weights
      float lg[NC];
      float top = -INFINITY;
      const int bt = a.table ? bias_step_bucket(-age, a.bias) : 0;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int j = k * 64 + lane;
        lg[k] = -INFINITY;
        if (j < ws * ws) {
          const int dh = j / ws, dw = j - dh * ws;
          if (cell_ok(y0 + dh, ay != 0.f, c.H) && cell_ok(x0 + dw, ax != 0.f, c.W)) {
            const float* tp = taps + dh * nt + dw;
            const float up = (1.f - ax) * tp[0] + ax * tp[1], dn = (1.f - ax) * tp[nt] + ax * tp[nt + 1];
            float sc = (1.f - ay) * up + ay * dn;
            if (a.table) {
              const int at = (bt * a.bias.nb + bias_bucket(Fh + (float)(dh - r), a.bias)) * a.bias.nb +
                             bias_bucket(Fw + (float)(dw - r), a.bias);
              sc += a.table[(long long)hd * a.bias.buckets + at];
            }
            sc *= a.scale;
            if (isfinite(sc)) lg[k] = sc;
          }
        }
        top = fmaxf(top, lg[k]);
      }
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
      if (top == -INFINITY) {  // no cell counts (the whole wave)
        wave_lds_sync();
        continue;
      }
      const float m2 = fmaxf(m, top);
      const float f = m == -INFINITY ? 0.f : expf(m - m2);
      m = m2;
      z *= f;
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i] *= f;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int j = k * 64 + lane;
        if (j < ws * ws) {
          const int dh = j / ws, dw = j - dh * ws;
          const float p = lg[k] == -INFINITY ? 0.f : expf(lg[k] - m);
          z += p;
          cells[(dh + 1) * pitch + dw + 1] = p;
        }
      }
      wave_lds_sync();
      // values: the cells' weights folded onto the taps
      for (int t0 = 0; t0 < nt * nt; t0 += TP) {
        const int t = t0 + tok;
        const int ty = t / nt, tx = t - ty * nt, y = y0 + ty, x = x0 + tx;
        if (t < nt * nt && y >= 0 && y < c.H && x >= 0 && x < c.W && vlive) {
          const float* cp = cells + ty * pitch + tx;  // cells (ty-1, tx-1) .. (ty, tx)
          const float up = ax * cp[0] + (1.f - ax) * cp[1], dn = ax * cp[pitch] + (1.f - ax) * cp[pitch + 1];
          float wgt = ay * up + (1.f - ay) * dn;
          if (wgt != 0.f) {
            wgt *= vsp[(y >> c.sh) * c.nbx + (x >> c.sh)];
            spread16(*reinterpret_cast<const uint4*>(vp + (unsigned)((y * c.W + x) * c.Cp + vec * 16)), wgt, acc);
          }
        }
      }
      wave_lds_sync();
    }
  // the wave's sums
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) z += __shfl_xor(z, o);
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int o = G; o < 64; o <<= 1) acc[i] += __shfl_xor(acc[i], o);
  if (tok == 0)
#pragma unroll
    for (int i = 0; i < 16; ++i) join_acc[wv][vec * 16 + i] = acc[i];
  if (lane == 0) {
    join_mz[wv][0] = m;
    join_mz[wv][1] = z;
  }
  __syncthreads();
  for (int ch = threadIdx.x; ch < c.Ch; ch += 64 * SPLIT) {
    float M = -INFINITY, Z = 0.f, o = 0.f;
#pragma unroll
    for (int i = 0; i < SPLIT; ++i) M = fmaxf(M, join_mz[i][0]);
    if (M != -INFINITY)
#pragma unroll
      for (int i = 0; i < SPLIT; ++i)
        if (join_mz[i][0] != -INFINITY) {
          const float f = expf(join_mz[i][0] - M);
          Z += f * join_mz[i][1];
          o += f * join_acc[i][ch];
        }
    const long long at = a.points ? qi * c.C + hd * c.Ch + ch
                                  : ((long long)b * c.C + hd * c.Ch + ch) * HW + (long long)h * c.W + w;
    a.out[at] = Z > 0.f ? o / Z : 0.f;
  }
}

template <int SPLIT>
static void run_attend_wave(const AttendArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.n * a.c.HD)), block(64 * SPLIT);
  if (a.c.nv == 1)
    hipLaunchKernelGGL((attend_wave_kernel<1, SPLIT>), grid, block, 0, s, a);
  else if (a.c.nv == 2)
    hipLaunchKernelGGL((attend_wave_kernel<2, SPLIT>), grid, block, 0, s, a);
  else if (a.c.nv <= 4)
    hipLaunchKernelGGL((attend_wave_kernel<4, SPLIT>), grid, block, 0, s, a);
  else if (a.c.nv <= 8)
    hipLaunchKernelGGL((attend_wave_kernel<8, SPLIT>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((attend_wave_kernel<16, SPLIT>), grid, block, 0, s, a);
}

snls_status launch_cache_attend(const float* q, const int32_t* points, long long n, const float* flows,
                                const int32_t* ages, const uint8_t* k_codes, const float* k_scales,
                                const uint8_t* v_codes, const float* v_scales, const float* table,
                                const CacheGeo& c, const Bias& bias, int ws, float scale, float* out, hipStream_t s) {
  const AttendArgs a{q, points, n, flows, ages, k_codes, k_scales, v_codes, v_scales, table, c, bias, ws, scale, out};
  if (points)
    run_attend_wave<4>(a, s);
  else
    run_attend_wave<1>(a, s);
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
