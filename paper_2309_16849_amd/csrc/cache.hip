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
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

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
// 8 x 8 blocks side by side; one thread per pixel.  The channels (up to NV * 16)
// stay in registers between the largest magnitude and the codes; read a second
// time instead, 128 channels at 480 x 854 take 286 us, not 144, 256 take 579,
// not 334 (at one wave a SIMD), 64 take 150, not 68.  Bound by memory: 3.9 TB/s
// at 64 channels, 3.6 at 128, 3.1 at 256, four fifths of it reads, where a large
// copy has 5.0 and the position bias, of the same mix, 5.3.  blockIdx.y = 0
// stores keys, 1 values.
template <int NV>
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
  const long long HW = (long long)c.H * c.W;
  const float* src = (blockIdx.y ? v : k) + ((long long)b * c.C + (long long)hd * c.Ch) * HW;
  const long long img = ((long long)b * c.S + slot) * c.HD + hd;
  uint8_t* codes = (blockIdx.y ? vc : kc) + img * HW * c.Cp;
  float* scales = (blockIdx.y ? vs : ks) + img * c.nby * c.nbx;
  const int tw = c.sh == 3 ? 32 : 16, th = 256 / tw;
  const int ly = threadIdx.x / tw, lx = threadIdx.x % tw;
  const int y = tile / tiles_x * th + ly, x = tile % tiles_x * tw + lx;
  const bool in = y < c.H && x < c.W;
  if (threadIdx.x < 4) top[threadIdx.x] = 0u;
  __syncthreads();
  const float* px = src + (in ? (long long)y * c.W + x : 0);
  float val[NV * 16];
  float amax = 0.f;
#pragma unroll
  for (int ch = 0; ch < NV * 16; ++ch) val[ch] = in && ch < c.Ch ? px[ch * HW] : 0.f;
#pragma unroll
  for (int ch = 0; ch < NV * 16; ++ch) {
    const float m = fabsf(val[ch]);
    amax = m < INFINITY ? fmaxf(amax, m) : amax;
  }
  // over the block's row in this wave, then over the workgroup (magnitudes order like their bits)
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  if ((lx & 7) == 0) atomicMax(&top[lx >> c.sh], __float_as_uint(amax));
  __syncthreads();
  const float scale = block_scale(__uint_as_float(top[lx >> c.sh]));
  if (!in) return;
  const float inv = 1.f / scale;  // exact; at most 2^126
  const int mask = (1 << c.sh) - 1;
  if ((ly & mask) == 0 && (lx & mask) == 0) scales[(y >> c.sh) * c.nbx + (x >> c.sh)] = scale;
  uint4* dst = reinterpret_cast<uint4*>(codes + ((long long)y * c.W + x) * c.Cp);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const float* f = val + 16 * j;
    if (j < c.nv)
      dst[j] = make_uint4(encode4(f[0], f[1], f[2], f[3], inv), encode4(f[4], f[5], f[6], f[7], inv),
                          encode4(f[8], f[9], f[10], f[11], inv), encode4(f[12], f[13], f[14], f[15], inv));
  }
}

snls_status launch_cache_store(const float* k, const float* v, const int32_t* slots, const CacheGeo& c,
                               uint8_t* k_codes, float* k_scales, uint8_t* v_codes, float* v_scales, hipStream_t s) {
  const int tw = c.sh == 3 ? 32 : 16, th = 256 / tw;
  const int tx = (c.W + tw - 1) / tw, ty = (c.H + th - 1) / th;
  // (one thread per pixel and head of the padded frame, which fit 30 bits)
  const dim3 grid((unsigned)(c.B * c.HD * tx * ty), 2);
#define SNLS_STORE(NV)                                                                                        \
  hipLaunchKernelGGL(cache_store_kernel<NV>, grid, dim3(256), 0, s, k, v, slots, c, k_codes, k_scales, v_codes, \
                     v_scales, tx, ty)
  switch (c.nv) {
    case 1: SNLS_STORE(1); break;
    case 2: SNLS_STORE(2); break;
    case 3: SNLS_STORE(3); break;
    case 4: SNLS_STORE(4); break;
    case 5: case 6: SNLS_STORE(6); break;
    case 7: case 8: SNLS_STORE(8); break;
    case 9: case 10: case 11: case 12: SNLS_STORE(12); break;
    default: SNLS_STORE(16); break;
  }
#undef SNLS_STORE
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
  float scale;  // of the table
  float sm;     // scale = sm * 2^se, |sm| in [0.5, 1) or 0
  int se;
  float* out;
};

// The range of scores.  A query's channels are brought to 2^kQTop by a power of
// two of the query's own, and that, the scale's and the block scale's meet in
// one factor per tap: neither scale * q nor q * code, nor a sum of these, leaves
// fp32 where the logit does not (channels below 2^-91 of a query's largest
// against keys of 2^100 aside).  Queries as they are, times the scale, lost
// logits of ordinary size for queries from 1e33 on.
constexpr int kQTop = 100;  // 256 products with codes of up to 448 stay below 2^118
// e of the largest magnitude, in [2^e, 2^(e+1)), or 0.  (Infinities need no care: no logit of such a query is finite.)
SNLS_DEV int exponent(float most) { return __builtin_amdgcn_frexp_expf(most) - 1; }
SNLS_DEV float key_factor(float scale, int e) {
  const float f = ldexpf(scale, e);
  return f > 3.402823466e38f ? 3.402823466e38f : f;  // (0 times it stays 0; NaN stays NaN)
}

// s plus the dot product of 16 codes with q; spread16: acc[i] += wgt * code i.
SNLS_DEV float dot16(uint4 t, const float* q, float s) {
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

// A sum of weighted values when the softmax's maximum rises and its weights
// fall by f.  A factor of 0 takes the values out, NaN among them: a value of
// weight 0 is not read either where the maximum was known before.
SNLS_DEV float faded(float x, float f) { return f == 0.f ? 0.f : x * f; }

// A cell at whole-pixel position y, plus a fraction or not, has its centre in
// [0, n-1].
SNLS_DEV bool cell_ok(int y, bool frac, int n) { return y >= 0 && (frac ? y < n - 1 : y < n); }

// One listed query and head, SPLIT waves: wave i takes the slots i, i + SPLIT, ...;
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
  const int b = a.points[3 * qi], h = a.points[3 * qi + 1], w = a.points[3 * qi + 2];
  const long long HW = (long long)c.H * c.W;
  const bool inb = b >= 0 && b < c.B && h >= 0 && h < c.H && w >= 0 && w < c.W;
  const int vec = lane & (G - 1), tok = lane / G;
  const bool vlive = vec < c.nv;
  float q[16], acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int ch = vec * 16 + i;
    q[i] = 0.f;
    acc[i] = 0.f;
    if (ch < c.Ch) q[i] = a.q[qi * c.C + hd * c.Ch + ch];  // (under way beside the point itself, inside or not)
  }
  // As much of the powers of two of query and scale as fits goes to q: all of it but at fp32's ends, where the cells get
  // the rest; what leaves fp32 before that leaves it with the rest too.
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(q[i]));
#pragma unroll
  for (int o = 1; o < G; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
  const int eq = exponent(most), top = min(max(eq + a.se, -60), kQTop);
  const int rest = __builtin_amdgcn_readfirstlane(eq + a.se - top);  // one query and head a wave
#pragma unroll
  for (int i = 0; i < 16; ++i) q[i] = ldexpf(q[i], top - eq) * a.sm;
  for (int i = lane; i < (ws + 2) * (ws + 2); i += 64) cells[i] = 0.f;
  float m = -INFINITY, z = 0.f;  // running maximum (of the wave) and this lane's sum
  if (inb)
    for (int s = wv; s < c.S; s += SPLIT) {
      const int age = a.ages[(long long)b * c.S + s];
      if (age < 0) continue;
      float Fh = 0.f, Fw = 0.f;
      if (a.flows) {
        Fh = a.flows[(qi * c.S + s) * 2];
        Fw = a.flows[(qi * c.S + s) * 2 + 1];
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
          d = dot16(*reinterpret_cast<const uint4*>(kp + (unsigned)((y * c.W + x) * c.Cp + vec * 16)), q, 0.f);
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
            float sc = ldexpf((1.f - ay) * up + ay * dn, rest);
            if (a.table) {
              const int at = (bt * a.bias.nb + bias_bucket(Fh + (float)(dh - r), a.bias)) * a.bias.nb +
                             bias_bucket(Fw + (float)(dw - r), a.bias);
              sc += a.scale * a.table[(long long)hd * a.bias.buckets + at];
            }
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
      for (int i = 0; i < 16; ++i) acc[i] = faded(acc[i], f);
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
          o += faded(join_acc[i][ch], f);
        }
    a.out[qi * c.C + hd * c.Ch + ch] = Z > 0.f ? o / Z : 0.f;
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

// --- four lanes per query ---
//
// Sixteen queries per wave.  The four lanes of a query read 64 consecutive
// bytes of a tap row at a time: R lanes hold the channels of a token, 16 * V
// each, and 4 / R tokens are read at once.  Whatever R, lane l ends up with
// the scores of the tap columns l, l + 4, ... and computes the cells of these
// columns; neighbouring columns are exchanged through DPP.  The rows of taps
// stream by: key row i completes cell row i - 1, whose weights complete the
// taps of value row i - 1; the softmax's maximum is a running one, so nothing
// but two rows is kept.
//
// Logits are held in base 2 (q and the table are multiplied by scale * log2 e
// as they are read: one rounding more per channel and entry, in place of one
// per cell, and the hardware's base-2 exponential, 1 ulp, in place of expf).
// The maximum follows the logits only in steps of more than kSlack, so that the
// outputs are rescaled once or twice per frame, not per row: weights are then at
// most 2^kSlack, far from fp32's limits.
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kSlack = 12.f;
// Loads of a tap row (K * R * V) up to which they stand together, the values'
// beside the keys', a row's arithmetic ahead of their use (4 heads of 16
// channels at 256 x 256 0.74 -> 0.70 ms, 64 channels at 480 x 854 1.53 -> 1.41
// ms); more would take the registers of half the waves.  Wider heads issue the
// loads of one column group (R * V) at a time (96 channels at 160 x 160 with 3
// slots 308 -> 193 us), and above 128 channels two waves a SIMD are worth some
// spilled registers (192 channels 440 -> 276 us).
constexpr int kTogether = 12;

// Keeps a loaded value from being read again, later, inside a branch.
SNLS_DEV void pin(uint4& t) { asm volatile("" : "+v"(t.x), "+v"(t.y), "+v"(t.z), "+v"(t.w)); }

// Lane i of each quad gets the value of lane P_i.
template <int P0, int P1, int P2, int P3>
SNLS_DEV float quad(float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(
      0, (int)__float_as_uint(v), P0 | (P1 << 2) | (P2 << 4) | (P3 << 6), 0xf, 0xf, true));
}

// A finite table entry stays finite in base 2 (a mask of the lowest value is
// no mask of -inf).
SNLS_DEV float table_base2(float t, float scale) {
  const float x = t * scale;
  return fabsf(x) < INFINITY ? fminf(fmaxf(x * kLog2e, -3.402823466e38f), 3.402823466e38f) : x;
}

// MX: scores from the matrix cores (heads of 17 to 128 channels; 64 channels at
// 480 x 854, 3 slots, 1.03 -> 0.78 ms, two heads of 32 at 256 x 256 0.23 -> 0.20).
// The windows of a wave's 16 queries overlap, so the box around them in a
// slot's frame is walked in tiles of 16 tokens, v_mfma_f32_16x16x32_f16 with
// tokens as rows and queries as columns, and each query's own taps of the
// product go to LDS, from where the rows of taps are read.  Codes are exact in
// fp16; q is split in two fp16 parts that hold 22 bits of a query's largest
// channel (scaled by a power of two per query): outputs are 3.9e-7 of the values
// off 64 bits on the 480 x 854 frame, plain fp32 1.7e-7; all 24 bits would be
// three parts and half as many products again.  A box is some four times a window
// (offsets carry an error of pixels), the matrix cores 30 times as fast as the
// vector units on such a product.  Where the box would be larger than the 16
// windows are together (offsets that differ by tens of pixels between
// neighbours), every window is a box of its own.  64 channels at 200 x 240, 3
// slots: equal offsets 104 us, neighbours' offsets 1 / 3 / 10 / 40 pixels apart
// 118 / 139 / 263 / 276, the vector units 144 to 157; the vector units' form as a
// second branch was faster at 40 pixels (204, not 275), but took 7% at 0, for its
// registers.
template <int CT>
constexpr int kBoxPitch = CT + 6;  // a row of taps with the three beside it that a group of four tokens may bring
template <int CT>
constexpr int kBoxQuery = CT * kBoxPitch<CT> + 1;  // floats of a query (odd: queries fall on different banks)

// 8 codes as fp16.
SNLS_DEV half8_t codes_f16(unsigned a, unsigned b) {
  const half2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.f, false);
  const half2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.f, true);
  const half2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.f, false);
  const half2_t p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.f, true);
  return half8_t{p0.x, p0.y, p1.x, p1.y, p2.x, p2.y, p3.x, p3.y};
}

// The loads of a tap row stand together, with no branch between them, so that
// they are under way at the same time: CT columns of taps are read whatever ws
// is (those past the window at the clamped address, unused).
//
// split (1, 2 or 4) waves share 16 queries, each takes every split-th slot,
// and the first joins their maxima, sums and outputs through LDS: for calls
// whose queries alone are too few waves for the chip.
// Waves a SIMD that the registers are held to (160 x 160 to 480 x 854, ws = 9):
// with the matrix cores 3 for heads up to 64 channels (64 channels 1.32 -> 1.08
// ms at 480 x 854, 48 channels 151 -> 132 us at 200 x 240; 4 spill), without
// them what the compiler takes (3 at 16 channels; 4 cost 1 to 7%), but 2 from
// two vectors a lane on: a register or two more leave one wave (6,000 points of
// 128 channels 120 us, not 94).
constexpr int attend_waves(int CT, int R, int V, bool MX) {
  if (MX && (V == 1 || (R == 1 && CT <= 10))) return 3;
  return V >= 2 ? 2 : 1;
}
template <int CT, int R, int V, bool POINTS, bool MX>
__global__ void __launch_bounds__(256, attend_waves(CT, R, V, MX)) attend_quad_kernel(AttendArgs a, int tiles_x, int tiles_y, int split) {
  static_assert(!(MX && POINTS), "boxes lie around neighbouring pixels");
  constexpr int K = (CT + 3) / 4;
  extern __shared__ float lds[];  // row buckets of the four waves' queries, the head's bias table, the boxes' scores
  const CacheGeo& c = a.c;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int l = lane & 3, sub = lane >> 2;
  const int groups = 4 / split, group = wv / split, part_of = wv % split;  // of 16 queries; of the slots
  const int ws = a.ws, r = ws / 2;
  const long long HW = (long long)c.H * c.W;
  // the wave's queries: 8 x 2 pixels of the workgroup's tile, or 16 listed points
  int b, hd, h, w, h0 = 0, w0 = 0;
  long long qi = 0;
  bool live;
  if constexpr (POINTS) {
    const long long blocks = (a.n + groups * 16 - 1) / (groups * 16);
    hd = (int)(blockIdx.x / blocks);
    qi = (blockIdx.x - hd * blocks) * (groups * 16) + group * 16 + sub;
    live = qi < a.n;
    if (!live) qi = a.n - 1;
    b = a.points[3 * qi];
    h = a.points[3 * qi + 1];
    w = a.points[3 * qi + 2];
  } else {
    // consecutive workgroups land on different XCDs: each XCD takes a
    // contiguous run of tiles, ordered in strips of 8 tiles, whose windows fit its L2
    const int tiles = tiles_x * tiles_y, total = tiles * c.B * c.HD, per = (total + 7) / 8;
    const int id = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (id >= total || (int)(blockIdx.x >> 3) >= per) return;  // the whole workgroup
    const int img = id / tiles, tile = id % tiles;
    b = img / c.HD;
    hd = img % c.HD;
    const int strip = tile / (8 * tiles_y), rest = tile % (8 * tiles_y), width = min(8, tiles_x - strip * 8);
    h0 = (rest / width * groups + group) * 2;
    w0 = (strip * 8 + rest % width) * 8;
    h = h0 + (sub >> 3);
    w = w0 + (sub & 7);
    live = h < c.H && w < c.W;
  }
  const bool stored = live;  // has a row of out
  if constexpr (POINTS) {
    live = live && b >= 0 && b < c.B && h >= 0 && h < c.H && w >= 0 && w < c.W;
    if (!live) b = 0;  // (without points b is uniform, and so are the addresses of the planes)
  }
  if (!live) h = w = 0;
  int* rowb = reinterpret_cast<int*>(lds) + threadIdx.x / 4 * 16;  // of this query: table row per tap row
  float* tab = lds + 64 * 16;
  for (int i = threadIdx.x; i < max(a.bias.buckets, 1); i += 256)
    tab[i] = a.table ? table_base2(a.table[(long long)hd * a.bias.buckets + i], a.scale) : 0.f;
  __syncthreads();
  const int lr = l & (R - 1);  // this lane's part of a token
  float q[MX ? 1 : V][16], acc[V][16];
  int voff[V];  // byte offset of the lane's vector v from its first
#pragma unroll
  for (int v = 0; v < V; ++v) {
    voff[v] = v * R + lr < c.nv ? v * R * 16 : 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int ch = (v * R + lr) * 16 + i;
      acc[v][i] = 0.f;
      if constexpr (!MX) q[v][i] = 0.f;
      if (!MX && live && ch < c.Ch)
        q[MX ? 0 : v][i] = POINTS ? a.q[qi * c.C + hd * c.Ch + ch]
                                  : a.q[((long long)b * c.C + hd * c.Ch + ch) * HW + (long long)h * c.W + w];
    }
  }
  int qexp = 0;  // undoes the query's power of two, and holds the scale's
  if constexpr (!MX) {
    float most = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(q[v][i]));
    most = fmaxf(most, quad<1, 0, 3, 2>(most));
    most = fmaxf(most, quad<2, 3, 0, 1>(most));
    const int up = kQTop - exponent(most);
    qexp = a.se - up;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 16; ++i) q[v][i] = ldexpf(q[v][i], up) * (a.sm * kLog2e);
  }
  const int lane0 = min(lr, c.nv - 1) * 16, rowbytes = c.W * c.Cp;
  // Matrix-core operand of query lane % 16: lanes of group lane / 16 hold the
  // channels of vector 4 j + group, its first and its second eight; with two
  // vectors the upper groups hold the low parts of the same channels instead.
  constexpr bool kPack = R * V == 2;
  constexpr int J = (R * V + 3) / 4;
  half8_t qh[MX ? J : 1][2], ql[MX && !kPack ? J : 1][2];
  const int n16 = lane & 15, g4 = lane >> 4;
  float* const stab = tab + max(a.bias.buckets, 1) + wv * 16 * kBoxQuery<CT>;
  if constexpr (MX) {
    const int hn = h0 + (n16 >> 3), wn = w0 + (n16 & 7);
    const bool inq = hn < c.H && wn < c.W;
    const float* qp = a.q + ((long long)b * c.C + hd * c.Ch) * HW + (inq ? (long long)hn * c.W + wn : 0);
    float x[J][16], most = 0.f;
#pragma unroll
    for (int jj = 0; jj < J; ++jj)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int ch = (kPack ? (g4 & 1) : 4 * jj + g4) * 16 + i;
        x[jj][i] = inq && ch < c.Ch ? qp[ch * HW] : 0.f;
        most = fmaxf(most, fabsf(x[jj][i]));
      }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // the largest channel to 2^14 .. 2^15, times 0.72 .. 1.45 just below fp16's end: channels 2^-14 of it still have all
    // of both parts
    const int up = 14 - exponent(most);
    qexp = a.se - up;
#pragma unroll
    for (int jj = 0; jj < J; ++jj)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float t = ldexpf(x[jj][i], up) * (a.sm * kLog2e);
        // one number for both parts: folded into the conversion the product may round to another hi than lo is the rest of
        asm volatile("" : "+v"(t));
        const _Float16 hi = (_Float16)t, lo = (_Float16)(t - (float)hi);
        if constexpr (kPack) {
          qh[jj][i / 8][i % 8] = g4 < 2 ? hi : lo;
        } else {
          qh[jj][i / 8][i % 8] = hi;
          ql[jj][i / 8][i % 8] = lo;
        }
      }
  }
  float m = -INFINITY, z = 0.f;
  for (int s = part_of; s < c.S; s += split) {
    const int age = a.ages[(long long)b * c.S + s];
    if (!POINTS && age < 0) continue;
    float Fh = 0.f, Fw = 0.f;
    if (a.flows) {
      const long long at = POINTS ? (qi * c.S + s) * 2 : (((long long)b * c.S + s) * 2 * HW + (long long)h * c.W + w);
      Fh = a.flows[at];
      Fw = a.flows[at + (POINTS ? 1 : HW)];
    }
    const bool on = live && age >= 0 && fabsf(Fh) < kFarDisp && fabsf(Fw) < kFarDisp;
    if (!__any(on)) continue;
    if (!on) Fh = Fw = 0.f;
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
    if constexpr (MX) {
      int ymin = on ? y0 : INT_MAX, ymax = on ? y0 : INT_MIN, xmin = on ? x0 : INT_MAX, xmax = on ? x0 : INT_MIN;
#pragma unroll
      for (int o = 4; o < 64; o <<= 1) {
        ymin = min(ymin, __shfl_xor(ymin, o));
        ymax = max(ymax, __shfl_xor(ymax, o));
        xmin = min(xmin, __shfl_xor(xmin, o));
        xmax = max(xmax, __shfl_xor(xmax, o));
      }
      const int yq = __shfl(y0, n16 * 4), xq = __shfl(x0, n16 * 4);  // window of query n16
      float* const sq = stab + n16 * kBoxQuery<CT>;
      // the box of the first taps ya .. yb, xa .. xb, clipped to the frame, in groups of four tokens that share a block
      auto walk = [&](int ya_, int yb_, int xa_, int xb_, bool test) {
        const int ry0 = __builtin_amdgcn_readfirstlane(min(max(ya_, 0), c.H - 1));
        const int ry1 = __builtin_amdgcn_readfirstlane(min(max(yb_ + ws, 0), c.H - 1));
        const int rx0 = __builtin_amdgcn_readfirstlane(min(max(xa_, 0), c.W - 1)) & ~3;
        const int rx1 = __builtin_amdgcn_readfirstlane(min(max(xb_ + ws, 0), c.W - 1));
        const int gw = (rx1 - rx0) / 4 + 1;
        const long long ng = (long long)(ry1 - ry0 + 1) * gw;
        if (test && ng > 16 * (ws + 1) * ((ws + 7) / 4)) return false;
        const int pairs = ((int)ng + 7) / 8;  // of tiles
        const int dq = 4 / gw, dr = 4 % gw;   // groups of a tile: rows and columns on
        const int ga = n16 >> 2;
        int ya = ry0 + ga / gw, xa = ga % gw, yd = ry0 + g4 / gw, xd = g4 % gw;  // group of the operand, of the result
        auto step = [&](int& y, int& x) {
          y += dq;
          x += dr;
          if (x >= gw) {
            x -= gw;
            ++y;
          }
        };
        // two tiles at a time; the next two are read while these are multiplied
        struct Pair {
          uint4 tok[2][J];
          float back[2];
          int dy[2], dx[2];
        } pr[2];
        auto fetch = [&](Pair& f) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const unsigned at = (unsigned)(min(ya, c.H - 1) * rowbytes) +
                                __umul24((unsigned)min(rx0 + 4 * xa + (n16 & 3), c.W - 1), (unsigned)c.Cp);
#pragma unroll
            for (int jj = 0; jj < J; ++jj)
              f.tok[u][jj] = *reinterpret_cast<const uint4*>(
                  kp + (at + (unsigned)(min(kPack ? (g4 & 1) : 4 * jj + g4, c.nv - 1) * 16)));
            f.back[u] = ksp[(unsigned)((min(yd, c.H - 1) >> c.sh) * c.nbx + ((rx0 + 4 * xd) >> c.sh))];
            f.dy[u] = yd - yq;
            f.dx[u] = rx0 + 4 * xd - xq + 3;
            step(ya, xa);
            step(yd, xd);
          }
        };
        fetch(pr[0]);
        for (int t = 0; t < pairs; t += 2)
#pragma unroll
          for (int turn = 0; turn < 2; ++turn) {
            if (t + turn >= pairs) break;
            const Pair& f = pr[turn];
            if (t + turn + 1 < pairs) fetch(pr[1 - turn]);
            f32x4 d[2], e[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              d[u] = e[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int jj = 0; jj < J; ++jj) {
                const uint4 w = f.tok[u][jj];
                const half8_t k0 = codes_f16(w.x, w.y), k1 = codes_f16(w.z, w.w);
                if constexpr (kPack) {
                  d[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qh[jj][0], d[u], 0, 0, 0);
                  e[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qh[jj][1], e[u], 0, 0, 0);
                } else {
                  e[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, ql[jj][0], e[u], 0, 0, 0);
                  d[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qh[jj][0], d[u], 0, 0, 0);
                  e[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, ql[jj][1], e[u], 0, 0, 0);
                  d[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qh[jj][1], d[u], 0, 0, 0);
                }
              }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if ((unsigned)f.dy[u] <= (unsigned)ws && (unsigned)f.dx[u] < (unsigned)(ws + 4)) {
                float* to = sq + f.dy[u] * kBoxPitch<CT> + f.dx[u];
                // (the powers of two in one step: the product with either alone may leave fp32)
                const float bm = __builtin_amdgcn_frexp_mantf(f.back[u]);
                const int be = __builtin_amdgcn_frexp_expf(f.back[u]) + qexp;
#pragma unroll
                for (int i = 0; i < 4; ++i) to[i] = ldexpf((d[u][i] + e[u][i]) * bm, be);
              }
          }
        return true;
      };
      if (!walk(ymin, ymax, xmin, xmax, true))
        for (int n = 0; n < 16; ++n) {
          const int y1 = __shfl(y0, 4 * n), x1 = __shfl(x0, 4 * n);
          walk(y1, y1, x1, x1, false);
        }
    }
    // byte offsets of the tap columns this lane reads; its own columns' scales
    // (a window meets at most three rows of blocks), validity and buckets
    int xoff[K][R];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int col = R == 1 ? 4 * k + l : R == 2 ? 4 * k + (l & 2) + i : 4 * k + i;
        xoff[k][i] = (int)__umul24((unsigned)min(max(x0 + col, 0), c.W - 1), (unsigned)c.Cp) + lane0;
      }
    float ksc[3][K], vsc[3][K];
    int cb[K];
    bool cok[K], tin[K];
    const int yb0 = y0 >> c.sh;
    // table index of (step, row bucket 0 ..) plus the column's; rows are looked up in LDS
    const int bt = bias_step_bucket(-age, a.bias) * a.bias.nb * a.bias.nb;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int col = 4 * k + l, x = x0 + col;
      tin[k] = x >= 0 && x < c.W && col <= ws;
      cok[k] = on && col < ws && cell_ok(x, ax != 0.f, c.W);
      const int xb = min(max(x, 0), c.W - 1) >> c.sh;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const unsigned at = (unsigned)(min(max(yb0 + i, 0), c.nby - 1) * c.nbx + xb);
        ksc[i][k] = key_factor(ksp[at], qexp);
        vsc[i][k] = vsp[at];
      }
      cb[k] = bt + bias_bucket(Fw + (float)(col - r), a.bias);
      rowb[col] = bias_bucket(Fh + (float)(col - 1 - r), a.bias) * a.bias.nb;  // for tap row col: cell row col - 1
    }
    wave_lds_sync();
    const bool fy = ay != 0.f;
    float hprev[K], pprev[K], p[K], vsk[K];
#pragma unroll
    for (int k = 0; k < K; ++k) hprev[k] = pprev[k] = p[k] = vsk[k] = 0.f;
    int yov = 0;  // byte offset of the value row
    constexpr bool kRow = K * R * V <= kTogether;
    constexpr int kBuf = kRow ? K * R * V : R * V;
    auto load_group = [&](const uint8_t* plane, int yoff, int k, uint4* to) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (4 * k + (R == 1 ? 0 : i) < CT)
#pragma unroll
          for (int v = 0; v < V; ++v)
            to[i * V + v] = *reinterpret_cast<const uint4*>(plane + (unsigned)(yoff + xoff[k][i] + (v ? voff[v] : 0)));
    };
    auto load_row = [&](const uint8_t* plane, int yoff, uint4* to) {
#pragma unroll
      for (int k = 0; k < K; ++k) load_group(plane, yoff, k, to + k * R * V);
    };
    for (int row = 0; row <= ws + 1; ++row) {
      const int y = y0 + row;
      const bool yin = (unsigned)y < (unsigned)c.H;
      const int yo = min(max(y, 0), c.H - 1) * rowbytes;
      const int dyb = (y >> c.sh) - yb0;
      uint4 kb[MX ? 1 : kBuf], vb[kBuf];
      if constexpr (!MX && kRow)
        if (row <= ws) load_row(kp, yo, kb);
      if constexpr (kRow) load_row(vp, yov, vb);
      float sc[K + 1];
#pragma unroll
      for (int k = 0; k <= K; ++k) sc[k] = 0.f;
      const int rb = rowb[min(row, 4 * K - 1)];
      if constexpr (MX) {
        if (row <= ws) {
          const float* from = stab + sub * kBoxQuery<CT> + row * kBoxPitch<CT> + 3 + l;
#pragma unroll
          for (int k = 0; k < K; ++k) sc[k] = yin && tin[k] ? from[4 * k] : 0.f;
        }
      } else if (row <= ws) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          uint4* kk = kRow ? kb + k * R * V : kb;
          if constexpr (!kRow) load_group(kp, yo, k, kk);
          float part[R];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            part[i] = 0.f;
            if (4 * k + (R == 1 ? 0 : i) < CT)
#pragma unroll
              for (int v = 0; v < V; ++v) part[i] = dot16(kk[i * V + v], q[v], part[i]);
          }
          float d;
          if constexpr (R == 1) {
            d = part[0];
          } else if constexpr (R == 2) {
            part[0] += quad<1, 0, 3, 2>(part[0]);
            part[1] += quad<1, 0, 3, 2>(part[1]);
            d = (l & 1) ? part[1] : part[0];
          } else {  // lane l keeps the sum of part l
            const float u0 = ((l & 1) ? part[1] : part[0]) + quad<1, 0, 3, 2>((l & 1) ? part[0] : part[1]);
            const float u1 = ((l & 1) ? part[3] : part[2]) + quad<1, 0, 3, 2>((l & 1) ? part[2] : part[3]);
            d = ((l & 2) ? u1 : u0) + quad<2, 3, 0, 1>((l & 2) ? u0 : u1);
          }
          const float sk = dyb <= 0 ? ksc[0][k] : dyb == 1 ? ksc[1][k] : ksc[2][k];
          sc[k] = yin && tin[k] ? d * sk : 0.f;
        }
      }
      const bool rok = (unsigned)(row - 1) < (unsigned)ws && cell_ok(y - 1, fy, c.H);
      float lg[K], top = -INFINITY;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float right = quad<1, 2, 3, 0>(l == 0 ? sc[k + 1] : sc[k]);  // column + 1
        const float hrow = fmaf(ax, right - sc[k], sc[k]);
        const float x = fmaf(ay, hrow - hprev[k], hprev[k]) + tab[rb + cb[k]];
        lg[k] = rok && cok[k] && fabsf(x) < INFINITY ? x : -INFINITY;
        top = fmaxf(top, lg[k]);
        hprev[k] = hrow;
      }
      top = fmaxf(top, quad<1, 0, 3, 2>(top));
      top = fmaxf(top, quad<2, 3, 0, 1>(top));
      const bool lift = top > m + kSlack;  // also from -inf
      if (__any(lift)) {
        const float m2 = lift ? top : m, f = lift ? __builtin_amdgcn_exp2f(m - top) : 1.f;
        m = m2;
        z *= f;
#pragma unroll
        for (int k = 0; k < K; ++k) pprev[k] *= f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[v][i] = faded(acc[v][i], f);
      }
      const float mm = fmaxf(m, -3.402823466e38f);  // nothing counted yet: weights 2^-inf
#pragma unroll
      for (int k = 0; k < K; ++k) {
        p[k] = __builtin_amdgcn_exp2f(lg[k] - mm);
        z += p[k];
      }
      if (row > 0) {  // values of the row above (its scales and validity were found with its keys)
        auto pin_group = [&](int k, uint4* t) {
#pragma unroll
          for (int n = 0; n < R * V; ++n)
            if (4 * k + (R == 1 ? 0 : n / V) < CT) pin(t[n]);
        };
        if constexpr (kRow) {
#pragma unroll
          for (int k = 0; k < K; ++k) pin_group(k, vb + k * R * V);
        }
        float g[K];
#pragma unroll
        for (int k = 0; k < K; ++k) g[k] = fmaf(ay, pprev[k] - p[k], p[k]);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          uint4* vk = kRow ? vb + k * R * V : vb;
          if constexpr (!kRow) {
            load_group(vp, yov, k, vk);
            pin_group(k, vk);
          }
          const float left = quad<3, 0, 1, 2>(l == 3 ? (k ? g[k ? k - 1 : 0] : 0.f) : g[k]);  // column - 1
          const float wgt = fmaf(ax, left - g[k], g[k]) * vsk[k];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float wi = R == 1 ? wgt
                             : R == 2 ? (i == 0 ? quad<0, 0, 2, 2>(wgt) : quad<1, 1, 3, 3>(wgt))
                                      : (i == 0   ? quad<0, 0, 0, 0>(wgt)
                                         : i == 1 ? quad<1, 1, 1, 1>(wgt)
                                         : i == 2 ? quad<2, 2, 2, 2>(wgt)
                                                  : quad<3, 3, 3, 3>(wgt));
            if (4 * k + (R == 1 ? 0 : i) < CT && wi != 0.f)
#pragma unroll
              for (int v = 0; v < V; ++v) spread16(vk[i * V + v], wi, acc[v]);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        pprev[k] = p[k];
        const float sv = dyb <= 0 ? vsc[0][k] : dyb == 1 ? vsc[1][k] : vsc[2][k];
        vsk[k] = yin && tin[k] ? sv : 0.f;
      }
      yov = yo;
    }
    wave_lds_sync();
  }
  // the waves that share the queries, one after the other
  if (split > 1) {
    float* buf = lds + group * (64 * (2 + 16 * V)) + lane;  // (over the buckets and the table)
    for (int j = 1; j < split; ++j) {
      __syncthreads();
      if (part_of == j) {
        buf[0] = m;
        buf[64] = z;
#pragma unroll
        for (int i = 0; i < 16 * V; ++i) buf[(2 + i) * 64] = acc[i / 16][i % 16];
      }
      __syncthreads();
      if (part_of == 0) {
        const float mj = buf[0], top = fmaxf(m, mj);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        const float fj = mj == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mj - top);
        m = top;
        z = z * f + buf[64] * fj;
#pragma unroll
        for (int i = 0; i < 16 * V; ++i)
          acc[i / 16][i % 16] = faded(acc[i / 16][i % 16], f) + faded(buf[(2 + i) * 64], fj);
      }
    }
    if (part_of != 0) return;
  }
  // sums over the quad: the weights' sum, and the outputs of lanes that hold the same channels
  z += quad<1, 0, 3, 2>(z);
  z += quad<2, 3, 0, 1>(z);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (R == 1) acc[v][i] += quad<1, 0, 3, 2>(acc[v][i]);
      if constexpr (R <= 2) acc[v][i] += quad<2, 3, 0, 1>(acc[v][i]);
    }
  if (!stored) return;
  const float inv = z > 0.f ? 1.f / z : 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int ch = (v * R + lr) * 16 + i;
      if (i / (4 * R) != l / R || ch >= c.Ch) continue;  // each lane stores its share
      const float o = z > 0.f ? acc[v][i] * inv : 0.f;
      if constexpr (POINTS)
        a.out[qi * c.C + hd * c.Ch + ch] = o;
      else
        a.out[((long long)b * c.C + hd * c.Ch + ch) * HW + (long long)h * c.W + w] = o;
    }
}

template <int CT, bool POINTS>
static void run_attend_quad(const AttendArgs& a, int split, hipStream_t s) {
  const CacheGeo& c = a.c;
  const int groups = 4 / split, tx = (c.W + 7) / 8, ty = (c.H + 2 * groups - 1) / (2 * groups);
  const long long blocks = POINTS ? (a.n + groups * 16 - 1) / (groups * 16) : (long long)c.B * tx * ty;
  const dim3 grid((unsigned)(POINTS ? blocks * c.HD : (blocks * c.HD + 7) / 8 * 8)), block(256);
  size_t lds = (64 * 16 + (a.table ? a.bias.buckets : 1)) * sizeof(float);
  // Scores from the matrix cores, where LDS for them fits the 64 KB that a launch may ask for (ws <= 9 whatever the
  // table).  3 slots, 200 x 240, offsets 1.5 pixels apart, vector units / matrix cores: 32 channels ws = 7 60 / 70 us,
  // ws = 9 107 / 96, ws = 11 124 / 137; 48 channels ws = 3 43 / 55, ws = 5 76 / 74; 64 channels ws = 3 40 / 49, ws = 5
  // 73 / 67, ws = 9 149 / 121, ws = 11 195 / 187; 128 channels ws = 3 71 / 88, ws = 5 124 / 129, ws = 7 182 / 171, ws = 9
  // 295 / 235, ws = 11 369 / 292; 16 channels: the tiles' other work is what the products were
  const size_t boxes = 4 * 16 * kBoxQuery<CT> * sizeof(float);
  static_assert((64 * 16 + SNLS_BIAS_MAX_BUCKETS + 4 * 16 * kBoxQuery<10>) * sizeof(float) <= 65536, "ws <= 9 always fits");
  const bool mx = lds + boxes <= 65536;
  auto room = [&](int V, bool with_boxes) {
    const size_t join = split > 1 ? (size_t)groups * 64 * (2 + 16 * V) * sizeof(float) : 0;
    const size_t own = lds + (with_boxes ? boxes : 0);
    return join > own ? join : own;
  };
#define SNLS_QUAD(R, V) \
  hipLaunchKernelGGL((attend_quad_kernel<CT, R, V, POINTS, false>), grid, block, room(V, false), s, a, tx, ty, split)
#define SNLS_QUAD_MX(R, V)                                                                                            \
  if constexpr (!POINTS && (R * V == 2 ? CT == 10 : CT >= 6 && CT <= 12)) {                                         \
    if (CT <= 10 || mx) {                                                                                           \
      hipLaunchKernelGGL((attend_quad_kernel<CT, R, V, false, true>), grid, block, room(V, true), s, a, tx, ty,     \
                         split);                                                                                    \
      break;                                                                                                        \
    }                                                                                                               \
  }                                                                                                                 \
  if constexpr (POINTS || !(R * V == 2 ? CT == 10 : CT >= 6 && CT <= 10)) SNLS_QUAD(R, V)
  switch (c.nv) {
    case 1: SNLS_QUAD(1, 1); break;
    case 2: SNLS_QUAD_MX(2, 1); break;
    case 3: SNLS_QUAD_MX(1, 3); break;
    case 4: SNLS_QUAD_MX(4, 1); break;
    case 6: SNLS_QUAD_MX(2, 3); break;
    case 5: case 7: case 8: SNLS_QUAD_MX(4, 2); break;
    case 9: case 10: case 11: case 12: SNLS_QUAD(4, 3); break;
    default: SNLS_QUAD(4, 4); break;
  }
#undef SNLS_QUAD_MX
#undef SNLS_QUAD
}

template <bool POINTS>
static void run_attend(const AttendArgs& a, hipStream_t s) {
  const CacheGeo& c = a.c;
  // waves per 16 queries: the chip has 1,024 places for a wave.  Split by 1 / 2 / 4 (4 slots, ws = 9): 4 heads of
  // 16 channels 46 / 25 / 17 us at 48 x 48 (576 waves), 46 / 32 / 34 us at 64 x 64 (1,024), 71 / 61 us at 96 x 96
  // (2,304), 97 / 93 us at 128 x 128 (4,096)
  const long long waves = (a.n + 15) / 16 * c.HD;
  int split = waves >= 4096 ? 1 : waves >= 1024 ? 2 : 4;
  while (split > c.S) split /= 2;
  if (a.ws <= 3)
    run_attend_quad<4, POINTS>(a, split, s);
  else if (a.ws <= 5)
    run_attend_quad<6, POINTS>(a, split, s);
  else if (a.ws <= 7)
    run_attend_quad<8, POINTS>(a, split, s);
  else if (a.ws <= 9)
    run_attend_quad<10, POINTS>(a, split, s);
  else if (a.ws <= 11)
    run_attend_quad<12, POINTS>(a, split, s);
  else
    run_attend_quad<16, POINTS>(a, split, s);
}

snls_status launch_cache_attend(const float* q, const int32_t* points, long long n, const float* flows,
                                const int32_t* ages, const uint8_t* k_codes, const float* k_scales,
                                const uint8_t* v_codes, const float* v_scales, const float* table,
                                const CacheGeo& c, const Bias& bias, int ws, float scale, float* out, hipStream_t s) {
  int se = 0;
  const float sm = frexpf(scale, &se);
  const AttendArgs a{q, points, n, flows, ages, k_codes, k_scales, v_codes, v_scales, table, c, bias, ws, scale, sm, se, out};
  // few points: 4, 8 or 16 waves each, which share its slots, for the shortest way through one query.  4 waves / quads
  // (6 slots, ws = 9): one head of 64 channels 30 / 51 us for 1,024 points, 56 / 52 us for 2,048; 4 heads of 16
  // channels 29 / 32 us for 512, 51 / 33 us for 1,024.  4 / 16 waves (16 slots): 12 heads 20.0 / 17.3 us for 16
  // points, 27 / 37 us for 64, where 4,096 waves are passed
  const long long single = n * c.HD;
  if (points && single <= 2048) {
    if (c.S > 8 && single * 16 <= 4096)
      run_attend_wave<16>(a, s);
    else if (c.S > 4 && single * 8 <= 4096)
      run_attend_wave<8>(a, s);
    else
      run_attend_wave<4>(a, s);
  } else if (points) {
    run_attend<true>(a, s);
  } else {
    run_attend<false>(a, s);
  }
  return hipGetLastError() == hipSuccess ? SNLS_OK : SNLS_ERR_HIP;
}

}  // namespace snls
