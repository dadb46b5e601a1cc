// validate.cpp -- host-only argument checks of the C ABI.  Nothing here
// touches the GPU, so every error path can be exercised on a machine
// without one.
#include <limits.h>
#include <math.h>

#include "layer.h"

namespace snls {

// Sizes stay below 2^31 per tensor dimension product where kernels index
// with 32-bit arithmetic inside a frame; whole tensors use 64-bit offsets.
static const long long kMaxPlane = 1LL << 30;

snls_status check_params(const snls_params* p, bool need_k, Geo* g) {
  if (!p) return SNLS_ERR_INVALID_ARG;
  if (p->struct_size != sizeof(snls_params)) return SNLS_ERR_INVALID_ARG;
  if (p->B < 1 || p->T < 1 || p->C < 1 || p->H < 1 || p->W < 1 || p->HD < 1) return SNLS_ERR_INVALID_ARG;
  if (p->C % p->HD != 0) return SNLS_ERR_INVALID_ARG;
  if (p->ws < 1 || p->wt < 0 || p->ps < 1 || p->stride0 < 1) return SNLS_ERR_INVALID_ARG;
  if (!(p->stride1 > 0.f) || !isfinite(p->stride1)) return SNLS_ERR_INVALID_ARG;
  if (p->dist_type != SNLS_DIST_PROD && p->dist_type != SNLS_DIST_L2) return SNLS_ERR_INVALID_ARG;
  if ((long long)p->H * p->W > kMaxPlane) return SNLS_ERR_UNSUPPORTED;
  // displacements of kFarDisp or more must leave every frame
  if (p->H >= (long long)kFarDisp || p->W >= (long long)kFarDisp) return SNLS_ERR_UNSUPPORTED;
  if (p->ws > 255 || p->ps > 255 || p->wt > 63) return SNLS_ERR_UNSUPPORTED;
  long long ncand = (long long)(2 * p->wt + 1) * p->ws * p->ws;
  if (ncand > INT_MAX / 4) return SNLS_ERR_UNSUPPORTED;
  if (p->k < 0 || p->k > ncand) return SNLS_ERR_INVALID_ARG;
  if (need_k && p->k < 1) return SNLS_ERR_INVALID_ARG;
  if (p->k > SNLS_MAX_K) return SNLS_ERR_UNSUPPORTED;
  if (g) {
    g->B = p->B; g->T = p->T; g->C = p->C; g->H = p->H; g->W = p->W; g->HD = p->HD;
    g->ws = p->ws; g->wt = p->wt; g->ps = p->ps; g->s0 = p->stride0; g->s1 = p->stride1;
    g->k = p->k; g->dist = p->dist_type;
    g->nH = (p->H - 1) / p->stride0 + 1;
    g->nW = (p->W - 1) / p->stride0 + 1;
    g->Ch = p->C / p->HD;
    g->r = p->ws / 2;
    g->lo = -(p->ps / 2);
    g->ncand = (int)ncand;
    g->nslot = 2 * p->wt;
    g->HW = (long long)p->H * p->W;
    g->rows = (long long)p->B * p->HD * p->T * g->nH * g->nW;
  }
  return SNLS_OK;
}

snls_status check_topk_args(int64_t rows, int32_t n_cand, int32_t k, int32_t dist_type) {
  if (rows < 0 || n_cand < 1 || k < 1 || k > n_cand) return SNLS_ERR_INVALID_ARG;
  if (dist_type != SNLS_DIST_PROD && dist_type != SNLS_DIST_L2) return SNLS_ERR_INVALID_ARG;
  if (k > SNLS_MAX_K) return SNLS_ERR_UNSUPPORTED;
  return SNLS_OK;
}

snls_status check_bias(const snls_bias_params* b, Bias* out) {
  if (!b || b->struct_size != sizeof(snls_bias_params)) return SNLS_ERR_INVALID_ARG;
  if (b->radius < 0 || b->n_edges < 0) return SNLS_ERR_INVALID_ARG;
  if (b->radius > 63 || b->n_edges > SNLS_BIAS_MAX_EDGES) return SNLS_ERR_UNSUPPORTED;
  for (int i = 0; i < b->n_edges; ++i)
    if (!isfinite(b->edges[i]) || !(b->edges[i] > (i ? b->edges[i - 1] : 0.f))) return SNLS_ERR_INVALID_ARG;
  const int nb = 2 * b->n_edges + 1;
  if ((2 * b->radius + 1) * nb * nb > SNLS_BIAS_MAX_BUCKETS) return SNLS_ERR_UNSUPPORTED;
  out->radius = b->radius;
  out->nE = b->n_edges;
  out->nb = nb;
  out->buckets = (2 * b->radius + 1) * nb * nb;
  for (int i = 0; i < SNLS_BIAS_MAX_EDGES; ++i) out->edges[i] = i < b->n_edges ? b->edges[i] : INFINITY;
  return SNLS_OK;
}

snls_status check_cache(const snls_cache_params* c, CacheGeo* out) {
  if (!c || c->struct_size != sizeof(snls_cache_params)) return SNLS_ERR_INVALID_ARG;
  if (c->B < 1 || c->slots < 1 || c->C < 1 || c->H < 1 || c->W < 1 || c->HD < 1 || c->block < 1)
    return SNLS_ERR_INVALID_ARG;
  if (c->C % c->HD != 0) return SNLS_ERR_INVALID_ARG;
  const int Ch = c->C / c->HD;
  if ((c->block != 8 && c->block != 16) || Ch > 256) return SNLS_ERR_UNSUPPORTED;
  if (c->H >= (long long)kFarDisp || c->W >= (long long)kFarDisp) return SNLS_ERR_UNSUPPORTED;
  const int Cp = (Ch + 15) / 16 * 16;
  // a token's byte offset inside its plane is 32-bit; planes are found with 64 bits
  if ((long long)c->H * c->W * Cp >= 1LL << 31) return SNLS_ERR_UNSUPPORTED;
  // a launch holds less than 2^32 threads, 4 per pixel and head of the padded frame
  const double pixels = (double)((c->H + 15) / 16 * 16) * ((c->W + 31) / 32 * 32);
  if ((double)c->B * c->HD * pixels >= 1073741824.0 || (double)c->B * c->slots >= 2147483648.0)
    return SNLS_ERR_UNSUPPORTED;
  out->B = c->B; out->S = c->slots; out->C = c->C; out->HD = c->HD; out->H = c->H; out->W = c->W;
  out->Ch = Ch;
  out->Cp = Cp;
  out->nv = Cp / 16;
  out->sh = c->block == 8 ? 3 : 4;
  out->nby = (c->H + c->block - 1) / c->block;
  out->nbx = (c->W + c->block - 1) / c->block;
  return SNLS_OK;
}

// Elements of (frames, C, pixels): offsets are 64-bit, grids strided.
static bool too_many(long long frames, long long channels, long long pixels) {
  return (double)frames * (double)channels * (double)pixels >= 274877906944.0;  // 2^38
}

snls_status check_norm(const snls_norm_params* np) {
  if (!np || np->struct_size != sizeof(snls_norm_params)) return SNLS_ERR_INVALID_ARG;
  if (np->C < 1 || np->frames < 0 || np->pixels < 1) return SNLS_ERR_INVALID_ARG;
  if (!isfinite(np->eps) || np->eps < 0.f) return SNLS_ERR_INVALID_ARG;
  if (!(np->drop >= 0.f && np->drop < 1.f)) return SNLS_ERR_INVALID_ARG;
  // (the place of a lane in its plane, and in the next, is a 32-bit offset in bytes)
  if (np->pixels >= 1 << 29 || np->C >= 1 << 16 || too_many(np->frames, np->C, np->pixels)) return SNLS_ERR_UNSUPPORTED;
  return SNLS_OK;
}

snls_status check_drop(float drop, uint32_t site, const uint64_t* rng, Drop* out) {
  if (!(drop >= 0.f && drop < 1.f)) return SNLS_ERR_INVALID_ARG;
  if (drop > 0.f && !rng) return SNLS_ERR_INVALID_ARG;
  out->rng = drop > 0.f ? reinterpret_cast<const unsigned long long*>(rng) : nullptr;
  out->thr = (unsigned)((double)drop * 4294967296.0);
  out->site = site;
  out->keep = (float)(1.0 / (1.0 - (double)drop));
  return SNLS_OK;
}

snls_status check_rotate(const snls_rotate_params* rp, bool inverse, Rotary* out) {
  if (!rp || rp->struct_size != sizeof(snls_rotate_params)) return SNLS_ERR_INVALID_ARG;
  if (rp->B < 1 || rp->T < 1 || rp->C < 1 || rp->H < 1 || rp->W < 1 || rp->HD < 1 || rp->C % rp->HD != 0)
    return SNLS_ERR_INVALID_ARG;
  if (rp->interleaved != 0 && rp->interleaved != 1) return SNLS_ERR_INVALID_ARG;
  long long total = 0;
  for (int a = 0; a < 3; ++a) {
    if (rp->pairs[a] < 0 || !isfinite(rp->theta[a]) || !(rp->theta[a] > 0.f)) return SNLS_ERR_INVALID_ARG;
    total += rp->pairs[a];
  }
  const int Ch = rp->C / rp->HD;
  if (2 * total > Ch) return SNLS_ERR_INVALID_ARG;
  if (total > SNLS_ROTATE_MAX_PAIRS) return SNLS_ERR_UNSUPPORTED;
  if ((long long)rp->H * rp->W >= kMaxPlane || too_many((long long)rp->B * rp->T, rp->C, (long long)rp->H * rp->W))
    return SNLS_ERR_UNSUPPORTED;
  out->B = rp->B; out->T = rp->T; out->C = rp->C; out->H = rp->H; out->W = rp->W; out->HD = rp->HD;
  out->Ch = Ch;
  out->total = (int)total;
  out->interleaved = rp->interleaved;
  out->row0 = rp->row0; out->col0 = rp->col0;
  int at = 0;
  for (int a = 0; a < 3; ++a) {
    out->pairs[a] = rp->pairs[a];
    // theta^(-i/n) / 2 pi as a product of i equal factors, in the 64 bits of a long
    // double: a factor is off by at most (ln(theta)/n + 2) 2^-64, a product by 2^-64
    // more, all of them by 2^-55, and the turns, rounded to 53 bits, by 1.25 * 2^-53
    // (an exponent i/n rounded to 53 bits costs ln(theta) i/n 2^-53: 10 * 2^-51 for
    // the largest theta).
    long double f = 1.0L / 6.28318530717958647692528676655900577L;
    const long double factor = rp->pairs[a] > 0 ? powl((long double)rp->theta[a], -1.0L / rp->pairs[a]) : 1.0L;
    for (int i = 0; i < rp->pairs[a]; ++i, f *= factor) out->turns[at++] = (double)(inverse ? -f : f);
  }
  return SNLS_OK;
}

snls_status check_project(const snls_project_params* pp) {
  if (!pp || pp->struct_size != sizeof(snls_project_params)) return SNLS_ERR_INVALID_ARG;
  if (pp->cin < 1 || pp->cout < 1 || pp->parts < 1 || pp->frames < 0 || pp->pixels < 1) return SNLS_ERR_INVALID_ARG;
  if (pp->cout % pp->parts != 0) return SNLS_ERR_INVALID_ARG;
  // (the place of a lane in its plane, or 16 planes on, is a 32-bit offset in bytes)
  if (pp->cin > SNLS_PROJECT_MAX_CIN || pp->cout >= 1 << 16 || pp->pixels >= 1 << 25) return SNLS_ERR_UNSUPPORTED;
  if (too_many(pp->frames, pp->cin, pp->pixels) || too_many(pp->frames, pp->cout, pp->pixels))
    return SNLS_ERR_UNSUPPORTED;
  return SNLS_OK;
}

}  // namespace snls
