// validate.cpp -- host-only argument checks of the C ABI.  Nothing here
// touches the GPU, so every error path can be exercised on a machine
// without one.
#include <limits.h>
#include <math.h>

#include "snls_internal.h"

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

}  // namespace snls
