// layer.h -- what the norm, dropout, rotary positions and 8-bit projections share
// (host and device side).  The search's and the attention's kernels do not include
// it: counter records of theirs are kept by the text of their sources and of
// snls_internal.h, and stay valid when these calls change.
#pragma once

#include "snls_internal.h"

namespace snls {

// A call's dropout, passed to kernels by value: an element stays where its word
// is at least `thr`.  rng == nullptr: nothing is dropped.
struct Drop {
  const unsigned long long* rng;  // device: seed, step
  unsigned thr, site;
  float keep;  // 1 / (1 - drop)
};

// The rotary positions of a call.  turns: angle per position of every pair in
// turns, the three axes one after the other.
struct Rotary {
  int B, T, C, H, W, HD, Ch;
  int pairs[3], total;  // total: their sum
  int interleaved, row0, col0;
  double turns[SNLS_ROTATE_MAX_PAIRS];
};

// Host-side checks (validate.cpp).  Return SNLS_OK or an error code; they never
// touch the GPU.
snls_status check_norm(const snls_norm_params* np);
snls_status check_drop(float drop, uint32_t site, const uint64_t* rng, Drop* out);
snls_status check_rotate(const snls_rotate_params* rp, bool inverse, Rotary* out);
snls_status check_project(const snls_project_params* pp);

// Device workspace of snls_norm_backward: partial sums of every channel.
size_t norm_backward_ws_bytes(const snls_norm_params& np);

#ifdef __HIPCC__
snls_status launch_norm(const float* x, const float* branch, const Drop& drop, const float* gamma, const float* beta,
                        const snls_norm_params& np, float* total, float* y, float* stats, hipStream_t s);
// grad_gamma == nullptr: no sums over the pixels
snls_status launch_norm_backward(const float* grad_y, const float* grad_total, const float* total, const float* stats,
                                 const float* gamma, const Drop& drop, const snls_norm_params& np, float* grad_x,
                                 float* grad_branch, float* grad_gamma, float* grad_beta, double* ws, hipStream_t s);
snls_status launch_dropout(const float* x, const float* residual, const Drop& drop, long long n, float* out,
                           hipStream_t s);
snls_status launch_rotate(const float* q, const float* k, const int64_t* times, const Rotary& r, float* q_out,
                          float* k_out, hipStream_t s);
snls_status launch_rotate_points(const float* q, const int32_t* points, long long n, const int64_t* times,
                                 const Rotary& r, float* out, hipStream_t s);
snls_status launch_project_pack(const float* w, int cin, int cout, int8_t* codes, float* scales, hipStream_t s);
snls_status launch_project(const float* x, const int8_t* codes, const float* scales, const float* bias,
                           const snls_project_params& pp, float* out, hipStream_t s);
#endif

}  // namespace snls
