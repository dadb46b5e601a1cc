// lanes.h -- runs of consecutive floats that a lane loads and stores at once
// (device side), at any 4-byte address.
#pragma once

#include "snls_internal.h"

#ifdef __HIPCC__

namespace snls {

template <int V>
struct __attribute__((packed, aligned(4))) Run {
  float v[V];
};

// The first cnt of V floats at `from`, 0 for the others.
template <int V>
SNLS_DEV void load_run(const float* from, int cnt, float* to) {
  if (cnt >= V) {
    const Run<V> r = *reinterpret_cast<const Run<V>*>(from);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = r.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = i < cnt ? from[i] : 0.f;
  }
}

template <int V>
SNLS_DEV void store_run(float* to, int cnt, const float* from) {
  if (cnt >= V) {
    Run<V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = from[i];
    *reinterpret_cast<Run<V>*>(to) = r;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < cnt) to[i] = from[i];
  }
}

// store_run past the caches (non-temporal): outputs of whole videos push inputs
// out of the 256 MB cache otherwise, and a kernel that reads them next gains
// nothing by their lying there (norm, rotation, projection and dropout in a row
// took 960 us with ordinary stores and 915 so at 525 MB a tensor, 188 and 177 at
// 105 MB, 24.4 and 23.9 at 4 MB).
template <int V>
SNLS_DEV void stream_run(float* to, int cnt, const float* from) {
  if (cnt >= V) {
    typedef float Vec __attribute__((ext_vector_type(V), aligned(4)));
    Vec r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = from[i];
    __builtin_nontemporal_store(r, reinterpret_cast<Vec*>(to));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < cnt) to[i] = from[i];
  }
}

// The float at `base` (the same for the wave: two scalar registers) and a lane's
// offset in bytes.
SNLS_DEV float load_at(const float* base, unsigned bytes) {
  return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(base) + bytes);
}
template <bool PAST>
SNLS_DEV void store_at(float* base, unsigned bytes, float v) {
  float* const to = reinterpret_cast<float*>(reinterpret_cast<char*>(base) + bytes);
  if constexpr (PAST)
    __builtin_nontemporal_store(v, to);
  else
    *to = v;
}

// Workgroup b of n in an order that gives each of the 8 XCDs, which take
// workgroups in turn, a run of neighbours: what two of them write of one cache
// line meets in one L2.
SNLS_DEV unsigned by_xcd(unsigned b, unsigned n) {
  const unsigned per = n / 8;
  return b < per * 8 ? (b & 7) * per + b / 8 : b;
}

}  // namespace snls

#endif  // __HIPCC__
