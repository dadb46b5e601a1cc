// philox.h -- dropout's mask (device side; the same for the norm of a residual
// sum, its gradients and the dropout on its own).
//
// Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011): four words of 32 bits from a counter of
// 128 bits and a key of 64.  Elements 4b .. 4b+3 take the words of block b, so
// a lane with four consecutive elements forms one block for them, or two where
// they straddle a border.
#pragma once

#include "layer.h"

#ifdef __HIPCC__

namespace snls {

struct Words {
  unsigned w[4];
};

// Both halves of a product of 32-bit numbers in one instruction (the compiler
// takes one for each half).
SNLS_DEV void wide_product(unsigned a, unsigned b, unsigned* hi, unsigned* lo) {
  unsigned long long r;
  unsigned long long carry;
  asm("v_mad_u64_u32 %0, %1, %2, %3, 0" : "=v"(r), "=s"(carry) : "s"(a), "v"(b));
  *hi = (unsigned)(r >> 32), *lo = (unsigned)r;
}

// The generator of a call: key and the counter's upper half.
struct Philox {
  unsigned k0, k1, step, site;
  SNLS_DEV explicit Philox(const Drop& d) {
    const unsigned long long seed = d.rng ? d.rng[0] : 0;
    k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
    step = d.rng ? (unsigned)d.rng[1] : 0, site = d.site;
  }
  SNLS_DEV Words block(long long b) const {
    unsigned c0 = (unsigned)b, c1 = (unsigned)(b >> 32), c2 = step, c3 = site, a = k0, e = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      unsigned h0, l0, h1, l1;
      wide_product(0xD2511F53u, c0, &h0, &l0);
      wide_product(0xCD9E8D57u, c2, &h1, &l1);
      c0 = h1 ^ c1 ^ a, c1 = l1, c2 = h0 ^ c3 ^ e, c3 = l0;
      a += 0x9E3779B9u, e += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
  }
  // Words of elements i .. i+V-1, V = 1, 2 or 4.
  template <int V>
  SNLS_DEV void run(long long i, unsigned* w) const {
    const int j = (int)(i & 3);
    const Words a = block(i >> 2);
    if constexpr (V == 1) {
      w[0] = j == 0 ? a.w[0] : j == 1 ? a.w[1] : j == 2 ? a.w[2] : a.w[3];
    } else if (j + V <= 4) {
#pragma unroll
      for (int n = 0; n < V; ++n) w[n] = V == 2 && j == 1 ? a.w[n + 1] : V == 2 && j == 2 ? a.w[n + 2] : a.w[n];
    } else {
      const Words b = block((i >> 2) + 1);
#pragma unroll
      for (int n = 0; n < V; ++n)
        w[n] = j == 1 ? (n < 3 ? a.w[n + 1 & 3] : b.w[0])
                      : j == 2 ? (n < 2 ? a.w[n + 2 & 3] : b.w[n - 2 & 3]) : (n < 1 ? a.w[3] : b.w[n - 1 & 3]);
    }
  }
};

// Value of lane M of the four lanes this one is among.
template <int M>
SNLS_DEV unsigned of_four(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, M * 0x55, 0xf, 0xf, false);
}

// Words of a lane's element in each of four lists, where four lanes hold four
// consecutive elements of a block in all of them (mine: this lane's place in its
// block, 0 .. 3): each forms the block of one list, `b`, and they exchange.
SNLS_DEV void share_blocks(const Words& b, int mine, unsigned* w) {
  auto pick = [&](unsigned a, unsigned c, unsigned d, unsigned e) {
    return mine & 2 ? (mine & 1 ? e : d) : (mine & 1 ? c : a);
  };
  w[0] = pick(of_four<0>(b.w[0]), of_four<0>(b.w[1]), of_four<0>(b.w[2]), of_four<0>(b.w[3]));
  w[1] = pick(of_four<1>(b.w[0]), of_four<1>(b.w[1]), of_four<1>(b.w[2]), of_four<1>(b.w[3]));
  w[2] = pick(of_four<2>(b.w[0]), of_four<2>(b.w[1]), of_four<2>(b.w[2]), of_four<2>(b.w[3]));
  w[3] = pick(of_four<3>(b.w[0]), of_four<3>(b.w[1]), of_four<3>(b.w[2]), of_four<3>(b.w[3]));
}

// The same for two lanes with two elements each (odd: this lane has the second
// two) in two lists.
SNLS_DEV void share_blocks(const Words& b, int odd, unsigned (*w)[2]) {
  auto partner = [](unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false); };
  const unsigned x = partner(odd ? b.w[0] : b.w[2]), y = partner(odd ? b.w[1] : b.w[3]);
  w[0][0] = odd ? x : b.w[0], w[0][1] = odd ? y : b.w[1];
  w[1][0] = odd ? b.w[2] : x, w[1][1] = odd ? b.w[3] : y;
}

SNLS_DEV float dropped(float x, unsigned word, const Drop& d) { return word >= d.thr ? x * d.keep : 0.f; }

}  // namespace snls

#endif  // __HIPCC__
