// Counter-based random numbers for dropout: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", 2011).  A mask is a function of (seed, step, site, element) and is drawn again wherever it is needed: nothing of it
// is stored.  Eight elements share one counter and take a 16-bit half of its four words each: half the multiplications of 32-bit
// numbers, which at four bytes an element would bound the kernels instead of the memory; a probability is then a multiple of
// 2^-16, and the factor of what is kept is that of the multiple.
#pragma once
#include "common.h"
#include "vec8.h"

namespace lp {

struct Drop {
  const uint64_t* rng;      // device: seed, step
  unsigned site, thr;       // dropped: number < thr (65536: all)
  float factor;             // 65536 / (65536 - thr)
};
// p of 0 drops nothing (rng is not read then); false: not a probability, or no generator
static inline bool make_drop(float p, const void* rng, unsigned site, Drop* d) {
  if (!(p >= 0.f && p <= 1.f)) return false;
  d->thr = (unsigned)((double)p * 65536.0 + 0.5);
  d->site = site;
  d->factor = d->thr < 65536 ? (float)(65536.0 / (65536.0 - d->thr)) : 0.f;
  d->rng = d->thr ? (const uint64_t*)rng : nullptr;
  return d->thr == 0 || (rng != nullptr && ((uintptr_t)rng & 7) == 0);
}

struct PhiloxKey { unsigned k0, k1, s0, s1; };
__device__ __forceinline__ PhiloxKey philox_key(const Drop& d) {
  PhiloxKey k = {0, 0, 0, 0};
  if (d.thr) {
    const uint64_t seed = d.rng[0], step = d.rng[1];
    k.k0 = (unsigned)seed; k.k1 = (unsigned)(seed >> 32);
    k.s0 = (unsigned)step; k.s1 = (unsigned)(step >> 32);
  }
  return k;
}
// The four words of counter (group, site, step).
__device__ __forceinline__ uint4 philox(const PhiloxKey& key, unsigned group, unsigned site) {
  unsigned c0 = group, c1 = site, c2 = key.s0, c3 = key.s1, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (unsigned)(b >> 32) ^ c1 ^ k0; c1 = (unsigned)b;
    c2 = (unsigned)(a >> 32) ^ c3 ^ k1; c3 = (unsigned)a;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}
__device__ __forceinline__ unsigned half_of(const uint4& w, int e) {       // number of element 8 * group + e
  const unsigned x = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
  return (e & 1) ? x >> 16 : x & 0xffffu;
}
// A dropped element is 0 whatever it was, an infinity or a NaN too.
__device__ __forceinline__ void drop8(const Drop& d, const PhiloxKey& key, unsigned group, float (&v)[8]) {
  const uint4 w = philox(key, group, d.site);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = half_of(w, e) >= d.thr ? v[e] * d.factor : 0.f;
}

}  // namespace lp
