// Writing the 8-bit cache of keys and values, and reading it back (cache.h has the layout).
//   append:  s' = max(s of the page's earlier tokens, the least power of two with max |x| / s' <= 448),  code = e4m3(x / s'); where s' > s
//            the page's earlier codes c become e4m3(c s / s')
//   read:    x = code s
// Bound by memory: one byte for every two or four.  A wave has a page, a head and a side (keys or values): an item of a lane is eight columns
// of sixteen tokens, so that both sides are read as they stand in the rows, and written as they stand in the page: eight bytes a token of the keys, sixteen
// a column of the values, transposed on the way in the lane's registers.
#include <type_traits>

#include "cache.h"
#include "vec8.h"

namespace lp {

namespace {

template <typename T> struct Rows { T *k, *v; int64_t ldk, ldv; };

template <typename T, bool VEC>
__device__ __forceinline__ void take8(const T* p, float (&v)[8]) {
  if constexpr (VEC) {
    load8(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f(p[e]);
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void put8(T* p, const float (&v)[8]) {
  if constexpr (VEC) {
    store8(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = from_f<T>(v[e]);
  }
}
// The least power of two s with most / s <= 448 = 1.75 * 2^8; 2^-126 at least, so that 1 / s is a number too.
__device__ __forceinline__ float scale_for(float most) {
  const unsigned u = __builtin_bit_cast(unsigned, most);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __builtin_bit_cast(float, (unsigned)(e < 1 ? 1 : e) << 23);
}
__device__ __forceinline__ bool finite(float v) { return (__builtin_bit_cast(unsigned, v) & 0x7f800000u) != 0x7f800000u; }
// An infinity has no code: it is held as a NaN.
__device__ __forceinline__ unsigned pack2(float a, float b, unsigned w, bool high) {
  const float nan = __builtin_bit_cast(float, 0x7fc00000u);
  a = finite(a) ? a : nan;
  b = finite(b) ? b : nan;
  return high ? __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, true) : __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
}
__device__ __forceinline__ unsigned pack4(float a, float b, float c, float d) { return pack2(c, d, pack2(a, b, 0, false), true); }
__device__ __forceinline__ void unpack4(unsigned w, float (&v)[4]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}
__device__ __forceinline__ unsigned rescale4(unsigned w, float ratio) {
  float v[4];
  unpack4(w, v);
  return pack4(v[0] * ratio, v[1] * ratio, v[2] * ratio, v[3] * ratio);
}

// What a wave works on: slot `slot` of sequence b holds the new rows row .. row + hi - lo - 1 at its tokens lo .. hi - 1.
struct Part { int page, h, lo, hi; int64_t row; };
__device__ __forceinline__ bool part_of(const CacheView& c, int64_t unit, int slots, Part* p) {
  const int h = (int)(unit % c.Hkv);
  const int64_t rest = unit / c.Hkv;
  const int b = (int)(rest / slots);
  if (b >= c.B) return false;
  const Sequence s = sequence_of(c, b);
  const int from = s.len - s.n, slot = (from >> c.shift) + (int)(rest % slots);      // from < 0: there is no page for those rows
  const int64_t base = (int64_t)slot << c.shift;
  const int64_t lo = from > base ? from - base : 0, end = s.len - base;
  p->lo = (int)lo;
  p->hi = (int)(end < ((int64_t)1 << c.shift) ? end : (int64_t)1 << c.shift);
  p->row = s.first + (base + lo - from);
  p->h = h;
  if (p->hi <= p->lo) return false;
  p->page = page_of(c, b, slot);
  return true;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_cache_append(CacheView c, Rows<const T> x, int slots) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = ((int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x) >> 6;
  const bool values = unit & 1;
  Part p;
  if (!part_of(c, unit >> 1, slots, &p) || p.page < 0) return;
  const int cols = c.dh / 8, size = 1 << c.shift;
  const T* rows = (values ? x.v + p.row * x.ldv : x.k + p.row * x.ldk) + p.h * c.dh;
  const int64_t ld = values ? x.ldv : x.ldk, where = (int64_t)p.page * c.Hkv + p.h;
  float* scale = (values ? c.vs : c.ks) + where;
  uint8_t* pool = (values ? c.v : c.k) + (where * c.dh << c.shift);

  const int first = p.lo >> 4, runs = ((p.hi + 15) >> 4) - first;
  float most = 0.f;
  for (int i = lane; i < runs * cols; i += 64) {
    const int r = first + i / cols, d = (i % cols) * 8;
#pragma unroll 4
    for (int t = 0; t < 16; ++t) {
      const int at = r * 16 + t;
      if (at < p.lo || at >= p.hi) continue;
      float v[8];
      take8<T, VEC>(rows + (at - p.lo) * ld + d, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = finite(v[e]) ? fmaxf(most, fabsf(v[e])) : most;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
  const float old = p.lo > 0 ? *scale : 0.f;
  const float need = scale_for(most), s = old > need ? old : need, inv = 1.f / s;
  const bool grown = p.lo > 0 && s > old;
  const float ratio = old / s;
  if (lane == 0) *scale = s;

  const int from = grown ? 0 : first, all = ((p.hi + 15) >> 4) - from;
  for (int i = lane; i < all * cols; i += 64) {
    const int r = from + i / cols, d = (i % cols) * 8;
    unsigned code[16][2];                // [token][columns]
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int at = r * 16 + t;
      code[t][0] = code[t][1] = 0;
      if (at < p.lo || at >= p.hi) continue;
      float v[8];
      take8<T, VEC>(rows + (at - p.lo) * ld + d, v);
      code[t][0] = pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      code[t][1] = pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    }
    if (!values) {
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int at = r * 16 + t;
        uint2* to = reinterpret_cast<uint2*>(pool + at * c.dh + d);
        if (at < p.lo) {
          if (!grown) continue;
          const uint2 w = *to;
          *to = make_uint2(rescale4(w.x, ratio), rescale4(w.y, ratio));
        } else if (at < p.hi) {
          *to = make_uint2(code[t][0], code[t][1]);
        }
      }
      continue;
    }
    const bool whole = r * 16 >= p.lo && r * 16 + 16 <= p.hi;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint8_t* to = pool + (d + e) * size + r * 16;
      unsigned w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        w[q] = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) w[q] |= (code[4 * q + t][e / 4] >> (8 * (e % 4)) & 0xffu) << (8 * t);
      }
      if (whole) {
        *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
      } else if (grown) {
        const uint4 was = *reinterpret_cast<const uint4*>(to);
        const unsigned o[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const unsigned moved = rescale4(o[q], ratio);
          unsigned out = 0;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int at = r * 16 + 4 * q + t;
            out |= (at < p.lo ? moved : at < p.hi ? w[q] : o[q]) & 0xffu << (8 * t);
          }
          w[q] = out;
        }
        *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          const int at = r * 16 + t;
          if (at >= p.lo && at < p.hi) to[t] = (uint8_t)(w[t / 4] >> (8 * (t % 4)));
        }
      }
    }
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_cache_read(CacheView c, Rows<T> x, int slots) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = ((int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x) >> 6;
  const bool values = unit & 1;
  Part p;
  if (!part_of(c, unit >> 1, slots, &p)) return;
  const int cols = c.dh / 8, size = 1 << c.shift;
  T* rows = (values ? x.v + p.row * x.ldv : x.k + p.row * x.ldk) + p.h * c.dh;
  const int64_t ld = values ? x.ldv : x.ldk, where = (int64_t)p.page * c.Hkv + p.h;
  const int first = p.lo >> 4, runs = ((p.hi + 15) >> 4) - first;
  const bool there = p.page >= 0;
  const float s = there ? (values ? c.vs : c.ks)[where] : 0.f;
  const uint8_t* pool = (values ? c.v : c.k) + (there ? where * c.dh << c.shift : 0);
  for (int i = lane; i < runs * cols; i += 64) {
    const int r = first + i / cols, d = (i % cols) * 8;
    unsigned w[8][4];                    // values: [column][tokens]
    if (values && there) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint4 q = *reinterpret_cast<const uint4*>(pool + (d + e) * size + r * 16);
        w[e][0] = q.x; w[e][1] = q.y; w[e][2] = q.z; w[e][3] = q.w;
      }
    }
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int at = r * 16 + t;
      if (at < p.lo || at >= p.hi) continue;
      float v[8];
      if (!there) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
      } else {
        unsigned a, b;
        if (values) {
          a = b = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a |= (w[e][t / 4] >> (8 * (t % 4)) & 0xffu) << (8 * e);
            b |= (w[4 + e][t / 4] >> (8 * (t % 4)) & 0xffu) << (8 * e);
          }
        } else {
          const uint2 q = *reinterpret_cast<const uint2*>(pool + at * c.dh + d);
          a = q.x;
          b = q.y;
        }
        float f[4], g[4];
        unpack4(a, f);
        unpack4(b, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = f[e] * s; v[4 + e] = g[e] * s; }
      }
      put8<T, VEC>(rows + (at - p.lo) * ld + d, v);
    }
  }
}

}  // namespace

bool cache_ok(const CacheView& c, int page) {
  if (page < 16 || page > 256 || (page & (page - 1))) return false;
  if (c.B < 0 || c.T < 1 || c.rows < 0 || c.Hkv < 1 || c.dh < 16 || c.dh > 256 || c.dh % 16) return false;
  if (c.max_pages < 1 || c.n_pages < 1 || c.B > 1 << 20 || c.T > 1 << 24 || c.Hkv > 4096) return false;
  if ((int64_t)c.max_pages * page > (int64_t)1 << 30) return false;
  if (!c.starts && (int64_t)c.B * c.T > c.rows) return false;
  return true;
}
bool cache_operands_ok(const CacheView& c) {
  return c.lens && c.table && c.k && c.v && c.ks && c.vs && (((uintptr_t)c.k | (uintptr_t)c.v) & 15) == 0;
}

namespace {
template <typename T, typename F>
hipError_t by_unit(const CacheView& c, const void* k, int64_t ldk, const void* v, int64_t ldv, F&& launch) {
  const int64_t width = (int64_t)c.Hkv * c.dh, widest = (int64_t)1 << 32;
  if (ldk < width || ldv < width || ldk > widest || ldv > widest) return hipErrorInvalidValue;
  if (c.B == 0 || c.rows == 0) return hipSuccess;
  if (!k || !v || !cache_operands_ok(c)) return hipErrorInvalidValue;
  const int slots = ((c.T + (1 << c.shift) - 2) >> c.shift) + 1;
  const int64_t blocks = ((int64_t)c.B * slots * c.Hkv * 2 + 3) / 4;
  constexpr int64_t most = 1 << 21;              // a launch has less than 2^32 threads along x
  if (blocks > most * 1024) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)((blocks + most - 1) / most));
  if (ldk % 8 == 0 && ldv % 8 == 0 && (((uintptr_t)k | (uintptr_t)v) & 15) == 0) launch(std::true_type(), grid, slots);
  else launch(std::false_type(), grid, slots);
  return hipGetLastError();
}
}  // namespace

hipError_t op_cache_append(const OpCtx& c, const CacheView& view, const void* k, int64_t ldk, const void* v, int64_t ldv) {
  auto go = [&](auto t) {
    typedef decltype(t) T;
    return by_unit<T>(view, k, ldk, v, ldv, [&](auto vec, dim3 grid, int slots) {
      k_cache_append<T, decltype(vec)::value><<<grid, 256, 0, c.stream>>>(view, Rows<const T>{(const T*)k, (const T*)v, ldk, ldv}, slots);
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

hipError_t op_cache_read(const OpCtx& c, const CacheView& view, void* k, int64_t ldk, void* v, int64_t ldv) {
  auto go = [&](auto t) {
    typedef decltype(t) T;
    return by_unit<T>(view, k, ldk, v, ldv, [&](auto vec, dim3 grid, int slots) {
      k_cache_read<T, decltype(vec)::value><<<grid, 256, 0, c.stream>>>(view, Rows<T>{(T*)k, (T*)v, ldk, ldv}, slots);
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

}  // namespace lp
