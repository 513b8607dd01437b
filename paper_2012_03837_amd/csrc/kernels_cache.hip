// Writing the 8-bit cache of keys and values, and reading it back (cache.h has the layout).
//   append:  s' = max(s of the page's earlier tokens, the least power of two with max |x| / s' <= 448),  code = e4m3(x / s'); where s' > s
//            the page's earlier codes c become e4m3(c s / s')
//   read:    x = code s
// Bound by memory: one byte for every two or four.  A lane has eight columns of a run of sixteen tokens, so that both sides are read as they
// stand in the rows, and written as they stand in the page: eight bytes a token of the keys, sixteen a column of the values, transposed on the way in the
// lane's registers.  What they take, bf16: single rows of 12 heads of 64 3.0 us (the launch), 192 of 16 heads 5.6; prompts of 256 to 2048, 8 heads of
// 128 (57 MB), 17.0 us, 8 of 2048 22.3, 4.5 TB/s; reading 4 x 4096 rows of 16 heads of 64 back (101 MB) 18.1 us, 5.6 TB/s.
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
// Codes of finite numbers and NaN.
__device__ __forceinline__ unsigned pack4(float a, float b, float c, float d) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
// An infinity has no code: it is held as a NaN.
__device__ __forceinline__ float coded(float v) { return finite(v) ? v : __builtin_bit_cast(float, 0x7fc00000u); }
__device__ __forceinline__ void unpack4(unsigned w, float (&v)[4]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}
__device__ __forceinline__ unsigned rescale4(unsigned w, float ratio) {
  float v[4];
  unpack4(w, v);
  return pack4(v[0] * ratio, v[1] * ratio, v[2] * ratio, v[3] * ratio);
}

// Slot `slot` of a sequence holds the new rows row .. row + hi - lo - 1 at its tokens lo .. hi - 1.
struct Part { int page, lo, hi; int64_t row; };
__device__ __forceinline__ bool part_of(const CacheView& c, int b, int nth, Part* p) {
  const Sequence s = sequence_of(c, b);
  const int from = s.len - s.n, slot = (from >> c.shift) + nth;      // from < 0: there is no page for those rows
  const int64_t base = (int64_t)slot << c.shift;
  const int64_t lo = from > base ? from - base : 0, end = s.len - base;
  p->lo = (int)lo;
  p->hi = (int)(end < ((int64_t)1 << c.shift) ? end : (int64_t)1 << c.shift);
  p->row = s.first + (base + lo - from);
  if (p->hi <= p->lo) return false;
  p->page = page_of(c, b, slot);
  return true;
}
// The larger of two numbers that are not negative; a NaN is larger than all.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_bit_cast(unsigned, a) > __builtin_bit_cast(unsigned, b) ? a : b; }
// The largest number of the `lanes` (a power of two) lanes of a head.
__device__ __forceinline__ float max_of_head(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v = larger(v, __shfl_xor(v, o, 64));
  return v;
}
// Absolute values compare as whole numbers do; those of infinities and NaN are kInfinite and more.
constexpr unsigned kInfinite = 0x7f800000u;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
__device__ __forceinline__ unsigned largest_bits(const bf16x8& v, unsigned most) {         // most: two halves, each with the largest of every second number
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  u16x2 m = __builtin_bit_cast(u16x2, most);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const unsigned u = w[e] & 0x7fff7fffu;
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, u));
  }
  return __builtin_bit_cast(unsigned, m);
}
__device__ __forceinline__ unsigned largest_bits(const f32x8& v, unsigned most) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float f = v[e];
    const unsigned u = __builtin_bit_cast(unsigned, f) & 0x7fffffffu;
    most = u > most ? u : most;
  }
  return most;
}
template <typename T> __device__ __forceinline__ unsigned as_float_bits(unsigned most) {
  if (sizeof(T) == 4) return most;
  const unsigned a = most << 16, b = most & 0xffff0000u;
  return a > b ? a : b;
}
__device__ __forceinline__ float largest(const float (&v)[8], float most) {
#pragma unroll
  for (int e = 0; e < 8; ++e) most = finite(v[e]) ? fmaxf(most, fabsf(v[e])) : most;
  return most;
}
// Eight columns (from d on) of a run's tokens that are there already, at a larger scale; tokens from `end` (of the page) on stay as they are.
__device__ __forceinline__ void move_keys(uint8_t* pool, int dh, int d, int run, int end, float ratio) {
  const int n = end - run * 16 < 16 ? end - run * 16 : 16;
#pragma unroll 4
  for (int t = 0; t < n; ++t) {
    uint2* p = reinterpret_cast<uint2*>(pool + (run * 16 + t) * dh + d);
    const uint2 w = *p;
    *p = make_uint2(rescale4(w.x, ratio), rescale4(w.y, ratio));
  }
}
__device__ __forceinline__ void move_values(uint8_t* pool, int size, int d, int run, int end, float ratio) {
#pragma unroll 2
  for (int e = 0; e < 8; ++e) {
    uint4* p = reinterpret_cast<uint4*>(pool + (d + e) * size + run * 16);
    const uint4 was = *p;
    unsigned o[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int left = end - run * 16 - 4 * q;
      const unsigned keep = left >= 4 ? 0u : left <= 0 ? 0xffffffffu : ~((1u << (8 * left)) - 1u);
      o[q] = (rescale4(o[q], ratio) & ~keep) | (o[q] & keep);
    }
    *p = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// One new row a sequence: a wave has a side and as many heads as it has lanes for, eight columns a lane.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_cache_append_one(CacheView c, Rows<const T> x, int lanes, int groups) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned unit = (blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave, b = unit / (2 * groups), part = unit - b * 2 * groups;
  if (b >= (unsigned)c.B) return;
  const bool values = part >= (unsigned)groups;
  const int h = (int)(values ? part - groups : part) * (64 / lanes) + lane / lanes, d = (lane & (lanes - 1)) * 8;
  Part p;
  if (!part_of(c, b, 0, &p) || p.page < 0 || h >= c.Hkv) return;
  const int size = 1 << c.shift;
  const int64_t where = (int64_t)p.page * c.Hkv + h;
  float* scale = (values ? c.vs : c.ks) + where;
  uint8_t* pool = (values ? c.v : c.k) + (where * c.dh << c.shift);
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const float old = p.lo > 0 ? *scale : 0.f;
  if (d < c.dh) take8<T, VEC>((values ? x.v + p.row * x.ldv : x.k + p.row * x.ldk) + h * c.dh + d, v);
  const float need = scale_for(max_of_head(largest(v, 0.f), lanes)), s = old > need ? old : need, inv = 1.f / s;
  if (d >= c.dh) return;
  if (d == 0) *scale = s;
  if (p.lo > 0 && s > old) {
    const float ratio = old / s;
    for (int r = 0; r * 16 < p.lo; ++r) {
      if (values) move_values(pool, size, d, r, p.lo, ratio);
      else move_keys(pool, c.dh, d, r, p.lo, ratio);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = coded(v[e]) * inv;
  const unsigned a = pack4(v[0], v[1], v[2], v[3]), w = pack4(v[4], v[5], v[6], v[7]);
  if (values) {
    uint8_t* to = pool + d * size + p.lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) to[e * size] = (uint8_t)((e < 4 ? a : w) >> (8 * (e % 4)));
  } else {
    *reinterpret_cast<uint2*>(pool + p.lo * c.dh + d) = make_uint2(a, w);
  }
}

// Several: a block has a page, a side and the heads that its 64 lanes have room for; a wave of W has every W-th run of sixteen tokens.  So rows are read
// in stretches of some heads, and what a page and head takes is found in one pass over LDS.  KEEP: pages of at most W runs, whose rows stay in registers between
// the largest number and the codes; otherwise they are read twice.
template <typename T, bool VEC, bool KEEP, int W>
__global__ void __launch_bounds__(64 * W, sizeof(T) == 2 && KEEP ? 4 : 2) k_cache_append(CacheView c, Rows<const T> x, int lanes, int groups, int slots) {
  typedef __attribute__((ext_vector_type(8))) T Raw;
  __shared__ float found[W][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned unit = blockIdx.y * gridDim.x + blockIdx.x, rest = unit / (2 * groups), part = unit - rest * 2 * groups, b = rest / slots;
  if (b >= (unsigned)c.B) return;
  const bool values = part >= (unsigned)groups;
  const int h = (int)(values ? part - groups : part) * (64 / lanes) + lane / lanes, d = (lane & (lanes - 1)) * 8;
  Part p;
  if (!part_of(c, b, rest - b * slots, &p) || p.page < 0) return;
  const bool there = h < c.Hkv && d < c.dh;
  const int size = 1 << c.shift;
  const int64_t where = (int64_t)p.page * c.Hkv + (there ? h : 0);
  float* scale = (values ? c.vs : c.ks) + where;
  uint8_t* pool = (values ? c.v : c.k) + (where * c.dh << c.shift);
  const T* rows = (values ? x.v + p.row * x.ldv : x.k + p.row * x.ldk) + h * c.dh + d;
  const int64_t ld = values ? x.ldv : x.ldk;
  const float old = p.lo > 0 ? *scale : 0.f;

  Raw raw[KEEP ? 16 : 1];
  auto read = [&](int at) {
    Raw v = Raw{};
    if (there && at >= p.lo && at < p.hi) {
      if constexpr (VEC) {
        v = *reinterpret_cast<const Raw*>(rows + (at - p.lo) * ld);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = rows[(at - p.lo) * ld + e];
      }
    }
    return v;
  };
  unsigned bits = 0;
  if constexpr (KEEP) {
#pragma unroll
    for (int t = 0; t < 16; ++t) raw[t] = read(wave * 16 + t);
#pragma unroll
    for (int t = 0; t < 16; ++t) bits = largest_bits(raw[t], bits);
  } else {
    for (int r = (p.lo >> 4) + wave; r * 16 < p.hi; r += W)
#pragma unroll 4
      for (int t = 0; t < 16; ++t) bits = largest_bits(read(r * 16 + t), bits);
  }
  found[wave][lane] = max_of_head(__builtin_bit_cast(float, as_float_bits<T>(bits)), lanes);
  __syncthreads();
  float most = 0.f;
#pragma unroll
  for (int q = 0; q < W; ++q) most = larger(most, found[q][lane]);
  // with infinities or NaN among them (the same in all waves) the finite ones are looked through by themselves
  const bool odd = __ballot(__builtin_bit_cast(unsigned, most) >= kInfinite) != 0;
  if (odd) {
    most = 0.f;
    for (int r = (p.lo >> 4) / W * W + wave; r * 16 < p.hi; r += W)
#pragma unroll 1
      for (int t = 0; t < 16; ++t) {
        const Raw x = read(r * 16 + t);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = to_f(x[e]);
        most = largest(v, most);
      }
    __syncthreads();
    found[wave][lane] = max_of_head(most, lanes);
    __syncthreads();
    most = 0.f;
#pragma unroll
    for (int q = 0; q < W; ++q) most = fmaxf(most, found[q][lane]);
    if constexpr (KEEP) {
#pragma unroll
      for (int t = 0; t < 16; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) raw[t][e] = from_f<T>(coded(to_f(raw[t][e])));
    }
  }
  const float need = scale_for(most), s = old > need ? old : need, inv = 1.f / s;
  if (!there) return;
  if constexpr (KEEP && sizeof(T) == 2) {
    // the rows stay as they are stored: their numbers, twice the registers, are not kept from the pass before
    typedef __attribute__((ext_vector_type(4))) unsigned U;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      U u = __builtin_bit_cast(U, raw[t]);
      asm volatile("" : "+v"(u));
      raw[t] = __builtin_bit_cast(Raw, u);
    }
  }
  if (wave == 0 && d == 0) *scale = s;                  // the old one has been read by all: it came before the barrier
  const bool grown = p.lo > 0 && s > old;
  const float ratio = old / s;
  // runs by the same wave in both: what is there already moves first, then the new tokens come
  auto write = [&](int r) {
    if (grown && r * 16 < p.lo) {
      if (values) move_values(pool, size, d, r, p.lo, ratio);
      else move_keys(pool, c.dh, d, r, p.lo, ratio);
    }
    if (r * 16 + 16 <= p.lo) return;
    auto codes = [&](int t) {            // eight columns of a token
      Raw x;
      if constexpr (KEEP) x = raw[t];
      else x = read(r * 16 + t);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_f(x[e]);
      if constexpr (!KEEP) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = coded(v[e]);
      }
      return make_uint2(pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv), pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
    };
    if (!values) {
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int at = r * 16 + t;
        if (at >= p.lo && at < p.hi) *reinterpret_cast<uint2*>(pool + at * c.dh + d) = codes(t);
      }
      return;
    }
    unsigned w[8][4];                    // [column]: sixteen tokens
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint2 c0 = codes(4 * q), c1 = codes(4 * q + 1), c2 = codes(4 * q + 2), c3 = codes(4 * q + 3);
#pragma unroll
      for (int e = 0; e < 8; ++e) {      // byte e % 4 of four tokens
        const unsigned pick = 0x0c0c0400u + 0x0101u * (e % 4);
        w[e][q] = __builtin_amdgcn_perm(e < 4 ? c1.x : c1.y, e < 4 ? c0.x : c0.y, pick) | __builtin_amdgcn_perm(e < 4 ? c3.x : c3.y, e < 4 ? c2.x : c2.y, pick) << 16;
      }
      __builtin_amdgcn_sched_barrier(0);      // four tokens' numbers at a time in registers, not all sixteen's
    }
    const bool whole = r * 16 >= p.lo && r * 16 + 16 <= p.hi;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint8_t* to = pool + (d + e) * size + r * 16;
      if (whole) {
        *reinterpret_cast<uint4*>(to) = make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]);
      } else {
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          const int at = r * 16 + t;
          if (at >= p.lo && at < p.hi) to[t] = (uint8_t)(w[e][t / 4] >> (8 * (t % 4)));
        }
      }
    }
  };
  if constexpr (KEEP) {                  // a wave has one run: no loop that numbers could be kept for
    if (wave * 16 < p.hi) write(wave);
  } else {
    for (int r = wave + (grown ? 0 : p.lo / (16 * W) * W); r * 16 < p.hi; r += W) write(r);
  }
}

// The same blocks, waves and lanes.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_cache_read(CacheView c, Rows<T> x, int lanes, int groups, int slots) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned unit = blockIdx.y * gridDim.x + blockIdx.x, rest = unit / (2 * groups), part = unit - rest * 2 * groups, b = rest / slots;
  if (b >= (unsigned)c.B) return;
  const bool values = part >= (unsigned)groups;
  const int h = (int)(values ? part - groups : part) * (64 / lanes) + lane / lanes, d = (lane & (lanes - 1)) * 8;
  Part p;
  if (!part_of(c, b, rest - b * slots, &p) || h >= c.Hkv || d >= c.dh) return;
  const int size = 1 << c.shift;
  const bool there = p.page >= 0;
  const int64_t where = (int64_t)(there ? p.page : 0) * c.Hkv + h;
  T* rows = (values ? x.v + p.row * x.ldv : x.k + p.row * x.ldk) + h * c.dh + d;
  const int64_t ld = values ? x.ldv : x.ldk;
  const float s = (values ? c.vs : c.ks)[where];
  const uint8_t* pool = (values ? c.v : c.k) + (where * c.dh << c.shift);
  for (int r = (p.lo >> 4) + wave; r * 16 < p.hi; r += 4) {
    uint2 w[16];                         // [token]: eight columns
    if (values) {
      unsigned q[8][4];                  // [column]: sixteen tokens
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint4 f = *reinterpret_cast<const uint4*>(pool + (d + e) * size + r * 16);
        q[e][0] = f.x; q[e][1] = f.y; q[e][2] = f.z; q[e][3] = f.w;
      }
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const unsigned pick = 0x0c0c0400u + 0x0101u * (t % 4);
        auto four = [&](int e) {
          return __builtin_amdgcn_perm(q[e + 1][t / 4], q[e][t / 4], pick) | __builtin_amdgcn_perm(q[e + 3][t / 4], q[e + 2][t / 4], pick) << 16;
        };
        w[t] = make_uint2(four(0), four(4));
      }
    } else {
#pragma unroll
      for (int t = 0; t < 16; ++t) w[t] = *reinterpret_cast<const uint2*>(pool + (r * 16 + t) * c.dh + d);
    }
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int at = r * 16 + t;
      if (at < p.lo || at >= p.hi) continue;
      float f[4], g[4], v[8];
      unpack4(w[t].x, f);
      unpack4(w[t].y, g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = there ? f[e] * s : 0.f;
        v[4 + e] = there ? g[e] * s : 0.f;
      }
      put8<T, VEC>(rows + (at - p.lo) * ld, v);
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
// Lanes of a head, groups of heads, slots of a sequence that new rows may stand in, and the grid of `units` a group, side and slot to a block.
template <typename T, typename F>
hipError_t by_unit(const CacheView& c, const void* k, int64_t ldk, const void* v, int64_t ldv, int units, F&& launch) {
  const int64_t width = (int64_t)c.Hkv * c.dh, widest = (int64_t)1 << 32;
  if (ldk < width || ldv < width || ldk > widest || ldv > widest) return hipErrorInvalidValue;
  if (c.B == 0 || c.rows == 0) return hipSuccess;
  if (!k || !v || !cache_operands_ok(c)) return hipErrorInvalidValue;
  const int lanes = c.dh <= 16 ? 2 : c.dh <= 32 ? 4 : c.dh <= 64 ? 8 : c.dh <= 128 ? 16 : 32, heads = 64 / lanes, groups = (c.Hkv + heads - 1) / heads;
  const int slots = ((c.T + (1 << c.shift) - 2) >> c.shift) + 1;
  const int64_t blocks = ((int64_t)c.B * slots * groups * 2 + units - 1) / units;
  constexpr int64_t most = 1 << 21;              // a launch has less than 2^32 threads along x
  if (blocks * units > (int64_t)1 << 31) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)((blocks + most - 1) / most));
  if (ldk % 8 == 0 && ldv % 8 == 0 && (((uintptr_t)k | (uintptr_t)v) & 15) == 0) launch(std::true_type(), grid, lanes, groups, slots);
  else launch(std::false_type(), grid, lanes, groups, slots);
  return hipGetLastError();
}
}  // namespace

hipError_t op_cache_append(const OpCtx& c, const CacheView& view, const void* k, int64_t ldk, const void* v, int64_t ldv) {
  auto go = [&](auto t) {
    typedef decltype(t) T;
    const Rows<const T> x{(const T*)k, (const T*)v, ldk, ldv};
    return by_unit<T>(view, k, ldk, v, ldv, view.T == 1 ? 4 : 1, [&](auto vec, dim3 grid, int lanes, int groups, int slots) {
      constexpr bool VEC = decltype(vec)::value;
      if (view.T == 1) k_cache_append_one<T, VEC><<<grid, 256, 0, c.stream>>>(view, x, lanes, groups);
      else if (view.shift == 4) k_cache_append<T, VEC, true, 1><<<grid, 64, 0, c.stream>>>(view, x, lanes, groups, slots);
      else if (view.shift == 5) k_cache_append<T, VEC, true, 2><<<grid, 128, 0, c.stream>>>(view, x, lanes, groups, slots);
      else if (view.shift == 6) k_cache_append<T, VEC, true, 4><<<grid, 256, 0, c.stream>>>(view, x, lanes, groups, slots);
      else if (view.shift == 7) k_cache_append<T, VEC, true, 8><<<grid, 512, 0, c.stream>>>(view, x, lanes, groups, slots);
      else if constexpr (std::is_same<T, bf16_t>::value) k_cache_append<T, VEC, true, 16><<<grid, 1024, 0, c.stream>>>(view, x, lanes, groups, slots);
      else k_cache_append<T, VEC, false, 8><<<grid, 512, 0, c.stream>>>(view, x, lanes, groups, slots);      // 128 registers do not hold sixteen rows in fp32
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

hipError_t op_cache_read(const OpCtx& c, const CacheView& view, void* k, int64_t ldk, void* v, int64_t ldv) {
  auto go = [&](auto t) {
    typedef decltype(t) T;
    const Rows<T> x{(T*)k, (T*)v, ldk, ldv};
    return by_unit<T>(view, k, ldk, v, ldv, 1, [&](auto vec, dim3 grid, int lanes, int groups, int slots) {
      k_cache_read<T, decltype(vec)::value><<<grid, 256, 0, c.stream>>>(view, x, lanes, groups, slots);
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

}  // namespace lp
