// The residual chain of a decoder layer: dropout of a branch, its addition to the stream, and the root-mean-square norm of the
// sum, in one pass over the data each way.
//   forward :  r = drop(x) (+ res),  rstd = (mean r^2 + eps)^-1/2,  y = r rstd g;  8 bits: y8 = e4m3(y / s), s = max |y| / 448
//   backward:  a = g dy,  dres = rstd (a - r rstd^2 mean(a r)) (+ add),  dx = drop'(dres),  dg = sum over rows of dy r rstd
// All are bound by memory: every tensor is read or written once, 16 bytes a lane, with the row in registers between its sums and
// its outputs.  A row belongs to LPR neighbouring lanes (8 to 64: rows of up to 512 elements fill a wave with several of them, as
// the norm over a head needs) or to a block of 256 or 1024 threads.  V = 8 elements a lane and step, one where a width or an
// address does not allow that.
#include "common.h"
#include "philox.h"

namespace lp {

hipError_t op_reduce_partials(const OpCtx& c, const float* partial, int nblk, int n, float* out, int accumulate);

namespace {

// ------------------------------------------------------------------------------------------------ dropout
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_dropout(const T* x, const T* res, T* y, size_t n, Drop d) {
  const PhiloxKey key = philox_key(d);
  const size_t groups = (n + 7) / 8, step = (size_t)gridDim.x * 256;
  for (size_t g = (size_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += step) {
    const size_t i = g * 8;
    float v[8], r[8];
    if (VEC && i + 8 <= n) {
      load8(x + i, v);
      if (res) load8(res + i, r);
      if (d.thr) drop8(d, key, (unsigned)g, v);
      if (res) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += r[e];
      }
      store8(y + i, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) { v[e] = i + e < n ? to_f(x[i + e]) : 0.f; r[e] = res && i + e < n ? to_f(res[i + e]) : 0.f; }
      if (d.thr) drop8(d, key, (unsigned)g, v);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < n) y[i + e] = from_f<T>(res ? v[e] + r[e] : v[e]);
    }
  }
}

// ------------------------------------------------------------------------------------------------ rows
// Sum (or maximum) over the lanes of a row, the same in all of them.
template <int LPR, bool MAX>
__device__ __forceinline__ float row_all(float v, float* sh) {
#pragma unroll
  for (int o = (LPR < 64 ? LPR : 64) / 2; o > 0; o >>= 1) {
    const float w = __shfl_xor(v, o, 64);
    v = MAX ? (v > w || v != v ? v : w) : v + w;      // a NaN stays
  }
  if constexpr (LPR > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < LPR / 64; ++w) v = MAX ? (v > sh[w] || v != v ? v : sh[w]) : v + sh[w];
  }
  return v;
}
template <int V, typename T>
__device__ __forceinline__ void load_v(const T* p, float (&v)[V]) {
  if constexpr (V == 8) load8(p, v);
  else v[0] = to_f(*p);
}
template <int V, typename T>
__device__ __forceinline__ void store_v(T* p, const float (&v)[V]) {
  if constexpr (V == 8) store8(p, v);
  else *p = from_f<T>(v[0]);
}
template <int V>
__device__ __forceinline__ void drop_v(const Drop& d, const PhiloxKey& key, size_t i, float (&v)[V]) {
  if constexpr (V == 8) drop8(d, key, (unsigned)(i >> 3), v);
  else v[0] = drop1(d, key, i, v[0]);
}
__device__ __forceinline__ unsigned char to_e4m3(float a) {
  return (unsigned char)(__builtin_amdgcn_cvt_pk_fp8_f32(a, a, 0, false) & 0xff);
}

constexpr int threads_of(int LPR) { return LPR > 256 ? LPR : 256; }

template <typename T, int LPR, int NCH, int V>
__global__ void __launch_bounds__(threads_of(LPR)) k_rms_fwd(const T* x, const T* res, const float* __restrict__ g, T* r, T* y,
                                                             unsigned char* __restrict__ y8, float* __restrict__ y8_scale,
                                                             float* __restrict__ rstd, int rows, int d, float eps, Drop dr) {
  __shared__ float sh[16];
  constexpr int RPB = threads_of(LPR) / LPR;
  const int lane = threadIdx.x % LPR, row = blockIdx.x * RPB + threadIdx.x / LPR;
  const bool live = row < rows;                 // rows share a wave: those past the end go along in its shuffles
  const size_t base = (size_t)row * d;
  const PhiloxKey key = philox_key(dr);
  const int d_live = live ? d : 0;
  float v[NCH][V], s = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = 0.f;
    if (j < d_live) load_v<V>(x + base + j, v[i]);
  }
  if (dr.thr) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int j = (lane + LPR * i) * V;
      if (j < d_live) drop_v<V>(dr, key, base + j, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * V;
    if (j < d_live) {
      if (res) {
        float t[V];
        load_v<V>(res + base + j, t);
#pragma unroll
        for (int e = 0; e < V; ++e) v[i][e] += t[e];
      }
      if (r) store_v<V>(r + base + j, v[i]);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) s += v[i][e] * v[i][e];
  }
  // the norm is that of the sum in 32 bits, not of its stored form: one rounding less on the way to y
  const float rs = 1.f / sqrtf(row_all<LPR, false>(s, sh) / (float)d + eps);
  if (rstd && live && lane == 0) rstd[row] = rs;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * V;
    if (j < d_live) {
      float gg[V];
      load_v<V>(g + j, gg);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[i][e] = v[i][e] * rs * gg[e];
        const float a = fabsf(v[i][e]);
        top = a > top || a != a ? a : top;
      }
      if (y) store_v<V>(y + base + j, v[i]);
    }
  }
  if (!y8) return;
  top = row_all<LPR, true>(top, sh);
  // a row so small that 1 / s would overflow takes the smallest normal number
  const float least = 1.17549435e-38f, scale = top == 0.f ? 1.f : top / 448.f < least ? least : top / 448.f, inv = 1.f / scale;
  if (!live) return;
  if (lane == 0) y8_scale[row] = scale;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * V;
    if (j < d) {
      if constexpr (V == 8) {
        int w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * h] * inv, v[i][4 * h + 1] * inv, 0, false);
          w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * h + 2] * inv, v[i][4 * h + 3] * inv, w[h], true);
        }
        *reinterpret_cast<int2*>(y8 + base + j) = make_int2(w[0], w[1]);
      } else {
        y8[base + j] = to_e4m3(v[i][0] * inv);
      }
    }
  }
}

// Blocks walk over the rows with a stride and keep the sums of dg of their columns in registers; partial[block][d].
template <typename T, int LPR, int NCH, int V>
__global__ void __launch_bounds__(threads_of(LPR)) k_rms_bwd(const T* dy, const T* r, const float* __restrict__ rstd,
                                                             const float* __restrict__ g, const T* add, T* dres, T* dx,
                                                             float* __restrict__ partial, int rows, int d, Drop dr) {
  constexpr int RPB = threads_of(LPR) / LPR;
  __shared__ float sh[16];
  extern __shared__ float sums[];               // [RPB][LPR * NCH * V], where a block has several rows
  const int lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  const PhiloxKey key = philox_key(dr);
  float gg[NCH][V], pg[NCH][V];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) { pg[i][e] = 0.f; gg[i][e] = 0.f; }
    if (j < d) load_v<V>(g + j, gg[i]);
  }
  for (int row0 = blockIdx.x * RPB; row0 < rows; row0 += gridDim.x * RPB) {
    const bool live = row0 + sub < rows;
    const int row = live ? row0 + sub : rows - 1;
    const size_t base = (size_t)row * d;
    const float rs = live ? rstd[row] : 0.f;
    float xh[NCH][V], a[NCH][V], s = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int j = (lane + LPR * i) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) { xh[i][e] = 0.f; a[i][e] = 0.f; }
      if (j < d && live) { load_v<V>(r + base + j, xh[i]); load_v<V>(dy + base + j, a[i]); }
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        xh[i][e] *= rs;
        pg[i][e] += a[i][e] * xh[i][e];
        a[i][e] *= gg[i][e];
        s += a[i][e] * xh[i][e];
      }
    s = row_all<LPR, false>(s, sh) / (float)d;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int j = (lane + LPR * i) * V;
      if (j >= d) continue;
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = rs * (a[i][e] - xh[i][e] * s);
      if (add) {
        float t[V];
        load_v<V>(add + base + j, t);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] += t[e];
      }
      if (dres) store_v<V>(dres + base + j, o);
      if (dx) {
        if (dr.thr) drop_v<V>(dr, key, base + j, o);
        store_v<V>(dx + base + j, o);
      }
    }
  }
  if (!partial) return;
  float* out = partial + (size_t)blockIdx.x * d;
  if constexpr (RPB == 1) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int j = (lane + LPR * i) * V;
      if (j < d)
#pragma unroll
        for (int e = 0; e < V; ++e) out[j + e] = pg[i][e];
    }
  } else {
    constexpr int W = LPR * NCH * V;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) sums[sub * W + (lane + LPR * i) * V + e] = pg[i][e];
    __syncthreads();
    for (int j = threadIdx.x; j < d; j += 256) {
      float t = 0.f;
      for (int q = 0; q < RPB; ++q) t += sums[q * W + j];
      out[j] = t;
    }
  }
}

// Lanes and steps of a row: fn(integral constants LPR, NCH, V).
template <int N> using Int = std::integral_constant<int, N>;
constexpr int kMaxWidth = 16384;
template <typename F>
hipError_t by_width(int d, bool vec, F&& fn) {
  if (vec) {
    if (d <= 64) return fn(Int<8>(), Int<1>(), Int<8>());
    if (d <= 128) return fn(Int<16>(), Int<1>(), Int<8>());
    if (d <= 256) return fn(Int<32>(), Int<1>(), Int<8>());
    if (d <= 512) return fn(Int<64>(), Int<1>(), Int<8>());
    if (d <= 1024) return fn(Int<64>(), Int<2>(), Int<8>());
    if (d <= 2048) return fn(Int<256>(), Int<1>(), Int<8>());
    if (d <= 4096) return fn(Int<256>(), Int<2>(), Int<8>());
    if (d <= 8192) return fn(Int<256>(), Int<4>(), Int<8>());
    return fn(Int<1024>(), Int<2>(), Int<8>());
  }
  if (d <= 64) return fn(Int<64>(), Int<1>(), Int<1>());
  if (d <= 512) return fn(Int<64>(), Int<8>(), Int<1>());
  if (d <= 2048) return fn(Int<256>(), Int<8>(), Int<1>());
  return fn(Int<1024>(), Int<16>(), Int<1>());
}
template <typename... P>
bool aligned16(P... p) { return ((((uintptr_t)p) | ...) & 15) == 0; }

// Blocks of the backward kernel: enough for every compute unit to hold several, few enough for the partial sums to stay small
// beside the tensors.
int bwd_blocks(int rows, int rpb) {
  const int all = (rows + rpb - 1) / rpb;
  return all < 1024 ? all : 1024;
}

}  // namespace

size_t rmsnorm_scratch(int rows, int d) { return rows < 1 || d < 1 ? 0 : (size_t)(rows < 1024 ? rows : 1024) * d; }

hipError_t op_dropout(const OpCtx& c, const void* x, const void* res, void* y, size_t n, float p, const void* rng, unsigned site) {
  Drop d;
  if (!make_drop(p, rng, site, &d) || n > ((size_t)1 << 35)) return hipErrorInvalidValue;
  if (n == 0) return hipSuccess;
  if (!x || !y) return hipErrorInvalidValue;
  const size_t groups = (n + 7) / 8;
  const int blocks = (int)((groups + 255) / 256 < 8192 ? (groups + 255) / 256 : 8192);
  const bool vec = aligned16(x, res, y);
  auto go = [&](auto t, auto v) {
    typedef decltype(t) T;
    k_dropout<T, decltype(v)::value><<<blocks, 256, 0, c.stream>>>((const T*)x, (const T*)res, (T*)y, n, d);
  };
  if (c.dt == BF16) { if (vec) go(bf16_t(), std::true_type()); else go(bf16_t(), std::false_type()); }
  else { if (vec) go(float(), std::true_type()); else go(float(), std::false_type()); }
  return hipGetLastError();
}

hipError_t op_rmsnorm_fwd(const OpCtx& c, const void* x, const void* res, const float* g, void* r, void* y, void* y8,
                          float* y8_scale, float* rstd, int rows, int d, float eps, float p, const void* rng, unsigned site) {
  Drop dr;
  if (rows < 0 || d < 1 || d > kMaxWidth || !make_drop(p, rng, site, &dr) || (size_t)rows * d > ((size_t)1 << 35)) return hipErrorInvalidValue;
  if (rows == 0) return hipSuccess;
  if (!x || !g || (!y && !y8) || (y8 && !y8_scale)) return hipErrorInvalidValue;
  const bool vec = d % 8 == 0 && aligned16(x, res, g, r, y) && ((uintptr_t)y8 & 7) == 0;
  auto go = [&](auto t) {
    typedef decltype(t) T;
    return by_width(d, vec, [&](auto lpr, auto nch, auto v) {
      constexpr int L = decltype(lpr)::value, N = decltype(nch)::value, V = decltype(v)::value, th = threads_of(L), rpb = th / L;
      k_rms_fwd<T, L, N, V><<<(rows + rpb - 1) / rpb, th, 0, c.stream>>>((const T*)x, (const T*)res, g, (T*)r, (T*)y,
                                                                       (unsigned char*)y8, y8_scale, rstd, rows, d, eps, dr);
      return hipGetLastError();
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

hipError_t op_rmsnorm_bwd(const OpCtx& c, const void* dy, const void* r, const float* rstd, const float* g, const void* add,
                          void* dres, void* dx, float* dg, int rows, int d, int accumulate, float p, const void* rng, unsigned site) {
  Drop dr;
  if (rows < 0 || d < 1 || d > kMaxWidth || !make_drop(p, rng, site, &dr) || (size_t)rows * d > ((size_t)1 << 35)) return hipErrorInvalidValue;
  if (rows == 0) return dg && !accumulate ? op_fill_f32(c, dg, d, 0.f) : hipSuccess;
  if (!dy || !r || !rstd || !g || (!dres && !dx && !dg)) return hipErrorInvalidValue;
  if (dg && (!c.partial || c.partial_elems < rmsnorm_scratch(rows, d))) return hipErrorInvalidValue;
  const bool vec = d % 8 == 0 && aligned16(dy, r, g, add, dres, dx);
  auto go = [&](auto t) {
    typedef decltype(t) T;
    return by_width(d, vec, [&](auto lpr, auto nch, auto v) {
      constexpr int L = decltype(lpr)::value, N = decltype(nch)::value, V = decltype(v)::value, th = threads_of(L), rpb = th / L;
      const int blocks = bwd_blocks(rows, rpb);
      k_rms_bwd<T, L, N, V><<<blocks, th, rpb > 1 ? rpb * L * N * V * 4 : 0, c.stream>>>(
          (const T*)dy, (const T*)r, rstd, g, (const T*)add, (T*)dres, (T*)dx, dg ? c.partial : nullptr, rows, d, dr);
      const hipError_t e = hipGetLastError();
      return e != hipSuccess || !dg ? e : op_reduce_partials(c, c.partial, blocks, d, dg, accumulate);
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

}  // namespace lp
