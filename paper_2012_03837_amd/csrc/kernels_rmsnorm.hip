// The residual chain of a decoder layer: dropout of a branch, its addition to the stream, and the root-mean-square norm of the
// sum, in one pass over the data each way.
//   forward :  r = drop(x) (+ res),  rstd = (mean r^2 + eps)^-1/2,  y = r rstd g;  8 bits: y8 = e4m3(y / s), s = max |y| / 448
//   backward:  a = g dy,  dres = rstd (a - r rstd^2 mean(a r)) (+ add),  dx = drop'(dres),  dg = sum over rows of dy r rstd
// All are bound by memory: every tensor is read or written once, 16 bytes a lane, with the row in registers between its sums and
// its outputs.  A row belongs to LPR neighbouring lanes (8 to 32 up to 256 elements, so that several rows share a wave, as the norm over a head
// needs; 64, a wave, up to 1024) or to a block of 256 to 1024 threads.  Eight neighbouring elements a lane and step; where the
// width or an address is no multiple of them (ODD) the same accesses stand anywhere and a row's last ones are taken singly.
// What they take, bf16 (tensors' bytes over the time; 8192 rows of 4096 are 67 MB a tensor):
//   dropout and addition, 8192 x 4096, and its gradient   63.9 us, 5.2 TB/s (335 MB)
//   forward, dropout, addition, 8192 x 768                13.6 us, 3.7 TB/s; with 8-bit output, 8192 x 4096, 46 us, 5.1 TB/s
//   backward, 8192 x 768                                  14.7 us, 4.3 TB/s, and 4.0 us for the sum of dg
//   4 rows of 1024                                        3.1 us: the launch
// A copy of 4 GB reaches 4.85 TB/s here, less than what reads more than it writes; tensors of some 10 MB end before the loads are in full flight.
#include "common.h"
#include "philox.h"

namespace lp {

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
// Eight elements as they stand in memory: loads that are asked for long before they are used.  ODD: on no boundary but an element's, and
// only the first n of them there (the others are zeros); 16 bytes may be loaded from anywhere.  bf16, dropout and addition, forward, with an
// element a lane and so: 16000 rows of 1001 39 and 25 us (5.1 TB/s), 37000 of 449 42 and 26, 100000 of 65 45 and 16; backward 41 and 32, 37 and 43,
// 50 and 29.
template <typename T> struct Raw;
template <> struct Raw<bf16_t> {
  typedef bf16x8 __attribute__((aligned(2))) Anywhere;
  bf16x8 a;
  template <bool ODD> __device__ __forceinline__ void load(const bf16_t* p, int n) {
    if (!ODD) {
      a = *reinterpret_cast<const bf16x8*>(p);
    } else if (n >= 8) {
      a = *reinterpret_cast<const Anywhere*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e) {
        const bf16_t x = p[e < n ? e : 0];      // all under way at once; in branches, as fp32 has them, each waits for the half before it
        a[e] = e < n ? x : (bf16_t)0.f;
      }
    }
  }
  __device__ __forceinline__ void zero() { a = (bf16x8)(bf16_t)0.f; }
  __device__ __forceinline__ float operator[](int e) const { return (float)a[e]; }
  // what has been computed from it so far is not kept in registers (a conversion costs less than twice the registers)
  __device__ __forceinline__ void again() {
    typedef __attribute__((ext_vector_type(4))) unsigned U;
    U w = __builtin_bit_cast(U, a);
    asm volatile("" : "+v"(w));
    a = __builtin_bit_cast(bf16x8, w);
  }
};
template <> struct Raw<float> {
  typedef f32x4 __attribute__((aligned(4))) Anywhere;
  f32x4 a, b;
  template <bool ODD> __device__ __forceinline__ void load(const float* p, int n) {
    if (!ODD) {
      a = *reinterpret_cast<const f32x4*>(p);
      b = *reinterpret_cast<const f32x4*>(p + 4);
    } else if (n >= 8) {
      a = *reinterpret_cast<const Anywhere*>(p);
      b = *reinterpret_cast<const Anywhere*>(p + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (e < n) a[e] = p[e];
        if (4 + e < n) b[e] = p[4 + e];
      }
    }
  }
  __device__ __forceinline__ void zero() { a = (f32x4)0.f; b = (f32x4)0.f; }
  __device__ __forceinline__ float operator[](int e) const { return e < 4 ? a[e] : b[e - 4]; }
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(a), "+v"(b)); }
};
template <bool ODD>
__device__ __forceinline__ void store_n(bf16_t* p, const float (&v)[8], int n) {
  if (!ODD) {
    store8(p, v);
  } else if (n >= 8) {
    bf16x8 t;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = (bf16_t)v[e];
    *reinterpret_cast<Raw<bf16_t>::Anywhere*>(p) = t;
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = (bf16_t)v[e];
  }
}
template <bool ODD>
__device__ __forceinline__ void store_n(float* p, const float (&v)[8], int n) {
  if (!ODD) {
    store8(p, v);
  } else if (n >= 8) {
    *reinterpret_cast<Raw<float>::Anywhere*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<Raw<float>::Anywhere*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = v[e];
  }
}
// A row that begins inside a group of eight would draw every group twice.  Its lanes draw them once, a counter each, and
// leave them in LDS, where element j's number stands at (first & 7) + j.
template <int LPR, int NCH> struct Numbers { uint4 w[LPR * NCH + 2]; };
template <int LPR, int NCH>
__device__ __forceinline__ void draw_row(const Drop& d, const PhiloxKey& key, size_t first, int width, Numbers<LPR, NCH>& num) {
  const int groups = ((int)(first & 7) + width + 7) >> 3;
  for (int k = threadIdx.x % LPR; k < groups; k += LPR) num.w[k] = philox(key, (unsigned)(first >> 3) + k, d.site);
}
template <bool ODD, int LPR, int NCH>
__device__ __forceinline__ void drop_row(const Drop& d, const PhiloxKey& key, size_t first, int j, const Numbers<LPR, NCH>& num, float (&v)[8]) {
  if constexpr (!ODD) {
    drop8(d, key, (unsigned)((first + j) >> 3), v);
  } else {
    const unsigned short* u = reinterpret_cast<const unsigned short*>(num.w) + (first & 7) + j;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = u[e] >= d.thr ? v[e] * d.factor : 0.f;
  }
}

constexpr int threads_of(int LPR) { return LPR > 256 ? LPR : 256; }

template <typename T, int LPR, int NCH, bool ODD>
__global__ void __launch_bounds__(threads_of(LPR)) k_rms_fwd(const T* x, const T* res, const float* __restrict__ g, T* r, T* y,
                                                             unsigned char* __restrict__ y8, float* __restrict__ y8_scale,
                                                             float* __restrict__ rstd, int rows, int d, float eps, Drop dr) {
  __shared__ float sh[16];
  constexpr int RPB = threads_of(LPR) / LPR;
  __shared__ Numbers<ODD ? LPR : 0, ODD ? NCH : 0> numbers[RPB];
  auto& num = numbers[threadIdx.x / LPR];
  const int lane = threadIdx.x % LPR, row = (blockIdx.y * gridDim.x + blockIdx.x) * RPB + threadIdx.x / LPR;
  const bool live = row < rows;                 // rows share a wave: those past the end go along in its shuffles
  const size_t base = (size_t)row * d;
  const int d_live = live ? d : 0;
  Raw<T> xr[NCH], rr[NCH];
  Raw<float> gr[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * 8;
    xr[i].zero();
    rr[i].zero();
    gr[i].zero();
    if (j < d_live) {
      xr[i].template load<ODD>(x + base + j, d - j);
      if (res) rr[i].template load<ODD>(res + base + j, d - j);
      gr[i].template load<ODD>(g + j, d - j);
    }
  }
  const PhiloxKey key = philox_key(dr);
  if constexpr (ODD) {
    if (dr.thr) {
      draw_row(dr, key, base, d, num);
      __syncthreads();
    }
  }
  float v[NCH][8], s = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = xr[i][e];
    if (dr.thr && (!ODD || j < d)) drop_row<ODD>(dr, key, base, j, num, v[i]);
    if (res) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] += rr[i][e];
    }
    if (r && j < d_live) store_n<ODD>(r + base + j, v[i], d - j);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[i][e] * v[i][e];
  }
  // the norm is that of the sum in 32 bits, not of its stored form: one rounding less on the way to y
  const float rs = 1.f / sqrtf(row_all<LPR, false>(s, sh) / (float)d + eps);
  if (rstd && live && lane == 0) rstd[row] = rs;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * 8;
    if (j < d_live) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[i][e] = v[i][e] * rs * gr[i][e];
        const float a = fabsf(v[i][e]);
        top = a > top || a != a ? a : top;
      }
      if (y) store_n<ODD>(y + base + j, v[i], d - j);
    }
  }
  if (!y8) return;
  top = row_all<LPR, true>(top, sh);
  // a row so small that 1 / s would overflow takes the smallest normal number
  const float least = 1.17549435e-38f, scale = top == 0.f ? 1.f : top / 448.f < least ? least : top / 448.f, inv = 1.f / scale;
  // the quotient as rounded once: a product with the rounded 1 / s, one unit off here and there, would move values next to the middle between
  // two 8-bit ones.  Its remainder corrects it; behind an infinite scale all that is finite is 0.
  const float back = scale < INFINITY ? scale : 0.f;
  auto quotient = [&](float a) {
    const float q = a * inv;
    return __builtin_fmaf(__builtin_fmaf(-q, back, a), inv, q);
  };
  if (!live) return;
  if (lane == 0) y8_scale[row] = scale;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * 8;
    if (j < d) {
      int w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[i][4 * h]), quotient(v[i][4 * h + 1]), 0, false);
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[i][4 * h + 2]), quotient(v[i][4 * h + 3]), w[h], true);
      }
      if (!ODD) {
        *reinterpret_cast<int2*>(y8 + base + j) = make_int2(w[0], w[1]);
      } else if (d - j >= 8) {
        typedef __attribute__((ext_vector_type(2))) int I2;
        typedef I2 __attribute__((aligned(1))) Anywhere;
        *reinterpret_cast<Anywhere*>(y8 + base + j) = I2{w[0], w[1]};
      } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (j + e < d) y8[base + j + e] = (unsigned char)(w[e / 4] >> 8 * (e % 4));
      }
    }
  }
}

// Blocks walk over the rows with a stride and keep the sums of dg of their columns in registers; partial[block][d].  A row stays in
// registers as it was loaded, and where that is little enough the next one's loads are under way beside it.  Where it is not, the compiler
// puts a few of them into scratch memory, bytes a lane: bf16 of odd widths 12 from 2049 on, 28 from 4097 on, 44 from 8193 on; fp32 28 for 2049 to 4096 and 52
// from 8193 on, of odd widths 20 for 513 to 1024, 44 from 2049 on, 68 from 4097 on, 88 from 8193 on.
template <typename T, int LPR, int NCH, bool ODD>
__global__ void __launch_bounds__(threads_of(LPR), 4) k_rms_bwd(const T* dy, const T* r, const float* __restrict__ rstd,
                                                             const float* __restrict__ g, const T* add, T* dres, T* dx,
                                                             float* __restrict__ partial, int rows, int d, Drop dr) {
  constexpr int RPB = threads_of(LPR) / LPR, REGS = NCH * 2 * (int)sizeof(T);
  constexpr bool AHEAD = REGS <= 4;
  __shared__ float sh[16];
  __shared__ Numbers<ODD ? LPR : 0, ODD ? NCH : 0> numbers[RPB];
  extern __shared__ float sums[];               // [RPB][LPR * NCH * 8], where a block has several rows
  const int lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  auto& num = numbers[sub];
  struct Row { Raw<T> r[NCH], y[NCH], a[NCH]; float rs; } now, next;
  auto fetch = [&](int row, Row& to) {
    const bool live = row < rows;               // rows share a wave: those past the end go along in its shuffles
    const size_t base = (size_t)row * d;
    to.rs = live ? rstd[row] : 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int j = (lane + LPR * i) * 8;
      to.r[i].zero();
      to.y[i].zero();
      to.a[i].zero();
      if (j < d && live) {
        to.r[i].template load<ODD>(r + base + j, d - j);
        to.y[i].template load<ODD>(dy + base + j, d - j);
        if (add) to.a[i].template load<ODD>(add + base + j, d - j);
      }
    }
  };
  if (AHEAD) fetch(blockIdx.x * RPB + sub, next);
  const PhiloxKey key = philox_key(dr);
  Raw<float> gg[NCH];
  float pg[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int j = (lane + LPR * i) * 8;
    gg[i].zero();
    if (j < d) gg[i].template load<ODD>(g + j, d - j);
#pragma unroll
    for (int e = 0; e < 8; ++e) pg[i][e] = 0.f;
  }
  for (int row0 = blockIdx.x * RPB; row0 < rows; row0 += gridDim.x * RPB) {
    const int row = row0 + sub;
    const bool live = row < rows;
    const size_t base = (size_t)row * d;
    if (AHEAD) {
      now = next;
      if (row0 + (int)gridDim.x * RPB < rows) fetch(row + gridDim.x * RPB, next);
    } else {
      fetch(row, now);
    }
    const float rs = now.rs;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float yx = now.y[i][e] * (now.r[i][e] * rs);
        pg[i][e] += yx;
        s += yx * gg[i][e];
      }
    s = row_all<LPR, false>(s, sh) / (float)d;
#pragma unroll
    for (int i = 0; i < NCH; ++i) { now.r[i].again(); now.y[i].again(); now.a[i].again(); }
    if constexpr (ODD) {
      if (dx && dr.thr) {
        __syncthreads();                        // the row before has been read
        draw_row(dr, key, base, d, num);
        __syncthreads();
      }
    }
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int j = (lane + LPR * i) * 8;
      if (j >= d) continue;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = rs * (now.y[i][e] * gg[i][e] - now.r[i][e] * rs * s);
        if (add) o[e] += now.a[i][e];
      }
      if (dres) store_n<ODD>(dres + base + j, o, d - j);
      if (dx) {
        if (dr.thr) drop_row<ODD>(dr, key, base, j, num, o);
        store_n<ODD>(dx + base + j, o, d - j);
      }
    }
  }
  if (!partial) return;
  float* out = partial + (size_t)blockIdx.x * d;
  if constexpr (RPB == 1) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int j = (lane + LPR * i) * 8;
      if (j < d)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!ODD || j + e < d) out[j + e] = pg[i][e];
    }
  } else {
    constexpr int W = LPR * NCH * 8;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[sub * W + (lane + LPR * i) * 8 + e] = pg[i][e];
    __syncthreads();
    for (int j = threadIdx.x; j < d; j += 256) {
      float t = 0.f;
      for (int q = 0; q < RPB; ++q) t += sums[q * W + j];
      out[j] = t;
    }
  }
}

// dg[j] (+)= the sum of partial[0 .. nblk)[j]: 16 columns and 64 groups of rows a block, added in a fixed order (the 64 columns of
// op_reduce_partials leave 12 blocks for a width of 768, each a chain of memory latencies: 6.7 us for 1024 rows).
__global__ void __launch_bounds__(1024) k_rms_sum(const float* __restrict__ partial, int nblk, int d, float* __restrict__ dg, int accumulate) {
  __shared__ float sh[64][17];
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4, j = blockIdx.x * 16 + c;
  float t = 0.f;
  if (j < d) {
    constexpr int U = 8;
    for (int b = q; b < nblk; b += 64 * U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = b + 64 * u < nblk ? partial[(size_t)(b + 64 * u) * d + j] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) t += v[u];
    }
  }
  sh[q][c] = t;
  __syncthreads();
  if (q < 8) {
    t = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) t += sh[8 * q + u][c];
    sh[8 * q][c] = t;
  }
  __syncthreads();
  if (q == 0 && j < d) {
    t = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) t += sh[8 * u][c];
    dg[j] = accumulate ? dg[j] + t : t;
  }
}

// Lanes and steps of a row: fn(integral constants LPR, NCH, ODD).
template <int N> using Int = std::integral_constant<int, N>;
constexpr int kMaxWidth = 16384;
bool shape_ok(int rows, int d) { return rows >= 0 && rows <= 1 << 30 && d >= 1 && d <= kMaxWidth && (size_t)rows * d <= (size_t)1 << 35; }
template <typename F>
hipError_t by_width(int d, bool vec, F&& fn) {
  // The rows' ends make the slowest wave of an odd row, and blocks of 1024 leave few others beside it (4000 rows of 8191, bf16, forward
  // 47 us with blocks of 512, 73 with 1024).
  auto go = [&](auto odd) {
    constexpr bool ODD = decltype(odd)::value;
    if (d <= 64) return fn(Int<8>(), Int<1>(), odd);
    if (d <= 128) return fn(Int<16>(), Int<1>(), odd);
    if (d <= 256) return fn(Int<32>(), Int<1>(), odd);
    if (d <= 512) return fn(Int<64>(), Int<1>(), odd);
    if (d <= 1024) return fn(Int<64>(), Int<2>(), odd);
    if (d <= 2048) return fn(Int<256>(), Int<1>(), odd);
    if (d <= 4096) return fn(Int<256>(), Int<2>(), odd);
    if (d <= 8192) return fn(Int<ODD ? 512 : 1024>(), Int<ODD ? 2 : 1>(), odd);
    return fn(Int<1024>(), Int<2>(), odd);
  };
  return vec ? go(std::false_type()) : go(std::true_type());
}
template <typename... P>
bool aligned16(P... p) { return ((((uintptr_t)p) | ...) & 15) == 0; }

// Blocks of the backward kernel: as many as the chip holds at once (four waves a SIMD), each with several rows where there are more,
// so that the partial sums stay small beside the tensors.
int bwd_blocks(int rows, int rpb, int lpr) {
  const int all = (rows + rpb - 1) / rpb, most = 262144 / (lpr > 256 ? lpr : 256);
  if (all <= most) return all;
  const int each = (all + most - 1) / most;      // the same number of rows for all
  return (all + each - 1) / each;
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
  if (!shape_ok(rows, d) || !make_drop(p, rng, site, &dr)) return hipErrorInvalidValue;
  if (rows == 0) return hipSuccess;
  if (!x || !g || (!y && !y8) || (y8 && !y8_scale)) return hipErrorInvalidValue;
  const bool vec = d % 8 == 0 && aligned16(x, res, g, r, y) && ((uintptr_t)y8 & 7) == 0;
  auto go = [&](auto t) {
    typedef decltype(t) T;
    return by_width(d, vec, [&](auto lpr, auto nch, auto odd) {
      constexpr int L = decltype(lpr)::value, N = decltype(nch)::value, th = threads_of(L), rpb = th / L;
      constexpr bool ODD = decltype(odd)::value;
      constexpr int most = 1 << 21;              // a launch has less than 2^32 threads along x
      const int blocks = (rows + rpb - 1) / rpb;
      k_rms_fwd<T, L, N, ODD><<<dim3(blocks < most ? blocks : most, (blocks + most - 1) / most), th, 0, c.stream>>>(
          (const T*)x, (const T*)res, g, (T*)r, (T*)y, (unsigned char*)y8, y8_scale, rstd, rows, d, eps, dr);
      return hipGetLastError();
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

hipError_t op_rmsnorm_bwd(const OpCtx& c, const void* dy, const void* r, const float* rstd, const float* g, const void* add,
                          void* dres, void* dx, float* dg, int rows, int d, int accumulate, float p, const void* rng, unsigned site) {
  Drop dr;
  if (!shape_ok(rows, d) || !make_drop(p, rng, site, &dr)) return hipErrorInvalidValue;
  if (rows == 0) return dg && !accumulate ? op_fill_f32(c, dg, d, 0.f) : hipSuccess;
  if (!dy || !r || !rstd || !g || (!dres && !dx && !dg)) return hipErrorInvalidValue;
  if (dg && (!c.partial || c.partial_elems < rmsnorm_scratch(rows, d))) return hipErrorInvalidValue;
  const bool vec = d % 8 == 0 && aligned16(dy, r, g, add, dres, dx);
  auto go = [&](auto t) {
    typedef decltype(t) T;
    return by_width(d, vec, [&](auto lpr, auto nch, auto odd) {
      constexpr int L = decltype(lpr)::value, N = decltype(nch)::value, th = threads_of(L), rpb = th / L;
      constexpr bool ODD = decltype(odd)::value;
      const int blocks = bwd_blocks(rows, rpb, L);
      k_rms_bwd<T, L, N, ODD><<<blocks, th, rpb > 1 ? rpb * L * N * 8 * 4 : 0, c.stream>>>(
          (const T*)dy, (const T*)r, rstd, g, (const T*)add, (T*)dres, (T*)dx, dg ? c.partial : nullptr, rows, d, dr);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess || !dg) return e;
      k_rms_sum<<<(d + 15) / 16, 1024, 0, c.stream>>>(c.partial, blocks, d, dg, accumulate);
      return hipGetLastError();
    });
  };
  return c.dt == BF16 ? go(bf16_t()) : go(float());
}

}  // namespace lp
