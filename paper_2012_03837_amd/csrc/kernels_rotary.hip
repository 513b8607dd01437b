// Rotary positions: neighbours (or the halves) of a head's first `rot` columns are the parts of a complex number, which is turned by the
// row's position times the pair's frequency and stretched by `scale`:
//   y = scale (a cos t - b sin t, a sin t + b cos t),  t = pos f_i;   backward: the transpose, t -> -t
// Bound by memory: every column is read and written once.  The angle is a product in 64 bits whose whole turns are taken off before it
// is cut to 32 (a position of 2^20 times 1 in 32 bits is off by 2^-5 of a radian); sines and cosines of a row are computed once, by
// the block that holds the row, and serve all its heads from LDS.  24 heads of 64 in bf16: 8192 rows 9.1 us, 5.5 TB/s; a few rows 2.4 us, the launch.
// Heads whose halves are no multiple of eight columns go element by element (2555 rows of 7 heads of 80, 40 of them turned: 5.6 us).
#include <math.h>
#include <type_traits>

#include "common.h"
#include "vec8.h"

namespace lp {

namespace {

struct RotaryArgs {
  int64_t ldx, ldy;
  const int32_t* pos;
  const double* freq;
  int rows, S, heads, dh, rot, per;      // per: rows of a block
  float scale;
  bool interleaved, back, same;          // same: y is x, columns behind rot stay
};

// VEC: sixteen bytes (bf16; thirty-two in fp32) an access, where heads, halves, rotated part and addresses are multiples of eight elements.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_rotary(const T* x, T* y, RotaryArgs a) {
  extern __shared__ float2 turn[];                      // [per][rot / 2]: cosine and sine, stretched
  const int half = a.rot / 2;
  const int64_t row0 = (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * a.per;
  const int rows = a.rows - row0 < a.per ? (int)(a.rows - row0) : a.per;       // none in the last blocks of a grid that is cut
  for (int i = threadIdx.x; i < rows * half; i += 256) {
    const int r = i / half, j = i - r * half;
    const int p = a.pos ? a.pos[row0 + r] : (int)((row0 + r) % a.S);
    const double t = (double)p * (a.freq[j] * 0.31830988618379067154);     // half turns
    float s, c;
    sincospif((float)(t - 2.0 * __builtin_rint(0.5 * t)), &s, &c);
    turn[i] = make_float2(a.scale * c, a.back ? -a.scale * s : a.scale * s);
  }
  __syncthreads();
  if constexpr (VEC) {
    // an item is eight columns of a head, or eight of each half; behind those that are turned come those that are copied
    const int turned = a.interleaved ? a.rot / 8 : half / 8, items = turned + (a.same ? 0 : (a.dh - a.rot) / 8);
    const int per_row = a.heads * items;
    for (int i = threadIdx.x; i < rows * per_row; i += 256) {
      const int r = i / per_row, h = (i - r * per_row) / items, j = i - r * per_row - h * items;
      const T* px = x + (row0 + r) * a.ldx + h * a.dh;
      T* py = y + (row0 + r) * a.ldy + h * a.dh;
      float u[8], v[8];
      if (j >= turned) {
        const int c = a.rot + (j - turned) * 8;
        load8(px + c, u);
        store8(py + c, u);
      } else if (a.interleaved) {
        const float2* t = turn + r * half + j * 4;
        load8(px + j * 8, u);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[2 * e] = u[2 * e] * t[e].x - u[2 * e + 1] * t[e].y;
          v[2 * e + 1] = u[2 * e] * t[e].y + u[2 * e + 1] * t[e].x;
        }
        store8(py + j * 8, v);
      } else {
        const float2* t = turn + r * half + j * 8;
        load8(px + j * 8, u);
        load8(px + half + j * 8, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = u[e] * t[e].x - v[e] * t[e].y;
          v[e] = u[e] * t[e].y + v[e] * t[e].x;
          u[e] = p;
        }
        store8(py + j * 8, u);
        store8(py + half + j * 8, v);
      }
    }
  } else {
    const int items = half + (a.same ? 0 : a.dh - a.rot), per_row = a.heads * items;
    for (int i = threadIdx.x; i < rows * per_row; i += 256) {
      const int r = i / per_row, h = (i - r * per_row) / items, j = i - r * per_row - h * items;
      const T* px = x + (row0 + r) * a.ldx + h * a.dh;
      T* py = y + (row0 + r) * a.ldy + h * a.dh;
      if (j >= half) {
        py[j + half] = px[j + half];
        continue;
      }
      const int c0 = a.interleaved ? 2 * j : j, c1 = a.interleaved ? c0 + 1 : c0 + half;
      const float2 t = turn[r * half + j];
      const float u = to_f(px[c0]), v = to_f(px[c1]);
      py[c0] = from_f<T>(u * t.x - v * t.y);
      py[c1] = from_f<T>(u * t.y + v * t.x);
    }
  }
}

}  // namespace

bool rotary_frequencies(double* freq, int rot, double base, double factor, double low, double high, double context) {
  if (!freq || rot < 2 || rot % 2 || !(base > 0) || !(factor > 0) || !(low <= high) || !(context >= 0) || __builtin_isinf(base) || __builtin_isinf(factor))
    return false;
  for (int i = 0; i < rot / 2; ++i) {
    const double f = pow(base, -2.0 * i / rot), turns = context * f / 6.283185307179586477;
    const double kept = turns >= high ? 1.0 : turns > low ? (turns - low) / (high - low) : 0.0;
    freq[i] = f * (kept + (1.0 - kept) / factor);
  }
  return true;
}

hipError_t op_rotary(const OpCtx& c, const void* x, int64_t ldx, void* y, int64_t ldy, const int32_t* pos, const double* freq, int rows,
                     int S, int heads, int dh, int rot, int interleaved, float scale, int backward) {
  if (rows < 0 || rows > 1 << 30 || S < 1 || heads < 1 || dh < 1 || dh > 512 || heads > (1 << 24) / dh || rot < 2 || rot > dh || rot % 2) return hipErrorInvalidValue;
  const int64_t width = (int64_t)heads * dh, widest = (int64_t)1 << 32;
  if (ldx < width || ldy < width || ldx > widest || ldy > widest || (x == y && ldx != ldy)) return hipErrorInvalidValue;
  if (rows == 0) return hipSuccess;
  if (!x || !y || !freq) return hipErrorInvalidValue;
  RotaryArgs a{ldx, ldy, pos, freq, rows, S, heads, dh, rot, 1, scale, interleaved != 0, backward != 0, x == y};
  const bool vec = dh % 8 == 0 && rot % (interleaved ? 8 : 16) == 0 && ldx % 8 == 0 && ldy % 8 == 0 && (((uintptr_t)x | (uintptr_t)y) & 15) == 0;
  // enough rows a block that its threads have three items each, while there are blocks for all compute units
  const int64_t items = vec ? width / 8 : width;
  while (a.per < 16 && a.per * items < 768 && rows / a.per > 512) a.per *= 2;
  const unsigned blocks = ((unsigned)rows + a.per - 1) / a.per;
  const size_t lds = (size_t)a.per * (rot / 2) * sizeof(float2);
  auto go = [&](auto t, auto v) {
    typedef decltype(t) T;
    constexpr unsigned most = 1u << 21;          // a launch has less than 2^32 threads along x
    k_rotary<T, decltype(v)::value><<<dim3(blocks < most ? blocks : most, (blocks + most - 1) / most), 256, lds, c.stream>>>((const T*)x, (T*)y, a);
  };
  if (c.dt == BF16) { if (vec) go(bf16_t(), std::true_type()); else go(bf16_t(), std::false_type()); }
  else { if (vec) go(float(), std::true_type()); else go(float(), std::false_type()); }
  return hipGetLastError();
}

}  // namespace lp
