// Linear attention with a decay for each head.  With l = exp(log_decay[h]) and the state S [dh, dh] in fp32,
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = dh^-1/2 q_t S_t   (position t included).
// Chunks of 64 positions: with X the state before a chunk, u = 0 .. 63 the position in it and e = 1,
//   O = dh^-1/2 ( ((Q K^T) . D) V + diag(l^{u + e}) Q X ),  D[u, w] = l^{u - w} for w <= u, otherwise 0,
//   X' = l^c X + sum_u l^{c - u - e} k_u v_u^T              (c: positions of the chunk, 64 but for the last).
// The gradients are the same map of other operands, so that one kernel serves both directions:
//   dQ = map(q <- dO, k <- V, v <- K),
//   dV = map(q <- K, k <- Q, v <- dO) and dK = map(q <- V, k <- dO, v <- Q) with the positions taken from the last to the first
//   and e = 0, where X' = sum l^{distance past the chunk} q dO^T is the gradient of the state.
// A long axis over few heads is cut into segments of whole chunks: k_linear_states leaves what each adds to the state,
// k_linear_scan turns that into the state before each, and the blocks of k_linear_walk go over their segments side by side.
//
// Products run on the matrix cores, 32 x 32 tiles; as in the softmax kernels the score tile is kept transposed, because the
// accumulators of K Q^T are the operand layout of the product behind it.  The state lives in fp32 accumulators, a 32 x 32 tile of it in
// each wave.  Whatever has more bits than the compute dtype (scores times decay, keys times decay, the state as an operand) is
// split into two bf16 parts (three where the state itself is an output): the parts' products are exact and summed in fp32.  With one part
// alone every such rounding adds an error as large as that of the rounded output.
#include "common.h"
#include "gemm_common.h"

namespace lp {

namespace {

constexpr int kChunk = 64;
constexpr float kLog2e = 1.4426950408889634f;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

// Eight values of the reduction index in a lane: the operand of one 16-deep product.
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { typedef bf16x8 V; };
template <> struct Frag<float> { typedef f32x8 V; };
__device__ __forceinline__ f32x16 mma(const bf16x8& a, const bf16x8& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const f32x8& a, const f32x8& b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ bf16x8 frag_row(const bf16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ f32x8 frag_row(const float* p) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
  f32x8 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) { r[e] = a[e]; r[4 + e] = b[e]; }
  return r;
}
// Operand whose reduction index is the row of an LDS tile: lane (n, hf) gets column c0 + n of rows r0 + 4 hf + {0..3} and
// r0 + 8 + 4 hf + {0..3}, the order of an accumulator's values; bf16 by the transposing read (its 16-lane groups: lane 4 r + c
// supplies four columns 4 c .. of row r and lane 4 c + e receives column 4 c + e of the four rows).
template <int LD>
__device__ __forceinline__ bf16x8 frag_col(const bf16_t (*s)[LD], int r0, int c0, int lane) {
  const int g = lane >> 4, l16 = lane & 15, hf = g >> 1;
  const bf16_t* p = &s[r0 + 4 * hf + (l16 >> 2)][c0 + 16 * (g & 1) + 4 * (l16 & 3)];
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p));
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 8 * LD));
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) { r[e] = lo[e]; r[4 + e] = hi[e]; }
  return r;
}
template <int LD>
__device__ __forceinline__ f32x8 frag_col(const float (*s)[LD], int r0, int c0, int lane) {
  const int n = lane & 31, hf = lane >> 5;
  f32x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = s[r0 + 8 * (e / 4) + 4 * hf + e % 4][c0 + n];
  return r;
}
// fp32 values as NP operands whose sum they are (to 2^-8 NP); one where the compute dtype is fp32.
template <int NP>
__device__ __forceinline__ void split(const f32x8& v, bf16x8 (&f)[NP]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float r = v[e];
#pragma unroll
    for (int s = 0; s < NP; ++s) { f[s][e] = (bf16_t)r; r -= (float)f[s][e]; }
  }
}
__device__ __forceinline__ void split(const f32x8& v, f32x8 (&f)[1]) { f[0] = v; }
template <typename V, int NP>
__device__ __forceinline__ f32x16 mma_parts(const V (&a)[NP], const V& b, f32x16 c) {      // smallest first
#pragma unroll
  for (int s = NP - 1; s >= 0; --s) c = mma(a[s], b, c);
  return c;
}
__device__ __forceinline__ void zero(f32x16& a) {
#pragma unroll
  for (int i = 0; i < 16; ++i) a[i] = 0.f;
}
// l^n, n >= 0; l^0 is 1 also for a decay to nothing (log_decay = -inf, which comes in as a large finite number)
__device__ __forceinline__ float power(float g2, int n) { return __builtin_amdgcn_exp2f(g2 * (float)n); }
__device__ __forceinline__ float decay_of(const float* log_decay, int h) {
  const float g = log_decay[h];
  return (g < -1e4f ? -1e4f : g) * kLog2e;
}

template <typename T> constexpr int kPerChunk = 16 / (int)sizeof(T);     // elements of a 16-byte load

// [64 rows][W columns] of a matrix on the way into LDS, in registers while the chunk before it is computed.  Rows from `rows`
// on and columns from `cols` on are zeros (and not read).  VEC: rows are whole 16-byte chunks on 16-byte boundaries.
template <typename T, int W, int NT, bool VEC>
struct TileRegs {
  static constexpr int E = kPerChunk<T>, CPR = W / E, N = (kChunk * CPR + NT - 1) / NT;
  static_assert(kChunk * CPR % NT == 0, "whole loads");
  typedef __attribute__((ext_vector_type(E))) T V;
  V v[N];
  __device__ __forceinline__ void load(const T* p, ptrdiff_t ld, int rows, int cols) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = threadIdx.x + NT * i, r = x / CPR, c = x % CPR * E;
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] = (T)0.f;
      if (r < rows) {
        const T* q = p + (ptrdiff_t)r * ld + c;
        if (VEC) {
          if (c < cols) v[i] = *reinterpret_cast<const V*>(q);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (c + e < cols) v[i][e] = q[e];
        }
      }
    }
  }
  template <int LD>
  __device__ __forceinline__ void store(T (*s)[LD]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = threadIdx.x + NT * i;
      *reinterpret_cast<V*>(&s[x / CPR][x % CPR * E]) = v[i];
    }
  }
  __device__ __forceinline__ bool non_finite() const {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) bad = bad || !(__builtin_fabsf((float)v[i][e]) < INFINITY);
    return bad;
  }
};

// One application of the map to all heads: matrices at head 0, row strides, and the states.
struct LinearJob {
  const void *q, *k, *v;
  void* out;
  int64_t ldq, ldk, ldv, ldo;      // elements
  const float* init;               // state that came in ([B, H, dh, dh], null: zeros), times in_scale, transposed if `turned`
  float* fin;                      // state that goes out, times out_scale (null: not wanted)
  const float* before;             // states before the segments ([B H, segments, dh, dh]), transposed if `turned`
  float in_scale, out_scale;
  int turned, back;                // back: positions from the last to the first, e = 0
};
constexpr int kJobs = 3;
struct LinearJobs { LinearJob j[kJobs]; };
struct LinearShape {
  int B, S, H, dh, segments, per;  // per: chunks of a segment
  float scale;
  const float* log_decay;
  const int32_t* lens;
  __device__ int length(int b) const {
    if (!lens) return S;
    const int n = lens[b];
    return n < 0 ? 0 : n > S ? S : n;
  }
};

// The state's tiles: wave w holds rows 32 (w & 1) (and + 64) and columns 32 (w >> 1).
template <int DK> constexpr int kTiles = DK == 128 ? 2 : 1;

// acc += sum over the chunk's positions of weight * k v^T, for the wave's tiles.
template <typename T, int DK, int NP, int LDK, int LDV>
__device__ __forceinline__ void add_outer(f32x16 (&state)[kTiles<DK>], const T (*ks)[LDK], const T (*vs)[LDV], const float* weight, int ib,
                                          int jb, int lane) {
  const int hf = lane >> 5;
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const typename Frag<T>::V b = frag_col<LDV>(vs, 16 * kk, 32 * jb, lane);
    f32x8 w;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(weight + 16 * kk + 8 * x + 4 * hf);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * x + e] = t[e];
    }
#pragma unroll
    for (int i = 0; i < kTiles<DK>; ++i) {
      const typename Frag<T>::V a = frag_col<LDK>(ks, 16 * kk, 32 * ib + 64 * i, lane);
      f32x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (float)a[e] * w[e];
      typename Frag<T>::V f[NP];
      split(p, f);
      state[i] = mma_parts(f, b, state[i]);
    }
  }
}

template <typename T, int DK, int DV, int NP>
struct WalkLds {
  __attribute__((aligned(16))) T k[kChunk][DK + 8];
  __attribute__((aligned(16))) T v[kChunk][DV + 8];
  __attribute__((aligned(16))) T state[NP][DV][DK + 8];      // transposed: columns of the state are rows here
  __attribute__((aligned(16))) float weight[kChunk];
  int bad;
};

// A block: one segment of one head and 32 or 64 columns of the state.  Waves share the chunk's queries (halves w & 1) and the columns
// (halves w >> 1).
template <typename T, int DK, int DV, bool VEC, bool FIN>
__global__ void __launch_bounds__(4 * DV) k_linear_walk(LinearJobs jobs, LinearShape sh, int units, int cols, int njobs) {
  constexpr int NT = 4 * DV, NP = sizeof(T) == 2 ? 2 : 1, NPS = sizeof(T) == 2 ? (FIN ? 3 : 2) : 1, NK = DK / 16, NTL = kTiles<DK>;
  typedef typename Frag<T>::V FV;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  WalkLds<T, DK, DV, NP>& sm = *reinterpret_cast<WalkLds<T, DK, DV, NP>*>(smem);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hf = lane >> 5;
  const int qb = wave & 1, jb = wave >> 1;
  // Blocks go to the eight dies by turns of their number: those that share a segment's rows are eight apart, on one die.
  const int subs = cols * njobs, group = blockIdx.x / (8 * subs), rest = blockIdx.x % (8 * subs);
  const int unit = group * 8 + rest % 8, sub = rest / 8;
  if (unit >= units) return;
  const LinearJob& job = jobs.j[sub / cols];
  const int col0 = sub % cols * DV;
  const int seg = unit % sh.segments, bh = unit / sh.segments, h = bh % sh.H, b = bh / sh.H, dh = sh.dh;
  const int len = sh.length(b), first = seg * sh.per * kChunk;
  const int last = first + sh.per * kChunk < sh.S ? first + sh.per * kChunk : sh.S;       // of the segment, padding included
  const int stop = last < len ? last : len;
  const float g2 = decay_of(sh.log_decay, h);
  const int e0 = job.back ? 0 : 1;
  const int hcols = dh - col0 < DV ? dh - col0 : DV;           // columns of the block that exist
  // position u of the walk is row `at + u * dir`
  const ptrdiff_t dir = job.back ? -1 : 1;
  const size_t at = (size_t)b * sh.S + (job.back && len > 0 ? len - 1 : 0);
  const T* qp = (const T*)job.q + (ptrdiff_t)at * job.ldq + h * dh;
  const T* kp = (const T*)job.k + (ptrdiff_t)at * job.ldk + h * dh;
  const T* vp = (const T*)job.v + (ptrdiff_t)at * job.ldv + h * dh + col0;
  T* op = (T*)job.out + (ptrdiff_t)at * job.ldo + h * dh + col0;

  // rows of the padding are zeros, whatever stands there in the inputs
  {
    T* pad = (T*)job.out + ((size_t)b * sh.S) * job.ldo + h * dh + col0;
    const int from = first > len ? first : len;
    for (int x = threadIdx.x; x < (last - from) * DV; x += NT)
      if (x % DV < hcols) pad[(ptrdiff_t)(from + x / DV) * job.ldo + x % DV] = (T)0.f;
  }

  f32x16 state[NTL];
  auto state_row = [&](int i, int v) { return 32 * qb + 64 * i + 8 * (v / 4) + 4 * hf + v % 4; };
  const int scol = col0 + 32 * jb + n;
  const bool owner = 32 * qb < DK;                             // heads of 32: the first of two waves holds the one tile
  {
    const bool whole = job.before != nullptr;
    const float* x0 = whole ? job.before + ((size_t)bh * sh.segments + seg) * dh * dh : job.init ? job.init + (size_t)bh * dh * dh : nullptr;
    const float f = whole ? 1.f : job.in_scale;
#pragma unroll
    for (int i = 0; i < NTL; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = state_row(i, v);
        state[i][v] = 0.f;
        if (x0 && r < dh && scol < dh) state[i][v] = f * (job.turned ? x0[(size_t)scol * dh + r] : x0[(size_t)r * dh + scol]);
      }
  }
  auto publish = [&]() {                                       // the state as an operand, for all waves
    if (!owner) return;
#pragma unroll
    for (int i = 0; i < NTL; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        typedef __attribute__((ext_vector_type(4))) T T4;
        T4 part[NP];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float r = state[i][4 * g + j];
#pragma unroll
          for (int s = 0; s < NP; ++s) { part[s][j] = (T)r; r -= (float)part[s][j]; }
        }
#pragma unroll
        for (int s = 0; s < NP; ++s) *reinterpret_cast<T4*>(&sm.state[s][32 * jb + n][state_row(i, 4 * g)]) = part[s];
      }
  };

  // decay between a query and the keys of its own 32 positions (nothing above the diagonal) and of the 32 before
  float near[16], far[16];
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int r = 8 * (v / 4) + 4 * hf + v % 4;
    near[v] = r <= n ? power(g2, n - r) * sh.scale : 0.f;
    far[v] = power(g2, 32 + n - r) * sh.scale;
  }
  const float carry = power(g2, 32 * qb + n + e0) * sh.scale;

  TileRegs<T, DK, NT, VEC> kr;
  TileRegs<T, DV, NT, VEC> vr;
  FV qf[NK], qn[NK];
  auto fetch = [&](int u0) {
    const int rows = stop - u0;
    kr.load(kp + (ptrdiff_t)u0 * dir * job.ldk, dir * job.ldk, rows, dh);
    vr.load(vp + (ptrdiff_t)u0 * dir * job.ldv, dir * job.ldv, rows, hcols);
    const int u = 32 * qb + n;
    const T* q = qp + (ptrdiff_t)(u0 + u) * dir * job.ldq;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      const int c = 16 * kk + 8 * hf;
#pragma unroll
      for (int e = 0; e < 8; ++e) qn[kk][e] = (T)0.f;
      if (u < rows) {
        if (VEC) {
          if (c < dh) qn[kk] = frag_row(q + c);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < dh) qn[kk][e] = q[c + e];
        }
      }
    }
  };
  if (first < stop) fetch(first);
  if (threadIdx.x == 0) sm.bad = -1;
  int counted = -1;
  for (int u0 = first; u0 < stop; u0 += kChunk) {
    const int c = stop - u0 < kChunk ? stop - u0 : kChunk;
    __syncthreads();                                           // the chunk before has been read
    kr.store(sm.k);
    vr.store(sm.v);
    if (vr.non_finite()) sm.bad = u0;
    publish();
    if (c != counted && threadIdx.x < kChunk) sm.weight[threadIdx.x] = (int)threadIdx.x < c ? power(g2, c - threadIdx.x - e0) : 0.f;
    counted = c;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) qf[kk] = qn[kk];
    __syncthreads();
    if (u0 + kChunk < stop) fetch(u0 + kChunk);
    const bool slow = sm.bad == u0;

    // what the earlier chunks give
    f32x16 o;
    zero(o);
#pragma unroll
    for (int s = NP - 1; s >= 0; --s)
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) o = mma(frag_row(&sm.state[s][32 * jb + n][16 * kk + 8 * hf]), qf[kk], o);
#pragma unroll
    for (int v = 0; v < 16; ++v) o[v] *= carry;
    if (!slow) {
      // and the chunk itself; the scores above the diagonal are left out by choice and not by a product with 0, so that an
      // infinity or a NaN in a later key reaches nobody
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i > qb) break;
        f32x16 p;
        zero(p);
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) p = mma(frag_row(&sm.k[32 * i + n][16 * kk + 8 * hf]), qf[kk], p);
        const bool diagonal = i == qb;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          f32x8 w;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int v = 8 * kk + e, r = 8 * (v / 4) + 4 * hf + v % 4;
            w[e] = diagonal ? (r <= n ? p[v] * near[v] : 0.f) : p[v] * far[v];
          }
          FV f[NP];
          split(w, f);
          const FV a = frag_col<DV + 8>(sm.v, 32 * i + 16 * kk, 32 * jb, lane);
#pragma unroll
          for (int s = NP - 1; s >= 0; --s) o = mma(a, f[s], o);
        }
      }
    } else {
      // A chunk with an infinity or a NaN among its values: row by row, the later ones left out (0 times infinity is not 0).
#pragma unroll 1
      for (int r = 0; r < c; ++r) {
        float s = 0.f;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
#pragma unroll
          for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)qf[kk][e], (float)sm.k[r][16 * kk + 8 * hf + e], s);
        s += __shfl_xor(s, 32, 64);
        const int away = 32 * qb + n - r;
        if (away < 0) continue;
        s *= power(g2, away) * sh.scale;
#pragma unroll
        for (int v = 0; v < 16; ++v) o[v] = __builtin_fmaf(s, (float)sm.v[r][32 * jb + 8 * (v / 4) + 4 * hf + v % 4], o[v]);
      }
    }
    if (u0 + 32 * qb + n < stop) {
      T* p = op + (ptrdiff_t)(u0 + 32 * qb + n) * dir * job.ldo + 32 * jb;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        typedef __attribute__((ext_vector_type(4))) T T4;
        const int x = 8 * g + 4 * hf;
        T4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (T)o[4 * g + j];
        if (VEC) {
          if (32 * jb + x < hcols) *reinterpret_cast<T4*>(p + x) = w;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (32 * jb + x + j < hcols) p[x + j] = w[j];
        }
      }
    }
    if (owner && (FIN || u0 + kChunk < stop)) {
      const float keep = power(g2, c);
#pragma unroll
      for (int i = 0; i < NTL; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) state[i][v] *= keep;
      add_outer<T, DK, NPS, DK + 8, DV + 8>(state, sm.k, sm.v, sm.weight, qb, jb, lane);
    }
  }
  if (FIN && job.fin && owner) {
    float* out = job.fin + (size_t)bh * dh * dh;
#pragma unroll
    for (int i = 0; i < NTL; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = state_row(i, v);
        if (r < dh && scol < dh) out[(size_t)r * dh + scol] = state[i][v] * job.out_scale;
      }
  }
}

// What a segment adds to the state: loc [B H, segments, dh, dh] for each job.  The last segment is needed only for the state that goes
// out.  A block takes 64 columns.
struct StateJob {
  const void *k, *v;
  int64_t ldk, ldv;
  float* loc;
  const float* init;
  float* fin;
  float in_scale, out_scale;
  int back;
};
struct StateJobs { StateJob j[2]; };

template <typename T, int DK, int DV, bool VEC>
__global__ void __launch_bounds__(4 * DV) k_linear_states(StateJobs jobs, LinearShape sh, int units, int cols, int njobs) {
  constexpr int NT = 4 * DV, NPS = sizeof(T) == 2 ? 3 : 1, NTL = kTiles<DK>;
  __shared__ __attribute__((aligned(16))) T ks[kChunk][DK + 8], vs[kChunk][DV + 8];
  __shared__ __attribute__((aligned(16))) float weight[kChunk];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hf = lane >> 5;
  const int ib = wave & 1, jb = wave >> 1;
  const int subs = cols * njobs, group = blockIdx.x / (8 * subs), rest = blockIdx.x % (8 * subs);
  const int unit = group * 8 + rest % 8, sub = rest / 8;
  if (unit >= units) return;
  const StateJob& job = jobs.j[sub / cols];
  const int col0 = sub % cols * DV;
  const int seg = unit % sh.segments, bh = unit / sh.segments, h = bh % sh.H, b = bh / sh.H, dh = sh.dh;
  if (seg == sh.segments - 1 && !job.fin) return;
  const int len = sh.length(b), first = seg * sh.per * kChunk;
  const int stop = first + sh.per * kChunk < len ? first + sh.per * kChunk : len;
  const float g2 = decay_of(sh.log_decay, h);
  const int e0 = job.back ? 0 : 1;
  const int hcols = dh - col0 < DV ? dh - col0 : DV;
  const ptrdiff_t dir = job.back ? -1 : 1;
  const size_t at = (size_t)b * sh.S + (job.back && len > 0 ? len - 1 : 0);
  const T* kp = (const T*)job.k + (ptrdiff_t)at * job.ldk + h * dh;
  const T* vp = (const T*)job.v + (ptrdiff_t)at * job.ldv + h * dh + col0;
  const bool owner = 32 * ib < DK;
  f32x16 state[NTL];
#pragma unroll
  for (int i = 0; i < NTL; ++i) zero(state[i]);
  TileRegs<T, DK, NT, VEC> kr;
  TileRegs<T, DV, NT, VEC> vr;
  auto fetch = [&](int u0) {
    kr.load(kp + (ptrdiff_t)u0 * dir * job.ldk, dir * job.ldk, stop - u0, dh);
    vr.load(vp + (ptrdiff_t)u0 * dir * job.ldv, dir * job.ldv, stop - u0, hcols);
  };
  if (first < stop) fetch(first);
  for (int u0 = first; u0 < stop; u0 += kChunk) {
    const int c = stop - u0 < kChunk ? stop - u0 : kChunk;
    __syncthreads();
    kr.store(ks);
    vr.store(vs);
    if (threadIdx.x < kChunk) weight[threadIdx.x] = (int)threadIdx.x < c ? power(g2, c - threadIdx.x - e0) : 0.f;
    __syncthreads();
    if (u0 + kChunk < stop) fetch(u0 + kChunk);
    if (owner) {
      const float keep = power(g2, c);
#pragma unroll
      for (int i = 0; i < NTL; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) state[i][v] *= keep;
      add_outer<T, DK, NPS, DK + 8, DV + 8>(state, ks, vs, weight, ib, jb, lane);
    }
  }
  if (!owner) return;
  float* out = job.loc + ((size_t)bh * sh.segments + seg) * dh * dh;
  const int scol = col0 + 32 * jb + n;
#pragma unroll
  for (int i = 0; i < NTL; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int r = 32 * ib + 64 * i + 8 * (v / 4) + 4 * hf + v % 4;
      if (r < dh && scol < dh) out[(size_t)r * dh + scol] = state[i][v];
    }
}

// In place: what a segment adds becomes the state before it.  One thread an element of the state.
__global__ void __launch_bounds__(256) k_linear_scan(StateJobs jobs, LinearShape sh) {
  const StateJob& job = jobs.j[blockIdx.z];
  const int bh = blockIdx.y, x = blockIdx.x * 256 + threadIdx.x, dd = sh.dh * sh.dh;
  if (x >= dd) return;
  const float g2 = decay_of(sh.log_decay, bh % sh.H);
  const int len = sh.length(bh / sh.H), span = sh.per * kChunk;
  float s = job.init ? job.init[(size_t)bh * dd + x] * job.in_scale : 0.f;
  float* p = job.loc + (size_t)bh * sh.segments * dd + x;
  constexpr int U = 8;                         // loads in flight
  for (int g = 0; g < sh.segments; g += U) {
    float add[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const bool there = g + i < sh.segments - 1 || (g + i == sh.segments - 1 && job.fin);
      add[i] = there ? p[(size_t)(g + i) * dd] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (g + i >= sh.segments) break;
      p[(size_t)(g + i) * dd] = s;
      const int left = len - (g + i) * span, c = left < 0 ? 0 : left < span ? left : span;
      s = power(g2, c) * s + add[i];
    }
  }
  if (job.fin) job.fin[(size_t)bh * dd + x] = s * job.out_scale;
}

// One position: the state is read, decayed, added to and written back; a wave takes `rows` of its rows at a time.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_step(const T* __restrict__ qkv, const float* __restrict__ log_decay, float* __restrict__ state,
                                                     T* __restrict__ o, int H, int dh, float scale) {
  __shared__ float q[128], k[128], v[128], part[256][4];
  const int bh = blockIdx.x, h = bh % H, b = bh / H;
  const T* row = qkv + (size_t)b * 3 * H * dh + h * dh;
  if ((int)threadIdx.x < dh) {
    q[threadIdx.x] = to_f(row[threadIdx.x]);
    k[threadIdx.x] = to_f(row[H * dh + threadIdx.x]);
    v[threadIdx.x] = to_f(row[2 * H * dh + threadIdx.x]);
  }
  const float l = power(decay_of(log_decay, h), 1);
  float* s = state + (size_t)bh * dh * dh;
  __syncthreads();
  const int per = (dh + 3) / 4, rows = 256 / per, c = threadIdx.x % per * 4, r0 = threadIdx.x / per;     // threads of a row
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  if (r0 < rows) {
    if (dh % 4 == 0 && ((uintptr_t)state & 15) == 0) {
      constexpr int U = 4;
      for (int r = r0; r < dh; r += U * rows) {
        f32x4 x[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (r + i * rows < dh) x[i] = *reinterpret_cast<const f32x4*>(s + (size_t)(r + i * rows) * dh + c);
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int rr = r + i * rows;
          if (rr < dh) {
            const float kr = k[rr], qr = q[rr];
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[i][e] = l * x[i][e] + kr * v[c + e]; acc[e] += qr * x[i][e]; }
            *reinterpret_cast<f32x4*>(s + (size_t)rr * dh + c) = x[i];
          }
        }
      }
    } else {
      for (int r = r0; r < dh; r += rows)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < dh) {
            const float x = l * s[(size_t)r * dh + c + e] + k[r] * v[c + e];
            s[(size_t)r * dh + c + e] = x;
            acc[e] += q[r] * x;
          }
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) part[threadIdx.x][e] = acc[e];
  __syncthreads();
  if ((int)threadIdx.x < dh) {
    float t = 0.f;
    for (int r = 0; r < rows; ++r) t += part[r * per + threadIdx.x / 4][threadIdx.x % 4];
    o[(size_t)b * H * dh + h * dh + threadIdx.x] = from_f<T>(t * scale);
  }
}

constexpr int kMaxHead = 128;

// Segments of a sequence: enough blocks for the chip, none of less than two chunks.
struct Cut { int segments, per; };
Cut cut_of(int B, int S, int H, int dh, int jobs) {
  const int chunks = (S + kChunk - 1) / kChunk;
  const long blocks = (long)B * H * jobs * (dh > 64 ? 2 : 1);
  long want = blocks > 0 ? (1024 + blocks - 1) / blocks : 1;
  const long most = chunks / 2 > 0 ? chunks / 2 : 1;
  if (want > most) want = most;
  Cut c;
  c.per = chunks > 0 ? (int)((chunks + want - 1) / want) : 1;
  c.segments = chunks > 0 ? (chunks + c.per - 1) / c.per : 1;
  return c;
}

// Launches a kernel for a head size; F is called with (integral DK, DV, bool VEC).
template <typename F>
hipError_t by_head(int dh, bool vec, F&& fn) {
  auto go = [&](auto v) {
    if (dh <= 32) return fn(std::integral_constant<int, 32>(), std::integral_constant<int, 32>(), v);
    if (dh <= 64) return fn(std::integral_constant<int, 64>(), std::integral_constant<int, 64>(), v);
    return fn(std::integral_constant<int, 128>(), std::integral_constant<int, 64>(), v);
  };
  return vec ? go(std::true_type()) : go(std::false_type());
}

template <typename T>
hipError_t walk(const OpCtx& c, const LinearJobs& jobs, int njobs, const LinearShape& sh, bool vec, bool fin) {
  const int cols = sh.dh > 64 ? 2 : 1, units = sh.B * sh.H * sh.segments;
  return by_head(sh.dh, vec, [&](auto dk, auto dv, auto v) {
    constexpr int DK = decltype(dk)::value, DV = decltype(dv)::value;
    constexpr bool VEC = decltype(v)::value;
    constexpr int lds = (int)sizeof(WalkLds<T, DK, DV, sizeof(T) == 2 ? 2 : 1>);
    const int blocks = (units + 7) / 8 * 8 * cols * njobs;
    auto go = [&](auto f) {
      constexpr bool FIN = decltype(f)::value;
      static LdsLimit limit;
      const hipError_t e = limit.raise(reinterpret_cast<const void*>(k_linear_walk<T, DK, DV, VEC, FIN>), lds);
      if (e != hipSuccess) return e;
      k_linear_walk<T, DK, DV, VEC, FIN><<<blocks, 4 * DV, lds, c.stream>>>(jobs, sh, units, cols, njobs);
      return hipGetLastError();
    };
    return fin ? go(std::true_type()) : go(std::false_type());
  });
}
template <typename T>
hipError_t states(const OpCtx& c, const StateJobs& jobs, int njobs, const LinearShape& sh, bool vec) {
  const int cols = sh.dh > 64 ? 2 : 1, units = sh.B * sh.H * sh.segments;
  const hipError_t e = by_head(sh.dh, vec, [&](auto dk, auto dv, auto v) {
    constexpr int DK = decltype(dk)::value, DV = decltype(dv)::value;
    k_linear_states<T, DK, DV, decltype(v)::value><<<(units + 7) / 8 * 8 * cols * njobs, 4 * DV, 0, c.stream>>>(jobs, sh, units, cols, njobs);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  k_linear_scan<<<dim3((sh.dh * sh.dh + 255) / 256, sh.B * sh.H, njobs), 256, 0, c.stream>>>(jobs, sh);
  return hipGetLastError();
}

bool shape_ok(int dt, int B, int S, int H, int dh) {
  return (dt == F32 || dt == BF16) && B >= 0 && S >= 0 && H >= 1 && dh >= 1 && dh <= kMaxHead && (int64_t)B * H <= 65535 &&
         (int64_t)3 * H * dh <= 0x7fffffff && S <= 0x7fffffff - 2 * kChunk;
}
LinearShape shape_of(const Cut& cut, const float* log_decay, const int32_t* lens, int B, int S, int H, int dh) {
  LinearShape sh;
  sh.B = B; sh.S = S; sh.H = H; sh.dh = dh; sh.segments = cut.segments; sh.per = cut.per;
  sh.scale = (float)(1.0 / sqrt((double)dh));
  sh.log_decay = log_decay; sh.lens = lens;
  return sh;
}
// 16-byte accesses: eight elements at a time in every row, on 16-byte boundaries
bool whole_chunks(int dh, std::initializer_list<const void*> bufs) {
  uintptr_t low = 0;
  for (const void* p : bufs) low |= (uintptr_t)p;
  return (low & 15) == 0 && dh % 8 == 0;
}

}  // namespace

size_t linear_attn_scratch(int B, int S, int H, int dh, bool backward) {
  if (!shape_ok(BF16, B, S, H, dh)) return 0;
  const Cut cut = cut_of(B, S, H, dh, backward ? 3 : 1);
  return cut.segments > 1 ? (size_t)B * H * cut.segments * dh * dh * (backward ? 2 : 1) : 0;
}

hipError_t op_linear_attn_fwd(const OpCtx& c, const void* qkv, const float* log_decay, const int32_t* lens, const float* s0, void* o,
                              float* s_out, int B, int S, int H, int dh) {
  ProfScope prof_(c, KC_ATTN_FWD);
  if (!shape_ok(c.dt, B, S, H, dh)) return hipErrorInvalidValue;
  if (B == 0) return hipSuccess;
  if (!log_decay || (S > 0 && (!qkv || !o))) return hipErrorInvalidValue;
  const Cut cut = cut_of(B, S, H, dh, 1);
  if (cut.segments > 1 && (!c.partial || c.partial_elems < linear_attn_scratch(B, S, H, dh, false))) return hipErrorInvalidValue;
  const LinearShape sh = shape_of(cut, log_decay, lens, B, S, H, dh);
  const bool vec = whole_chunks(dh, {qkv, o});
  const size_t e = dtype_size(c.dt), d = (size_t)H * dh;
  const char* p = (const char*)qkv;
  LinearJobs jobs = {};
  LinearJob& j = jobs.j[0];
  j.q = p; j.k = p + d * e; j.v = p + 2 * d * e; j.out = o;
  j.ldq = j.ldk = j.ldv = 3 * d; j.ldo = d;
  j.init = s0; j.fin = s_out; j.in_scale = j.out_scale = 1.f;
  if (cut.segments > 1) {
    StateJobs st = {};
    st.j[0].k = j.k; st.j[0].v = j.v; st.j[0].ldk = st.j[0].ldv = 3 * d; st.j[0].loc = c.partial;
    st.j[0].init = s0; st.j[0].fin = s_out; st.j[0].in_scale = st.j[0].out_scale = 1.f;
    const hipError_t err = c.dt == BF16 ? states<bf16_t>(c, st, 1, sh, vec) : states<float>(c, st, 1, sh, vec);
    if (err != hipSuccess) return err;
    j.before = c.partial; j.fin = nullptr;
  }
  const bool fin = j.fin != nullptr;
  return c.dt == BF16 ? walk<bf16_t>(c, jobs, 1, sh, vec, fin) : walk<float>(c, jobs, 1, sh, vec, fin);
}

hipError_t op_linear_attn_bwd(const OpCtx& c, const void* qkv, const float* log_decay, const int32_t* lens, const float* s0,
                              const void* dout, const float* ds_out, void* dqkv, float* ds0, int B, int S, int H, int dh) {
  ProfScope prof_(c, KC_ATTN_BWD);
  if (!shape_ok(c.dt, B, S, H, dh)) return hipErrorInvalidValue;
  if (B == 0) return hipSuccess;
  if (!log_decay || (S > 0 && (!qkv || !dout || !dqkv))) return hipErrorInvalidValue;
  const Cut cut = cut_of(B, S, H, dh, 3);
  if (cut.segments > 1 && (!c.partial || c.partial_elems < linear_attn_scratch(B, S, H, dh, true))) return hipErrorInvalidValue;
  const LinearShape sh = shape_of(cut, log_decay, lens, B, S, H, dh);
  const bool vec = whole_chunks(dh, {qkv, dout, dqkv});
  const size_t e = dtype_size(c.dt), d = (size_t)H * dh;
  const char *q = (const char*)qkv, *k = q + d * e, *v = k + d * e;
  char* dq = (char*)dqkv;
  const float up = (float)sqrt((double)dh);        // the states of the way back are kept without the factor dh^-1/2
  auto job = [&](const void* jq, int64_t ldq, const void* jk, int64_t ldk, const void* jv, int64_t ldv, void* out, int back) {
    LinearJob j = {};
    j.q = jq; j.ldq = ldq; j.k = jk; j.ldk = ldk; j.v = jv; j.ldv = ldv; j.out = out; j.ldo = 3 * d; j.back = back;
    j.in_scale = back ? up : 1.f; j.out_scale = sh.scale;
    j.init = back ? ds_out : s0;
    return j;
  };
  const int64_t w = 3 * d;
  LinearJobs jobs;
  jobs.j[0] = job(dout, d, v, w, k, w, dq, 0);                      // dQ
  jobs.j[1] = job(k, w, q, w, dout, d, dq + 2 * d * e, 1);          // dV
  jobs.j[2] = job(v, w, dout, d, q, w, dq + d * e, 1);              // dK
  jobs.j[0].turned = jobs.j[2].turned = 1;
  jobs.j[1].fin = ds0;
  if (cut.segments > 1) {
    float* back = c.partial + (size_t)B * H * cut.segments * dh * dh;
    StateJobs st = {};
    st.j[0].k = k; st.j[0].v = v; st.j[0].ldk = st.j[0].ldv = w; st.j[0].loc = c.partial; st.j[0].init = s0; st.j[0].in_scale = 1.f;
    st.j[1].k = q; st.j[1].v = dout; st.j[1].ldk = w; st.j[1].ldv = d; st.j[1].loc = back; st.j[1].init = ds_out; st.j[1].fin = ds0;
    st.j[1].in_scale = up; st.j[1].out_scale = sh.scale; st.j[1].back = 1;
    const hipError_t err = c.dt == BF16 ? states<bf16_t>(c, st, 2, sh, vec) : states<float>(c, st, 2, sh, vec);
    if (err != hipSuccess) return err;
    jobs.j[0].before = c.partial; jobs.j[1].before = jobs.j[2].before = back;
    jobs.j[1].fin = nullptr;
  }
  const bool fin = jobs.j[1].fin != nullptr;
  return c.dt == BF16 ? walk<bf16_t>(c, jobs, 3, sh, vec, fin) : walk<float>(c, jobs, 3, sh, vec, fin);
}

hipError_t op_linear_attn_step(const OpCtx& c, const void* qkv, const float* log_decay, float* state, void* o, int B, int H, int dh) {
  ProfScope prof_(c, KC_ATTN_FWD);
  if ((c.dt != F32 && c.dt != BF16) || B < 0 || H < 1 || dh < 1 || dh > kMaxHead || (int64_t)B * H > 0x7fffffff ||
      (int64_t)3 * H * dh > 0x7fffffff) return hipErrorInvalidValue;
  if (B == 0) return hipSuccess;
  if (!qkv || !log_decay || !state || !o) return hipErrorInvalidValue;
  const float scale = (float)(1.0 / sqrt((double)dh));
  if (c.dt == BF16) k_linear_step<bf16_t><<<B * H, 256, 0, c.stream>>>((const bf16_t*)qkv, log_decay, state, (bf16_t*)o, H, dh, scale);
  else k_linear_step<float><<<B * H, 256, 0, c.stream>>>((const float*)qkv, log_decay, state, (float*)o, H, dh, scale);
  return hipGetLastError();
}

}  // namespace lp
