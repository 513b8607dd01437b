// Linear attention with a decay for each head.  With l = exp(log_decay[h]) and the state S [dh, dh] in fp32,
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = dh^-1/2 q_t S_t   (position t included).
// Chunks of 32 positions: with X the state before a chunk, u = 0 .. 31 the position in it and e = 1,
//   O = dh^-1/2 ( ((Q K^T) . D) V + diag(l^{u + e}) Q X ),  D[u, w] = l^{u - w} for w <= u, otherwise 0,
//   X' = l^c X + sum_u l^{c - u - e} k_u v_u^T              (c: positions of the chunk, 32 but for the last).
// The gradients are the same map of other operands, so that one kernel serves both directions:
//   dQ = map(q <- dO, k <- V, v <- K),
//   dV = map(q <- K, k <- Q, v <- dO) and dK = map(q <- V, k <- dO, v <- Q) with the positions taken from the last to the first
//   and e = 0, where X' = sum l^{distance past the chunk} q dO^T is the gradient of the state.
// A long axis over few heads is cut into segments of whole chunks: k_linear_states leaves what each adds to the state,
// k_linear_scan turns that into the state before each, and the blocks of k_linear_walk go over their segments side by side.
//
// Products run on the matrix cores, 32 x 32 tiles.  A wave keeps 32 columns of the state, all rows of them, in fp32 accumulators, and
// the waves of a head share the chunk's q, k and v through LDS.  The accumulators' layout is that of an operand whose reduction
// index is the row, so that the state and the scores K Q^T go from one product to the next without leaving the registers (but for fp32 heads of
// 65 to 96, where the compiler puts 48 to 164 bytes a lane into scratch memory, and bf16 heads of 97 to 128 with a final state, 32).
// Heads of up to 64: two waves for every 32 columns, one with the state, which multiplies it with the chunk's queries and then
// adds the chunk to it, and one with the chunk's own scores and their product with the values, which adds both parts of the output.
// Wider heads, whose state fills the registers anyway: one wave does both.
// Whatever has more bits than the compute dtype (scores times decay, values times decay, the state as an operand) is
// split into three bf16 parts, which hold all its 24 bits: the parts' products are exact and summed in fp32.
#include "common.h"
#include "gemm_common.h"

namespace lp {

namespace {

constexpr int kChunk = 32;
template <typename T> constexpr int kParts = sizeof(T) == 2 ? 3 : 1;       // operands that hold an fp32 value
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
// Operand whose reduction index is the column of an LDS tile: eight of sixteen columns, at 4 hf + {0..3} and 8 + 4 hf + {0..3}, the order
// of an accumulator's values; p points at the row's column 4 hf.
template <typename T>
__device__ __forceinline__ typename Frag<T>::V frag_row(const T* p) {
  typedef __attribute__((ext_vector_type(4))) T T4;
  const T4 a = *reinterpret_cast<const T4*>(p), b = *reinterpret_cast<const T4*>(p + 8);
  typename Frag<T>::V r;
#pragma unroll
  for (int e = 0; e < 4; ++e) { r[e] = a[e]; r[4 + e] = b[e]; }
  return r;
}
// Operand whose reduction index is the row of an LDS tile: lane (n, hf) gets column c0 + n of rows r0 + 4 hf + {0..3} and
// r0 + 8 + 4 hf + {0..3}; bf16 by the transposing read (its 16-lane groups: lane 4 r + c
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
// fp32 values as NP operands whose sum they are (three: all 24 bits); one where the compute dtype is fp32.  Each part is the upper half of what the
// parts before it leave, so that a pair takes one byte permutation a part (8 x 1024 positions, 12 heads of 64, forward and backward: 97 us with parts
// rounded by conversions, 91 so; with two parts, which leave 2^-17 of every such value, 81).
template <int NP>
__device__ __forceinline__ void split(const f32x8& v, bf16x8 (&f)[NP]) {
  typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
  u32x4 w[NP];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a = v[2 * e], b = v[2 * e + 1];
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      const unsigned ia = __builtin_bit_cast(unsigned, a), ib = __builtin_bit_cast(unsigned, b);
      w[s][e] = __builtin_amdgcn_perm(ib, ia, 0x07060302u);
      a -= __builtin_bit_cast(float, ia & 0xffff0000u);
      b -= __builtin_bit_cast(float, ib & 0xffff0000u);
    }
  }
#pragma unroll
  for (int s = 0; s < NP; ++s) f[s] = __builtin_bit_cast(bf16x8, w[s]);
}
__device__ __forceinline__ void split(const f32x8& v, f32x8 (&f)[1]) { f[0] = v; }
template <typename V, int NP>
__device__ __forceinline__ f32x16 mma_parts(const V (&a)[NP], const V& b, f32x16 c) {      // smallest first
#pragma unroll
  for (int s = NP - 1; s >= 0; --s) c = mma(a[s], b, c);
  return c;
}
template <typename V, int NP>
__device__ __forceinline__ f32x16 mma_parts(const V& a, const V (&b)[NP], f32x16 c) {
#pragma unroll
  for (int s = NP - 1; s >= 0; --s) c = mma(a, b[s], c);
  return c;
}
template <int NP>
__device__ __forceinline__ void split_half(const f32x16& v, int kk, bf16x8 (&f)[NP]) {     // values 8 kk .. of an accumulator
  f32x8 t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = v[8 * kk + e];
  split(t, f);
}
__device__ __forceinline__ void split_half(const f32x16& v, int kk, f32x8 (&f)[1]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[0][e] = v[8 * kk + e];
}
__device__ __forceinline__ void zero(f32x16& a) {
#pragma unroll
  for (int i = 0; i < 16; ++i) a[i] = 0.f;
}
// l^n, n >= 0; l^0 is 1 also for a decay to nothing (log_decay = -inf, which comes in as a large finite number)
__device__ __forceinline__ float power(float g2, int n) { return __builtin_amdgcn_exp2f(g2 * (float)n); }
// l^n for a chain of products, one after another: rounded to 24 bits it would be off by the same share every time (4096 chunks of decays of
// 1 - 2^-17: 1e-4 of the state), so that what rounding leaves out goes into the next factor, and the product of all is off by one unit.
struct Chain {
  float by, rest, off;
  __device__ __forceinline__ Chain(float g2, int n) {
    const float x = g2 * (float)n;
    by = __builtin_amdgcn_exp2f(x);
    rest = by < 0.5f ? 0.f : expm1f(x * 0.69314718056f) - (by - 1.f);      // lower ones leave nothing after some steps
    off = 0.f;
  }
  __device__ __forceinline__ float next() {
    const float t = off + rest, f = by + t;
    off = t - (f - by);
    return f;
  }
};
__device__ __forceinline__ float decay_of(const float* log_decay, int h) {
  const float g = log_decay[h];
  return (g < -1e4f ? -1e4f : g) * kLog2e;
}

// [R rows][W columns] of a matrix on the way into LDS, in registers while the chunk before it is computed, by a block of NT
// threads.  Rows past the sequence repeat its last one (they meet scores that are left out, weights of 0 and
// outputs that are not stored) and columns past `cols` are zeros.  VEC: rows are whole 16-byte loads on 16-byte boundaries.
template <typename T, int W, int R, int NT, bool VEC>
struct TileRegs {
  static constexpr int E = 16 / (int)sizeof(T), CPR = W / E, N = R * CPR / NT;
  static_assert(R * CPR % NT == 0, "whole loads");
  typedef __attribute__((ext_vector_type(E))) T V;
  V v[N];
  unsigned off[N];             // bytes behind the chunk's lowest row
  // rows of a chunk with `count` positions; back: position 0 is the highest row
  __device__ __forceinline__ void rows(int ld, bool back, int count, int cols) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = threadIdx.x + NT * i, r = x / CPR, c = x % CPR * E;
      const int rr = r < count ? r : count - 1, m = back ? count - 1 - rr : rr;
      off[i] = (__umul24(m, ld) + (c < cols ? c : 0)) * (unsigned)sizeof(T);
    }
  }
  __device__ __forceinline__ void load(const T* low, int cols) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const char* p = reinterpret_cast<const char*>(low) + off[i];
      if (VEC) {
        v[i] = *reinterpret_cast<const V*>(p);
      } else {
        const int c = (threadIdx.x + NT * i) % CPR * E;
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = reinterpret_cast<const T*>(p)[c + e < cols ? e : 0];
      }
    }
  }
  template <int LD>
  __device__ __forceinline__ void store(T (*s)[LD], int cols) {
    if (cols < W) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = (threadIdx.x + NT * i) % CPR * E + e < cols ? v[i][e] : (T)0.f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = threadIdx.x + NT * i;
      *reinterpret_cast<V*>(&s[x / CPR][x % CPR * E]) = v[i];
    }
  }
  // whether one is an infinity or a NaN
  __device__ __forceinline__ bool non_finite() const {
    typedef __attribute__((ext_vector_type(4))) unsigned U;
    // without its sign and one exponent step up, such a number (and no other) has the sign's bit set
    constexpr unsigned size = sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu, step = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
    unsigned bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const U w = (__builtin_bit_cast(U, v[i]) & size) + step;
      bad |= w[0] | w[1] | w[2] | w[3];
    }
    return (bad & ~size) != 0;
  }
};

// One application of the map to all heads: matrices at head 0, row strides, and the states.
struct LinearJob {
  const void *q, *k, *v;
  void* out;
  int ldq, ldk, ldv, ldo;          // elements
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

// What a block works on: its job, sequence, head and stretch of positions.
struct Place {
  int job, seg, bh, h, len, first, last, stop;
  size_t row0;                 // the sequence's first row
  float g2;
};
// Blocks go to the eight dies by turns of their number, x first: the jobs (y) of one segment, which share its rows, run on one die.
__device__ __forceinline__ bool place(const LinearShape& sh, int units, Place& p) {
  const unsigned unit = blockIdx.z * 8 + blockIdx.x;
  p.job = blockIdx.y;
  if (unit >= (unsigned)units) return false;
  const unsigned bh = sh.segments > 1 ? unit / (unsigned)sh.segments : unit, b = bh / (unsigned)sh.H;
  p.bh = bh;
  p.seg = unit - bh * sh.segments;
  p.h = bh - b * sh.H;
  p.len = sh.length(b);
  p.first = p.seg * sh.per * kChunk;
  p.last = p.first + sh.per * kChunk < sh.S ? p.first + sh.per * kChunk : sh.S;       // padding included
  p.stop = p.last < p.len ? p.last : p.len;
  p.row0 = (size_t)b * sh.S;
  p.g2 = decay_of(sh.log_decay, p.h);
  return true;
}
template <typename T>
__device__ __forceinline__ const T* column(const void* m, size_t row, int ld, int h, int dh) {
  return (const T*)m + (row * ld + (size_t)h * dh);
}
// Lowest row of the chunk of `count` positions from u0 on.
template <typename T>
__device__ __forceinline__ const T* lowest(const T* p, int ld, bool back, int u0, int count) {
  return p + (ptrdiff_t)(back ? -(u0 + count - 1) : u0) * ld;
}
__device__ __forceinline__ int acc_row(int v, int hf) { return 8 * (v / 4) + 4 * hf + v % 4; }      // of an accumulator's value

// state += sum over the chunk's positions of k (weight v)^T: all rows, columns 32 col ..
template <typename T, int DK, int LD>
__device__ __forceinline__ void add_outer(f32x16 (&state)[DK / 32], const T (*ks)[LD], const T (*vs)[LD], const float* weight, int col, int lane) {
  const int hf = lane >> 5;
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    const typename Frag<T>::V v = frag_col<LD>(vs, 16 * kk, 32 * col, lane);
    f32x8 w;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(weight + 16 * kk + 8 * x + 4 * hf);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * x + e] = (float)v[4 * x + e] * t[e];
    }
    typename Frag<T>::V f[kParts<T>];
    split(w, f);
#pragma unroll
    for (int i = 0; i < DK / 32; ++i) state[i] = mma_parts(frag_col<LD>(ks, 16 * kk, 32 * i, lane), f, state[i]);
  }
}
template <int ND>
__device__ __forceinline__ void scale(f32x16 (&state)[ND], float by) {
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) state[i][v] *= by;
}

// Between the rows of a tile: 16 bytes spread what a wave reads of 32 neighbouring rows or of 4 rows, 64 bytes each, over the banks,
// but for 128 bf16, which are the banks' period (1024 heads of 1024 positions, forward and backward: 358 + 1017 us with 16 bytes in the walk, 357 + 1009 with
// 80; the states kernel, whose blocks hold twice the rows, loses by them: 32 heads of 2048 positions 56.5 + 104 with 16, 59 + 107 with 80).
template <typename T> constexpr int kPad = 16 / (int)sizeof(T);
template <typename T, int DK> constexpr int kWalkPad = sizeof(T) == 2 && DK == 128 ? 40 : kPad<T>;
template <typename T, int DK>
struct Tile { __attribute__((aligned(16))) T q[kChunk][DK + kWalkPad<T, DK>], k[kChunk][DK + kWalkPad<T, DK>], v[kChunk][DK + kWalkPad<T, DK>]; };
template <typename T, int DK>
struct WalkLds {
  Tile<T, DK> t[2];
  __attribute__((aligned(16))) float weight[2][kChunk];             // of whole chunks, and of the last
  int bad[2];
  f32x4 earlier[2][DK <= 64 ? DK / 32 : 1][4][64];                  // two roles, by turns: as the accumulators hold it (one role: not used)
};

// Waves for 32 columns: two of up to 64 wide heads (96 heads of 64, 1024 positions, forward: 32 us; with one, which does not fit the registers of three waves a
// SIMD, 48), one of wider ones, forward and backward, us, one and two: bf16, 128 wide, 1024 heads of 1024 positions 357 + 1009 and 369 + 1060, 32 heads of 2048
// 56.5 + 104 and 59.5 + 111, but 64 heads 81 + 193 and 86 + 146; fp32, which two would suit, 40 heads of 2048 136 + 356 and 124 + 322.
template <int DK> constexpr int kRoles = DK <= 64 ? 2 : 1;
template <typename T, int DK> constexpr int kWavesPerSimd = DK <= 64 ? 3 : sizeof(T) * DK == 512 ? 1 : 2;

// A block: one segment of one head.  bf16, a walk alone: 16 heads of 64, 16384 positions, cut, 35 us (134 MB of tensors, 3.8 TB/s); 96 heads of 1024
// positions 17 us cut (3 TB/s), its three backward jobs uncut 61 to 66 (88 MB).  Where the card is full, memory bounds it (512 heads of
// 1024 positions: forward 63 us, 4.3 TB/s); where it is not, the wave with the state, for which a chunk takes about 3500 clocks, one step waiting for
// the other: LDS, splitting the state, products, LDS.  Two such waves with half of the rows each gained a sixth of that and lost more to the wider
// blocks (with two bf16 parts a value instead of three, 16 heads of 16384: 52 + 98 us became 57 + 106).
template <typename T, int DK, bool VEC, bool FIN>
__global__ void __launch_bounds__(2 * kRoles<DK> * DK, (kWavesPerSimd<T, DK>)) k_linear_walk(LinearJobs jobs, LinearShape sh, int units) {
  constexpr int ROLES = kRoles<DK>, NT = 2 * ROLES * DK, NP = kParts<T>, ND = DK / 32;
  constexpr int LD = DK + kWalkPad<T, DK>;
  typedef typename Frag<T>::V FV;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  WalkLds<T, DK>& sm = *reinterpret_cast<WalkLds<T, DK>*>(smem);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hf = lane >> 5;
  const int col = wave < ND ? wave : wave - ND;
  Place at;
  if (!place(sh, units, at)) return;
  const LinearJob job = jobs.j[at.job];
  const int dh = sh.dh, e0 = job.back ? 0 : 1, first = at.first, stop = at.stop;
  const bool back = job.back != 0, full = dh == DK;
  // position u of the walk is row `row + u * dir`
  const int dir = back ? -1 : 1;
  const size_t row = at.row0 + (back && at.len > 0 ? at.len - 1 : 0);
  const int head = kChunk < stop - first ? kChunk : stop - first;                // positions of the first chunk
  const T* qp = lowest(column<T>(job.q, row, job.ldq, at.h, dh), job.ldq, back, first, head);
  const T* kp = lowest(column<T>(job.k, row, job.ldk, at.h, dh), job.ldk, back, first, head);
  const T* vp = lowest(column<T>(job.v, row, job.ldv, at.h, dh), job.ldv, back, first, head);

  TileRegs<T, DK, kChunk, NT, VEC> qr, kr, vr;
  int left = stop - first;                                   // positions not yet asked for
  auto rows = [&](int count) {
    qr.rows(job.ldq, back, count, dh);
    kr.rows(job.ldk, back, count, dh);
    vr.rows(job.ldv, back, count, dh);
  };
  auto fetch = [&]() {
    const int count = left < kChunk ? left : kChunk;
    if (count < kChunk) rows(count);
    qr.load(qp, dh);
    kr.load(kp, dh);
    vr.load(vp, dh);
    left -= count;
    const int by = back ? -(left < kChunk ? left : kChunk) : kChunk;             // to the lowest row of the next chunk
    qp += (ptrdiff_t)by * job.ldq;
    kp += (ptrdiff_t)by * job.ldk;
    vp += (ptrdiff_t)by * job.ldv;
  };
  auto leave = [&](int slot, int u0) {
    qr.store(sm.t[slot].q, dh);
    kr.store(sm.t[slot].k, dh);
    if (vr.non_finite()) sm.bad[slot] = u0;
    vr.store(sm.t[slot].v, dh);
    if (left > 0) fetch();
  };
  if (first < stop) {
    rows(head);
    fetch();
  }
  // rows of the padding are zeros, whatever stands there in the inputs
  {
    T* pad = const_cast<T*>(column<T>(job.out, at.row0, job.ldo, at.h, dh));
    const int from = first > at.len ? first : at.len;
    for (int64_t x = threadIdx.x; x < (int64_t)(at.last - from) * DK; x += NT)
      if ((int)(x % DK) < dh) pad[(size_t)(from + x / DK) * job.ldo + x % DK] = (T)0.f;
  }
  const int rest = (stop - first) % kChunk;
  if (threadIdx.x < kChunk) {
    const int u = threadIdx.x;
    sm.weight[0][u] = power(at.g2, kChunk - u - e0);
    sm.weight[1][u] = u < rest ? power(at.g2, rest - u - e0) : 0.f;
  }
  if (threadIdx.x < 2) sm.bad[threadIdx.x] = -1;

  // The parts of the work on a chunk.
  f32x16 state[ND];
  const int scol = 32 * col + n;
  auto pull = [&]() {                                        // the wave's columns of the state before the segment
    const bool whole = job.before != nullptr;
    const float* x0 = whole ? job.before + ((size_t)at.bh * sh.segments + at.seg) * dh * dh : job.init ? job.init + (size_t)at.bh * dh * dh : nullptr;
#pragma unroll
    for (int i = 0; i < ND; ++i) zero(state[i]);
    if (!x0) return;
    if (full) {
      const float* x = job.turned ? x0 + scol * DK + 4 * hf : x0 + scol + 4 * hf * DK;
      if (job.turned) {
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) state[i][v] = x[32 * i + acc_row(v, 0)];
      } else {
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) state[i][v] = x[(32 * i + acc_row(v, 0)) * DK];
      }
    } else {
      const int cc = scol < dh ? scol : dh - 1, by_row = job.turned ? 1 : dh, by_col = job.turned ? dh : 1;
      const float* x = x0 + cc * by_col;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 32 * i + acc_row(v, hf);
          state[i][v] = x[(r < dh ? r : dh - 1) * by_row];
        }
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) state[i][v] = 32 * i + acc_row(v, hf) < dh && scol < dh ? state[i][v] : 0.f;
    }
    if (!whole && job.in_scale != 1.f) scale(state, job.in_scale);
  };
  auto earlier = [&](const Tile<T, DK>& t) {                 // what the chunks before give, without its decay
    f32x16 o = (f32x16)0.f;
#pragma unroll
    for (int kk = 0; kk < 2 * ND; ++kk) {
      FV f[NP];
      split_half(state[kk / 2], kk % 2, f);
      o = mma_parts(f, frag_row<T>(&t.q[n][16 * kk + 4 * hf]), o);
    }
    return o;
  };
  auto own = [&](const Tile<T, DK>& t, f32x16 o, const float (&near)[16], bool slow, int c) {      // what the chunk itself adds
    if (!slow) {
      // the scores above the diagonal are left out by choice and not by a product with 0, so that an infinity or a NaN in a later
      // key reaches nobody
      f32x16 p = (f32x16)0.f;
#pragma unroll
      for (int kk = 0; kk < 2 * ND; ++kk) p = mma(frag_row<T>(&t.k[n][16 * kk + 4 * hf]), frag_row<T>(&t.q[n][16 * kk + 4 * hf]), p);
#pragma unroll
      for (int v = 0; v < 16; ++v) p[v] = acc_row(v, hf) <= n ? p[v] * near[v] : 0.f;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        FV f[NP];
        split_half(p, kk, f);
        o = mma_parts(frag_col<LD>(t.v, 16 * kk, 32 * col, lane), f, o);
      }
    } else {
      // A chunk with an infinity or a NaN among its values: row by row, the later ones left out (0 times infinity is not 0).
#pragma unroll 1
      for (int r = 0; r < c; ++r) {
        float s = 0.f;
#pragma unroll
        for (int kk = 0; kk < 2 * ND; ++kk) {
          const FV k = frag_row<T>(&t.k[r][16 * kk + 4 * hf]), q = frag_row<T>(&t.q[n][16 * kk + 4 * hf]);
#pragma unroll
          for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)q[e], (float)k[e], s);
        }
        s += __shfl_xor(s, 32, 64);
        if (r > n) continue;
        s *= power(at.g2, n - r) * sh.scale;
#pragma unroll
        for (int v = 0; v < 16; ++v) o[v] = __builtin_fmaf(s, (float)t.v[r][32 * col + acc_row(v, hf)], o[v]);
      }
    }
    return o;
  };
  auto decays = [&](float (&near)[16]) {                     // between a query and the keys, dh^-1/2
#pragma unroll
    for (int v = 0; v < 16; ++v) near[v] = acc_row(v, hf) <= n ? power(at.g2, n - acc_row(v, hf)) * sh.scale : 0.f;
  };
  T* to = const_cast<T*>(column<T>(job.out, row, job.ldo, at.h, dh)) + ((ptrdiff_t)(first + n) * dir * job.ldo + 32 * col);
  auto put = [&](const f32x16& o, int c) {
    if (n < c) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        typedef __attribute__((ext_vector_type(4))) T T4;
        const int x = 8 * g + 4 * hf;
        T4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (T)o[4 * g + j];
        if (VEC) {
          if (full || 32 * col + x < dh) *reinterpret_cast<T4*>(to + x) = w;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (32 * col + x + j < dh) to[x + j] = w[j];
        }
      }
    }
    to += (ptrdiff_t)kChunk * dir * job.ldo;
  };
  const float carry = power(at.g2, n + e0) * sh.scale;
  Chain whole(at.g2, kChunk);
  auto add = [&](const Tile<T, DK>& t, int c) {              // the chunk to the state
    scale(state, c == kChunk ? whole.next() : power(at.g2, c));
    add_outer<T, DK, LD>(state, t.k, t.v, sm.weight[c < kChunk], col, lane);
  };
  auto finish = [&]() {
    if (!FIN || !job.fin) return;
    float* out = job.fin + (size_t)at.bh * dh * dh;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = 32 * i + acc_row(v, hf);
        if (full || (r < dh && scol < dh)) out[r * dh + scol] = state[i][v] * job.out_scale;
      }
  };

  // All waves go through the same chunks, a barrier each: behind it the chunk's tile is there and, two roles, what the chunks before
  // the last one give to that one, whose output then goes out.  The other tile is written behind the barrier, when nobody reads it any more.
  if constexpr (ROLES == 1) {
    pull();
    float near[16];
    decays(near);
    __syncthreads();
    if (first < stop) leave(0, first);
    for (int u0 = first, slot = 0; u0 < stop; u0 += kChunk, slot ^= 1) {
      const int c = stop - u0 < kChunk ? stop - u0 : kChunk;
      __syncthreads();
      const Tile<T, DK>& t = sm.t[slot];
      put(own(t, earlier(t) * carry, near, sm.bad[slot] == u0, c), c);
      if (FIN || u0 + kChunk < stop) add(t, c);
      if (u0 + kChunk < stop) leave(slot ^ 1, u0 + kChunk);
    }
    finish();
  } else if (wave < ND) {
    pull();
    __syncthreads();
    if (first < stop) leave(0, first);
    for (int u0 = first, slot = 0; u0 < stop; u0 += kChunk, slot ^= 1) {
      const int c = stop - u0 < kChunk ? stop - u0 : kChunk;
      __syncthreads();
      const f32x16 o = earlier(sm.t[slot]);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = o[4 * g + j];
        sm.earlier[slot][col][g][lane] = w;
      }
      if (FIN || u0 + kChunk < stop) add(sm.t[slot], c);
      if (u0 + kChunk < stop) leave(slot ^ 1, u0 + kChunk);
    }
    __syncthreads();
    finish();
  } else {
    float near[16];
    decays(near);
    f32x16 o;                                                // of the last chunk, what it adds itself
    auto last = [&](int slot, int c) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 w = sm.earlier[slot][col][g][lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[4 * g + j] += w[j] * carry;
      }
      put(o, c);
    };
    __syncthreads();
    if (first < stop) leave(0, first);
    for (int u0 = first, slot = 0; u0 < stop; u0 += kChunk, slot ^= 1) {
      const int c = stop - u0 < kChunk ? stop - u0 : kChunk;
      __syncthreads();
      if (u0 > first) last(slot ^ 1, kChunk);
      o = own(sm.t[slot], (f32x16)0.f, near, sm.bad[slot] == u0, c);
      if (u0 + kChunk < stop) leave(slot ^ 1, u0 + kChunk);
    }
    __syncthreads();
    if (first < stop) last((stop - first - 1) / kChunk & 1, (stop - first - 1) % kChunk + 1);
  }
}

// What a segment adds to the state: loc [B H, segments, dh, dh] for each job.  The last segment is needed only for the state that goes
// out.
struct StateJob {
  const void *k, *v;
  int ldk, ldv;
  float* loc;
  const float* init;
  float* fin;
  float in_scale, out_scale;
  int back;
};
struct StateJobs { StateJob j[2]; };

// Two waves for every 32 columns, which take a half of every 64 positions each; their sums are added at the end.  16 heads of 64, 16384
// positions, bf16: 22 us for the 67 MB of k and v, 3 TB/s.
template <typename T, int DK, bool VEC>
__global__ void __launch_bounds__(4 * DK) k_linear_states(StateJobs jobs, LinearShape sh, int units) {
  constexpr int ND = DK / 32, LD = DK + kPad<T>, R = 2 * kChunk;
  struct Lds { __attribute__((aligned(16))) T k[2][R][LD], v[2][R][LD]; __attribute__((aligned(16))) float weight[2][R]; };
  extern __shared__ __attribute__((aligned(16))) char smem[];
  Lds& sm = *reinterpret_cast<Lds*>(smem);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hf = lane >> 5;
  const int half = wave / ND, col = wave % ND;
  Place at;
  if (!place(sh, units, at)) return;
  const StateJob job = jobs.j[at.job];
  if (at.seg == sh.segments - 1 && !job.fin) return;
  const int dh = sh.dh, e0 = job.back ? 0 : 1, first = at.first, stop = at.stop;
  const bool back = job.back != 0, full = dh == DK;
  const size_t row = at.row0 + (back && at.len > 0 ? at.len - 1 : 0);
  const int head = R < stop - first ? R : stop - first;
  const T* kp = lowest(column<T>(job.k, row, job.ldk, at.h, dh), job.ldk, back, first, head);
  const T* vp = lowest(column<T>(job.v, row, job.ldv, at.h, dh), job.ldv, back, first, head);
  f32x16 state[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) zero(state[i]);
  TileRegs<T, DK, R, 4 * DK, VEC> kr, vr;
  int left = stop - first;
  auto fetch = [&]() {
    const int count = left < R ? left : R;
    if (count < R) {
      kr.rows(job.ldk, back, count, dh);
      vr.rows(job.ldv, back, count, dh);
    }
    kr.load(kp, dh);
    vr.load(vp, dh);
    left -= count;
    const int by = back ? -(left < R ? left : R) : R;
    kp += (ptrdiff_t)by * job.ldk;
    vp += (ptrdiff_t)by * job.ldv;
  };
  if (first < stop) {
    kr.rows(job.ldk, back, head, dh);
    vr.rows(job.ldv, back, head, dh);
    fetch();
  }
  const int rest = (stop - first) % R;
  if (threadIdx.x < R) {
    const int u = threadIdx.x;
    sm.weight[0][u] = power(at.g2, R - u - e0);
    sm.weight[1][u] = u < rest ? power(at.g2, rest - u - e0) : 0.f;
  }
  Chain whole(at.g2, R);
  for (int u0 = first, slot = 0; u0 < stop; u0 += R, slot ^= 1) {
    const int c = stop - u0 < R ? stop - u0 : R;
    kr.store(sm.k[slot], dh);                                // read by nobody since the last barrier
    vr.store(sm.v[slot], dh);
    if (left > 0) fetch();
    __syncthreads();
    scale(state, c == R ? whole.next() : power(at.g2, c));
    add_outer<T, DK, LD>(state, sm.k[slot] + kChunk * half, sm.v[slot] + kChunk * half, sm.weight[c < R] + kChunk * half, col, lane);
  }
  // the second halves' sums go through the tiles' memory
  float* part = reinterpret_cast<float*>(smem) + col * (ND * 16 * 64);
  __syncthreads();
  if (half == 1) {
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) part[(i * 16 + v) * 64 + lane] = state[i][v];
  }
  __syncthreads();
  if (half == 1) return;
  float* out = job.loc + ((size_t)at.bh * sh.segments + at.seg) * dh * dh;
  const int scol = 32 * col + n;
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int r = 32 * i + acc_row(v, hf);
      if (full || (r < dh && scol < dh)) out[r * dh + scol] = state[i][v] + part[(i * 16 + v) * 64 + lane];
    }
}
template <typename T, int DK>
constexpr int state_lds() {
  const int tiles = 2 * 2 * 2 * kChunk * (DK + kPad<T>) * (int)sizeof(T) + 2 * 2 * kChunk * 4, sums = DK / 32 * (DK / 32) * 16 * 64 * 4;
  return tiles > sums ? tiles : sums;
}

// In place: what a segment adds becomes the state before it.  A thread takes V neighbouring elements of the state:
// a chain of one multiplication and addition a segment, so that the loads in flight bound it (47 segments of 16 heads of 64: 9.1 us, 25 MB).
template <int V>
__global__ void __launch_bounds__(256) k_linear_scan(StateJobs jobs, LinearShape sh) {
  typedef __attribute__((ext_vector_type(V))) float FV;
  const StateJob job = jobs.j[blockIdx.z];
  const int bh = blockIdx.y, x = (blockIdx.x * 256 + threadIdx.x) * V, dd = sh.dh * sh.dh;
  if (x >= dd) return;
  float* p = job.loc + (size_t)bh * sh.segments * dd + x;
  const int last = job.fin ? sh.segments : sh.segments - 1;    // segments whose addition is there
  constexpr int U = 8;                                         // loads in flight
  FV add[U], s = (FV)0.f;
  auto fetch = [&](int g) {
#pragma unroll
    for (int i = 0; i < U; ++i) add[i] = g + i < last ? *reinterpret_cast<const FV*>(p + (size_t)(g + i) * dd) : (FV)0.f;
  };
  fetch(0);
  if (job.init) s = *reinterpret_cast<const FV*>(job.init + (size_t)bh * dd + x) * job.in_scale;
  const float g2 = decay_of(sh.log_decay, bh % sh.H);
  const int len = sh.length(bh / sh.H), span = sh.per * kChunk;
  Chain whole(g2, span);
  for (int g = 0; g < sh.segments; g += U) {
    FV now[U];
#pragma unroll
    for (int i = 0; i < U; ++i) now[i] = add[i];
    if (g + U < sh.segments) fetch(g + U);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (g + i >= sh.segments) break;
      *reinterpret_cast<FV*>(p + (size_t)(g + i) * dd) = s;
      const int left = len - (g + i) * span, c = left < 0 ? 0 : left < span ? left : span;
      s = (c == span ? whole.next() : power(g2, c)) * s + now[i];
    }
  }
  if (job.fin) *reinterpret_cast<FV*>(job.fin + (size_t)bh * dd + x) = s * job.out_scale;
}

// One position, a block for each head: the state is read, decayed, added to and written back in one pass, four neighbouring elements a thread and
// four rows of them in flight.  Bound by the state's bytes (192 sequences of 16 heads of 64, bf16: 16.8 us for 101 MB, of which the last-level cache holds a part:
// 6 TB/s), with few heads by the launch (12 heads: 3.7 us).
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
  // x l, near 1 as x + x (l - 1): l rounded itself would be off by the same share token after token
  const float g2 = decay_of(log_decay, h);
  const bool near = g2 > -1.f;
  const float by = near ? expm1f(g2 * 0.69314718056f) : power(g2, 1);
  auto next = [&](float x, float kv) { return __builtin_fmaf(x, by, near ? kv + x : kv); };
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
            for (int e = 0; e < 4; ++e) { x[i][e] = next(x[i][e], kr * v[c + e]); acc[e] += qr * x[i][e]; }
            *reinterpret_cast<f32x4*>(s + (size_t)rr * dh + c) = x[i];
          }
        }
      }
    } else {
      for (int r = r0; r < dh; r += rows)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < dh) {
            const float x = next(s[(size_t)r * dh + c + e], k[r] * v[c + e]);
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

// Segments of a sequence: as many as make three blocks a compute unit up to 64 wide, two of wider heads, one in fp32 beyond 96 (there two where one would be less
// than three segments), but none of less than four chunks, and no cut into two, which costs two more launches and a second pass over k and v.  Three, two and one
// are what runs at once in bf16 beyond 32 and in fp32 beyond 96; up to 32 wide LDS holds six blocks in bf16 and four in fp32, in fp32 33 to 64 wide two and
// 65 to 96 wide one.  Whole calls, forward and backward, us:
//   blocks of 64 wide heads, 384 / 768 / 1024     bf16  16 heads, 16384 positions  67 + 147, 60 + 116, 65 + 129;  96 heads, 1024 positions  32 + 56, 32 + 56, 32 + 58
//                                                 fp32  32 heads, 2048 positions  49 + 95, 41 + 82, 41 + 97
//   of 32 wide heads, 384 / 768 / 1024            bf16  32 heads, 2048 positions  20 + 33, 19 + 24, 19 + 26;  16 heads, 16384 positions  44 + 98, 41 + 59, 32 + 72
//                                                 fp32  31 + 59, 25 + 39, 25 + 39;  83 + 204, 57 + 119, 52 + 100
//   of 128 wide heads, 256 / 512 / 768            bf16  32 heads, 2048 positions  53 + 190, 56 + 104, 58 + 102;  128 heads  206 + 291, 137 + 291, 161 + 292
//                                                 fp32  40 heads  134 + 507, 153 + 355, 168 + 351;  80 heads  251 + 518, 267 + 518, 296 + 663
//   of 96 wide heads, 256 / 512 / 768             40 heads, 2048 positions  bf16  54 + 173, 49 + 87, 55 + 99;  fp32  136 + 571, 149 + 361, 154 + 351
//   of four chunks at least, or two: 32 heads of 64 in fp32, 2048 positions, forward 42 and 55; or six: 35 heads in fp32, 511 positions, which are
//   then not cut, 25 and 42
//   uncut, or in two: 8 heads of 64, 300 positions 16 + 16, 19.5 + 20; 96 heads of 64, 1024 positions, backward 56.6, 57.2; 64 heads of 128, 2048 positions,
//   backward 193, 177; 80 of them in fp32 517, 693
struct Cut { int segments, per; };
Cut cut_of(int dt, int B, int S, int H, int dh, int jobs) {
  const int chunks = (S + kChunk - 1) / kChunk, alone = dt == F32 && dh > 96;
  const long blocks = B > 0 ? (long)B * H * jobs : 1, once = 256 * (dh <= 64 ? 3 : alone ? 1 : 2);
  long want = once / blocks;
  if (alone && want < 3) want = 2 * once / blocks;
  const long most = chunks / 4;
  if (want > most) want = most;
  if (want < 3) want = 1;
  Cut c;
  c.per = chunks > 0 ? (int)((chunks + want - 1) / want) : 1;
  c.segments = chunks > 0 ? (chunks + c.per - 1) / c.per : 1;
  return c;
}

size_t cut_elems(const Cut& c, int B, int H, int dh, bool backward) {
  return c.segments > 1 ? (size_t)B * H * c.segments * dh * dh * (backward ? 2 : 1) : 0;
}

// Calls fn(integral DK, bool VEC) for a head size.
template <typename F>
hipError_t by_head(int dh, bool vec, F&& fn) {
  auto go = [&](auto v) {
    if (dh <= 32) return fn(std::integral_constant<int, 32>(), v);
    if (dh <= 64) return fn(std::integral_constant<int, 64>(), v);
    if (dh <= 96) return fn(std::integral_constant<int, 96>(), v);
    return fn(std::integral_constant<int, 128>(), v);
  };
  return vec ? go(std::true_type()) : go(std::false_type());
}

template <typename T>
hipError_t walk(const OpCtx& c, const LinearJobs& jobs, int njobs, const LinearShape& sh, bool vec, bool fin) {
  const int units = sh.B * sh.H * sh.segments;
  const dim3 blocks(8, njobs, (units + 7) / 8);
  return by_head(sh.dh, vec, [&](auto dk, auto v) {
    constexpr int DK = decltype(dk)::value, lds = (int)sizeof(WalkLds<T, DK>), threads = 2 * kRoles<DK> * DK;
    constexpr bool VEC = decltype(v)::value;
    auto go = [&](auto f) {
      constexpr bool FIN = decltype(f)::value;
      static LdsLimit limit;
      const hipError_t e = limit.raise(reinterpret_cast<const void*>(k_linear_walk<T, DK, VEC, FIN>), lds);
      if (e != hipSuccess) return e;
      k_linear_walk<T, DK, VEC, FIN><<<blocks, threads, lds, c.stream>>>(jobs, sh, units);
      return hipGetLastError();
    };
    return fin ? go(std::true_type()) : go(std::false_type());
  });
}
template <typename T>
hipError_t states(const OpCtx& c, const StateJobs& jobs, int njobs, const LinearShape& sh, bool vec) {
  const int units = sh.B * sh.H * sh.segments;
  const dim3 blocks(8, njobs, (units + 7) / 8);
  const hipError_t e = by_head(sh.dh, vec, [&](auto dk, auto v) {
    constexpr int DK = decltype(dk)::value, lds = state_lds<T, DK>();
    constexpr bool VEC = decltype(v)::value;
    static LdsLimit limit;
    const hipError_t le = limit.raise(reinterpret_cast<const void*>(k_linear_states<T, DK, VEC>), lds);
    if (le != hipSuccess) return le;
    k_linear_states<T, DK, VEC><<<blocks, 4 * DK, lds, c.stream>>>(jobs, sh, units);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  uintptr_t low = 0;
  for (int i = 0; i < njobs; ++i) low |= (uintptr_t)jobs.j[i].loc | (uintptr_t)jobs.j[i].init | (uintptr_t)jobs.j[i].fin;
  const int dd = sh.dh * sh.dh;
  if (dd % 4 == 0 && (low & 15) == 0) k_linear_scan<4><<<dim3((dd / 4 + 255) / 256, sh.B * sh.H, njobs), 256, 0, c.stream>>>(jobs, sh);
  else k_linear_scan<1><<<dim3((dd + 255) / 256, sh.B * sh.H, njobs), 256, 0, c.stream>>>(jobs, sh);
  return hipGetLastError();
}

bool shape_ok(int dt, int B, int S, int H, int dh) {
  return (dt == F32 || dt == BF16) && B >= 0 && S >= 0 && S <= 1 << 30 && H >= 1 && dh >= 1 && dh <= kMaxHead &&
         (int64_t)B * H <= 8 * 65535 &&         // grid; more than one segment a sequence only where there are few
         (int64_t)3 * H * dh < 1 << 24;         // offsets inside a chunk: 24-bit rows, 32-bit bytes
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
  size_t n = 0;
  for (int dt : {F32, BF16})                     // enough for either compute dtype
    if (shape_ok(dt, B, S, H, dh)) n = std::max(n, cut_elems(cut_of(dt, B, S, H, dh, backward ? 3 : 1), B, H, dh, backward));
  return n;
}

hipError_t op_linear_attn_fwd(const OpCtx& c, const void* qkv, const float* log_decay, const int32_t* lens, const float* s0, void* o,
                              float* s_out, int B, int S, int H, int dh) {
  ProfScope prof_(c, KC_ATTN_FWD);
  if (!shape_ok(c.dt, B, S, H, dh)) return hipErrorInvalidValue;
  if (B == 0) return hipSuccess;
  if (!log_decay || (S > 0 && (!qkv || !o))) return hipErrorInvalidValue;
  const Cut cut = cut_of(c.dt, B, S, H, dh, 1);
  if (cut.segments > 1 && (!c.partial || c.partial_elems < cut_elems(cut, B, H, dh, false))) return hipErrorInvalidValue;
  const LinearShape sh = shape_of(cut, log_decay, lens, B, S, H, dh);
  const bool vec = whole_chunks(dh, {qkv, o});
  const size_t e = dtype_size(c.dt);
  const int d = H * dh;
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
  const Cut cut = cut_of(c.dt, B, S, H, dh, 3);
  if (cut.segments > 1 && (!c.partial || c.partial_elems < cut_elems(cut, B, H, dh, true))) return hipErrorInvalidValue;
  const LinearShape sh = shape_of(cut, log_decay, lens, B, S, H, dh);
  const bool vec = whole_chunks(dh, {qkv, dout, dqkv});
  const size_t e = dtype_size(c.dt);
  const int d = H * dh;
  const char *q = (const char*)qkv, *k = q + d * e, *v = k + d * e;
  char* dq = (char*)dqkv;
  const float up = (float)sqrt((double)dh);        // the states of the way back are kept without the factor dh^-1/2
  auto job = [&](const void* jq, int ldq, const void* jk, int ldk, const void* jv, int ldv, void* out, int back) {
    LinearJob j = {};
    j.q = jq; j.ldq = ldq; j.k = jk; j.ldk = ldk; j.v = jv; j.ldv = ldv; j.out = out; j.ldo = 3 * d; j.back = back;
    j.in_scale = back ? up : 1.f; j.out_scale = sh.scale;
    j.init = back ? ds_out : s0;
    return j;
  };
  const int w = 3 * d;
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
  if ((c.dt != F32 && c.dt != BF16) || B < 0 || H < 1 || dh < 1 || dh > kMaxHead || (int64_t)B * H >= 1 << 24 ||
      (int64_t)3 * H * dh > 0x7fffffff) return hipErrorInvalidValue;
  if (B == 0) return hipSuccess;
  if (!qkv || !log_decay || !state || !o) return hipErrorInvalidValue;
  const float scale = (float)(1.0 / sqrt((double)dh));
  if (c.dt == BF16) k_linear_step<bf16_t><<<B * H, 256, 0, c.stream>>>((const bf16_t*)qkv, log_decay, state, (bf16_t*)o, H, dh, scale);
  else k_linear_step<float><<<B * H, 256, 0, c.stream>>>((const float*)qkv, log_decay, state, (float*)o, H, dh, scale);
  return hipGetLastError();
}

}  // namespace lp
