// Attention over the 8-bit cache (cache.h has the layout): o = softmax(q k^T dh^-1/2) v over a sequence's positions, without or with those
// behind the row's own.
//
// The rows of a sequence that read one head of the cache, n new tokens times the G query heads that share it, are the columns of a tile;
// 64 tokens of the cache are its rows.  A wave keeps both products transposed, on the 16 x 16 x 32 matrix instruction:
//   S^T[token, column] = K Q^T,   O^T[dh, column] += V^T P^T
// Lane l has column l % 16 of S^T; which tokens the rows of K stand for is free, and they are dealt so that the lane's sixteen
// scores belong to the tokens 16 (l / 16) .. + 15, in order: what it then needs of V^T for each of its columns of a head is one access of sixteen bytes, the operand of
// two products, and sixteen tokens never leave a page, so that a lane has one page, one scale of the keys and one of the
// values.  Neither scores nor weights go through LDS.
// Codes become bf16 by one conversion instruction, exactly.  The scales multiply scores and weights in fp32.  Weights enter the second
// product as the sum of two bf16 parts (three where the call is in fp32, whose queries are cut in three as well): what is left out is 2^-16 of a weight (2^-24), so
// that an output is off by its own rounding and no more.  A third part in bf16 would turn the rounding of one output in a hundred and cost 3 % of 192 single tokens (heads of 128, 166 -> 171 us) and 7 % of eight rows.
#include <type_traits>

#include "cache.h"
#include "vec8.h"

namespace lp {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kWaves = 4;                                  // of a block where axes are divided

struct AttnArgs {
  const void* q;
  void* o;
  float *lse, *part;        // part: what the pieces of a divided axis leave
  int64_t ldq, ldo;
  int H, G, causal, tiles;  // tiles: column tiles of a sequence, at most
  unsigned by_g;            // 2^32 / G, rounded up: quotients of numbers below 2^12 by products; not for 1
  int target;               // pieces that the axes are divided into, about (0: none is divided)
  bool vec;
  float scale;
};

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Eight codes, as the numbers they are.
__device__ __forceinline__ bf16x8 codes8(unsigned a, unsigned b) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  bf16x8 v;
  v[0] = p[0]; v[1] = p[1]; v[2] = q[0]; v[3] = q[1]; v[4] = r[0]; v[5] = r[1]; v[6] = s[0]; v[7] = s[1];
  return v;
}
// Eight numbers as sums of N bf16 parts, each the nearest to what the ones before leave: two leave 2^-16 of a number, three nothing.
template <int N>
__device__ __forceinline__ void split8(float (&r)[8], bf16x8 (&f)[N]) {
#pragma unroll
  for (int s = 0; s < N; ++s) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[s][e] = (bf16_t)r[e];
    if (s + 1 < N) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] -= (float)f[s][e];
    }
  }
}
// 0xff where a byte is a NaN's code.
__device__ __forceinline__ unsigned nan_bytes(unsigned w) {
  const unsigned hit = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (hit >> 7) * 0xffu;
}

// The largest of three; NaN count only where there is nothing else.  In C, which becomes the instruction of that name: scores come straight from the matrix
// unit, and the compiler sees to the wait states (8 behind a 16 x 16 x 32 product, 12 behind one of 32 x 32 x 16) for its own instructions only, not for those of inline asm.
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// What a block works on.
struct Work { int b, h, tile, piece, pieces, slot; };

// Sums over the lanes up to a lane's own; the last one's is the sum of all.  (Sixteen by sixteen lanes, then across: 6 additions without LDS.)
__device__ __forceinline__ unsigned running_sum(unsigned v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // lanes 1, 2, 4 and 8 before, in a row of sixteen
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // a row's last lane to the next row, in rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // lane 31 to rows 2 and 3
  return v;
}

// The axes are cut so that all pieces have the same number of tiles, whatever the sequences' lengths: as many as leave about `target` pieces in
// all.  Pieces are numbered through sequences, heads, column tiles and the axis; this finds piece `id`, alike in every wave and without a barrier.  The host has
// seen to it that the sums fit 32 bits.
__device__ __forceinline__ bool find_work(const CacheView& c, const AttnArgs& a, int width, unsigned id, Work* w) {
  const unsigned number = id;
  const int lane = threadIdx.x & 63;
  auto size_of = [&](int b, unsigned* tiles) {               // of a head: column tiles, and tiles of the axis
    const Sequence s = sequence_of(c, b);
    *tiles = (unsigned)(s.len + 63) >> 6;
    return ((unsigned)s.n * a.G + width - 1) / width;
  };
  unsigned all = 0, tiles = 0, columns = 0;
  for (int b = lane; b < c.B; b += 64) {
    columns = size_of(b, &tiles);
    all += columns * tiles;
  }
  all = (unsigned)__builtin_amdgcn_readlane((int)running_sum(all), 63) * c.Hkv;
  unsigned each = (all + a.target - 1) / a.target;
  if (each < kWaves) each = kWaves;
  for (int b0 = 0; b0 < c.B; b0 += 64) {
    const int b = b0 + lane;
    if (c.B > 64) {
      columns = tiles = 0;
      if (b < c.B) columns = size_of(b, &tiles);
    }
    const unsigned pieces = tiles > each ? (tiles + each - 1) / each : 1;
    const unsigned n = columns * c.Hkv * pieces, run = running_sum(n);
    const unsigned long long past = __ballot(id < run);
    if (past) {
      const int at = __builtin_ctzll(past);
      const unsigned i = id - (unsigned)(__builtin_amdgcn_readlane((int)run, at) - __builtin_amdgcn_readlane((int)n, at));
      const unsigned ps = __builtin_amdgcn_readlane((int)pieces, at), cs = __builtin_amdgcn_readlane((int)columns, at);
      const unsigned pair = ps == 1 ? i : i / ps, h = cs == 1 ? pair : pair / cs;
      w->b = b0 + at;
      w->piece = (int)(i - pair * ps);
      w->pieces = (int)ps;
      w->h = (int)h;
      w->tile = (int)(pair - h * cs);
      w->slot = (int)number;
      return true;
    }
    id -= (unsigned)__builtin_amdgcn_readlane((int)run, 63);
  }
  return false;
}
// What pieces leave: for every (sequence, head, column tile) its first piece and their number, then for every piece sums of `width` columns, largest scores
// and sums of weights.
__device__ __forceinline__ int64_t piece_at(int pairs, int width, int dh, int64_t slot) {
  return ((pairs * 2 + 15) & ~15) + slot * width * (dh + 2);
}
__device__ __forceinline__ void note_pieces(const CacheView& c, const AttnArgs& a, const Work& w) {
  if (w.piece == 0 && threadIdx.x == 0)
    reinterpret_cast<int2*>(a.part)[((int64_t)w.b * c.Hkv + w.h) * a.tiles + w.tile] = make_int2(w.slot, w.pieces);
}
// Tiles of a piece: [first, last).
__device__ __forceinline__ void tiles_of(int tiles, int piece, int pieces, int* first, int* last) {
  const int each = (tiles + pieces - 1) / pieces;
  *first = piece * each;
  *last = *first + each < tiles ? *first + each : tiles;
}

// A column's row of q and o, and its head's first column there.
struct Column { int64_t row; int head, t; bool there; };
__device__ __forceinline__ Column column_of(const Sequence& s, const AttnArgs& a, int h, int col) {
  Column c;
  c.t = col / a.G;
  c.there = c.t < s.n;
  c.row = s.first + c.t;
  c.head = h * a.G + col - c.t * a.G;
  return c;
}

template <typename T>
__device__ __forceinline__ void put4(T* p, f32x4 v, bool vec) {
  if constexpr (std::is_same<T, float>::value) {
    if (vec) { *reinterpret_cast<f32x4*>(p) = v; return; }
  } else {
    bf16x4 t;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (bf16_t)v[e];
    if (vec) { *reinterpret_cast<bf16x4*>(p) = t; return; }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) p[e] = from_f<T>(v[e]);
}
// The end of a row: its sum of weights l (negative: all its scores are minus infinity), their maximum m in powers of two.  No token: zeros.
__device__ __forceinline__ float over(float m, float l) {
  if (m == -INFINITY && l == 0.f) return 0.f;                        // times this, the sums are zeros
  return l < 0.f ? __builtin_bit_cast(float, 0x7fc00000u) : 1.f / l;
}
__device__ __forceinline__ float log_sum(float m, float l) { return m == -INFINITY && l <= 0.f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2; }

// The larger of the numbers of the four lanes of a column.
__device__ __forceinline__ float max_of_column(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned x = r[0], y = r[1];         // copied: a bit cast straight from a vector's element takes the first one
  const float m = fmaxf(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
  const unsigned n = __builtin_bit_cast(unsigned, m);
  const auto q = __builtin_amdgcn_permlane16_swap(n, n, false, false);
  const unsigned e = q[0], f = q[1];
  return fmaxf(__builtin_bit_cast(float, e), __builtin_bit_cast(float, f));
}

// ND: head size in units of 64 columns, rounded up.  NC: column tiles of 16.  W: waves, each with every W-th tile of 64 tokens.  ONE: a tile is in one
// page (pages of 64 tokens or more), whose address is a scalar; otherwise each lane finds its runs' pages.  The keys of the next tile are on their way while one is
// worked on, and the page number of the one after that; its values while its scores are computed.  Loads are never skipped: where there is no page, page 0
// is read and its scores and values are taken out, and columns behind the head's repeat its last sixteen, against zeros of the query.
template <typename T, int ND, int NC, int W, bool ONE>
__global__ void __launch_bounds__(64 * W, ND * NC <= 2 ? 2 : 1) k_cache_attn(CacheView c, AttnArgs a) {
  constexpr int QP = std::is_same<T, float>::value ? 3 : 1, WP = std::is_same<T, float>::value ? 3 : 2, NJ = 4 * ND;
  constexpr int kPad = 64 * ND + 4, width = 16 * NC, kFrags = (NC * ND * 2 + W - 1) / W;
  // the queries, and when the axis is done what waves hand to each other
  constexpr int kQueries = NC * ND * 2 * QP * 64 * 16, kJoin = W * width * (kPad + 2) * 4;
  __shared__ __align__(16) char lds[kQueries > kJoin ? kQueries : kJoin];
  auto sq = reinterpret_cast<bf16x8(*)[64]>(lds);
  auto so = reinterpret_cast<float(*)[width][kPad]>(lds);
  auto sml = reinterpret_cast<float2(*)[width]>(lds + W * width * kPad * 4);
  Work w;
  const unsigned id = blockIdx.y * gridDim.x + blockIdx.x;
  if (a.target) {
    if (!find_work(c, a, width, id, &w)) return;
    note_pieces(c, a, w);
  } else {
    const unsigned pair = a.tiles == 1 ? id : id / a.tiles;
    w.tile = (int)(id - pair * a.tiles);
    w.b = (int)(pair / c.Hkv);
    w.h = (int)(pair - w.b * c.Hkv);
    w.piece = w.slot = 0;
    w.pieces = 1;
    if (w.b >= c.B) return;
  }
  const Sequence s = sequence_of(c, w.b);
  const int col0 = w.tile * width, columns = s.n * a.G;
  if (col0 >= columns) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const int dh = c.dh, page = 1 << c.shift;
  const int64_t page_bytes = (int64_t)c.Hkv * dh << c.shift;
  // a column's token among the new ones: there are few columns, so that the quotient by G is a product
  auto new_of = [&](int col) { return a.G == 1 ? col : (int)__umulhi((unsigned)col, a.by_g); };
  auto limit = [&](int t) {
    const int v = a.causal ? s.len - s.n + t + 1 : s.len;
    return v < 0 ? 0 : v;
  };

  // queries on their way
  float qv[kFrags][8];
#pragma unroll
  for (int u = 0; u < kFrags; ++u) {
    const int f = wave + u * W, half = f & 1, cc = f / 2 % ND, d = cc * 64 + g * 16 + half * 8, col = col0 + f / (2 * ND) * 16 + i, t = new_of(col);
#pragma unroll
    for (int e = 0; e < 8; ++e) qv[u][e] = 0.f;
    if (f < NC * ND * 2 && t < s.n && d < dh) {
      const T* p = (const T*)a.q + (s.first + t) * a.ldq + (w.h * a.G + col - t * a.G) * dh + d;
      if (a.vec) {
        load8(p, qv[u]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) qv[u][e] = to_f(p[e]);
      }
    }
  }

  // visible tokens of the first and of the last column there is, and of the lane's columns (0: none)
  const int lo = limit(new_of(col0)), hi = limit(new_of(col0 + width < columns ? col0 + width - 1 : columns - 1));
  int lim[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int t = new_of(col0 + n * 16 + i);
    lim[n] = t < s.n ? limit(t) : 0;
  }
  int tile, last;
  if (w.pieces == 1) {
    tile = 0;
    last = (hi + 63) >> 6;
  } else {
    tiles_of((s.len + 63) >> 6, w.piece, w.pieces, &tile, &last);
    if (last > (hi + 63) >> 6) last = (hi + 63) >> 6;
  }
  tile += wave;

  struct Pages { int k, v; };            // of the tokens whose keys, and whose scores and values, the lane has
  struct Keys { uint4 k[4][ND]; };
  auto pages_of = [&](int t) {
    if constexpr (ONE) {
      const int p = __builtin_amdgcn_readfirstlane(page_of(c, w.b, t * 64 >> c.shift));
      return Pages{p, p};
    } else {
      const int kt = t * 64 + 16 * (i >> 2), vt = t * 64 + 16 * g;
      return Pages{kt < hi ? page_of(c, w.b, kt >> c.shift) : -1, vt < hi ? page_of(c, w.b, vt >> c.shift) : -1};
    }
  };
  const uint8_t *kh = c.k + ((int64_t)w.h * dh << c.shift), *vh = c.v + ((int64_t)w.h * dh << c.shift);
  unsigned koff[ND];
#pragma unroll
  for (int cc = 0; cc < ND; ++cc) {
    const int d = cc * 64 + g * 16;
    koff[cc] = (unsigned)((ONE ? 16 * (i >> 2) + (i & 3) : i & 3) * dh + (d < dh ? d : dh - 16));
  }
  const unsigned voff = ((unsigned)i << c.shift) + (ONE ? 16 * g : 0);
  auto load = [&](int t, const Pages& p, Keys& x) {
    const int at = (ONE ? t * 64 : t * 64 + 16 * (i >> 2)) & (page - 1);
    const uint8_t* kp = kh + ((p.k < 0 ? 0 : p.k) * page_bytes + at * dh);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int cc = 0; cc < ND; ++cc) x.k[u][cc] = *reinterpret_cast<const uint4*>(kp + u * 4 * dh + koff[cc]);
  };
  Keys one, two;
  Pages now{-1, -1}, ahead{-1, -1};
  if (tile < last) {
    now = pages_of(tile);
    load(tile, now, one);
    if (tile + W < last) ahead = pages_of(tile + W);
  }

#pragma unroll
  for (int u = 0; u < kFrags; ++u) {
    const int f = wave + u * W;
    bf16x8 parts[QP];
    split8<QP>(qv[u], parts);
    if (f < NC * ND * 2) {
#pragma unroll
      for (int q = 0; q < QP; ++q) sq[f * QP + q][lane] = parts[q];
    }
  }
  __syncthreads();

  f32x4 acc[NC][NJ];
  float m[NC], l[NC];
  bool seen[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = -INFINITY;
    l[n] = 0.f;
    seen[n] = false;
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto attend = [&](int t, const Keys& x, Keys& next) {
    const int tok = t * 64, vt = tok + 16 * g, pv = now.v;
    uint4 vr[NJ];
    float ks, vs;
    {
      const int p = pv < 0 ? 0 : pv;
      const int64_t where = (int64_t)p * c.Hkv + w.h;
      ks = c.ks[where];
      vs = c.vs[where];
      const uint8_t* vp = vh + (p * page_bytes + ((ONE ? tok : vt) & (page - 1)));
#pragma unroll
      for (int j = 0; j < NJ; ++j) vr[j] = *reinterpret_cast<const uint4*>(vp + ((j * 16 < dh ? j * 16 : dh - 16) << c.shift) + voff);
    }
    if (t + W < last) {
      load(t + W, ahead, next);
      now = ahead;
      if (t + 2 * W < last) ahead = pages_of(t + 2 * W);
    }
    const bool masked = tok + 64 > lo || (ONE ? pv < 0 : __ballot(pv < 0) != 0);
    f32x4 sc[NC][4];
#pragma unroll
    for (int cc = 0; cc < ND; ++cc)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8 kf[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) kf[u] = half ? codes8(x.k[u][cc].z, x.k[u][cc].w) : codes8(x.k[u][cc].x, x.k[u][cc].y);
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
          for (int q = QP - 1; q >= 0; --q) {
            const bf16x8 qf = sq[((n * ND + cc) * 2 + half) * QP + q][lane];
#pragma unroll
            for (int u = 0; u < 4; ++u) sc[n][u] = mma(kf[u], qf, cc == 0 && half == 0 && q == QP - 1 ? f32x4{} : sc[n][u]);
          }
      }

    // where there is no page its scale, which may be anything, is none
    ks = pv < 0 ? 1.f : ks * a.scale;
    vs = pv < 0 ? 0.f : vs;
    bf16x8 wf[NC][2][WP];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      if (masked) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool ok = vt + u * 4 + r < lim[n] && pv >= 0;
            sc[n][u][r] = ok ? sc[n][u][r] : -INFINITY;
            seen[n] |= ok;
          }
      } else {
        seen[n] = true;
      }
      float best = -INFINITY;
#pragma unroll
      for (int u = 0; u < 4; ++u) best = max3(max3(best, sc[n][u][0], sc[n][u][1]), sc[n][u][2], sc[n][u][3]);
      const float top = fmaxf(max_of_column(best * ks), m[n]), base = top == -INFINITY ? 0.f : top;
      if (__ballot(top > m[n])) {
        const float f = __builtin_amdgcn_exp2f(m[n] - base);
        l[n] *= f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[n][j] *= f;
        m[n] = top;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][2 * half + e / 4][e % 4], ks, -base));
          l[n] += p[e];
          p[e] *= vs;
        }
        split8<WP>(p, wf[n][half]);
      }
    }

    if (masked) {
      // what stands behind the last visible token, or in no page, is not read as a number
      const int left = pv < 0 ? 0 : hi - vt;
      unsigned keep[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int b = left - 4 * q;
        keep[q] = b >= 4 ? 0xffffffffu : b <= 0 ? 0u : (1u << (8 * b)) - 1u;
      }
      unsigned any = 0;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        vr[j].x &= keep[0]; vr[j].y &= keep[1]; vr[j].z &= keep[2]; vr[j].w &= keep[3];
        if (lo < hi) any |= nan_bytes(vr[j].x) | nan_bytes(vr[j].y) | nan_bytes(vr[j].z) | nan_bytes(vr[j].w);
      }
      // A NaN's product is a NaN also with the weight of a column that does not see it.  So it leaves the product, and the columns that do
      // see one are told by a product of their own: ones where there is a NaN, times ones where a column sees.
      if (__ballot(any != 0)) {
        bf16x8 see[NC][2];
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < 8; ++e) see[n][half][e] = (bf16_t)(vt + half * 8 + e < lim[n] ? 1.f : 0.f);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const unsigned b[4] = {nan_bytes(vr[j].x), nan_bytes(vr[j].y), nan_bytes(vr[j].z), nan_bytes(vr[j].w)};
          const bf16x8 one0 = codes8(b[0] & 0x38383838u, b[1] & 0x38383838u), one1 = codes8(b[2] & 0x38383838u, b[3] & 0x38383838u);
          vr[j].x &= ~b[0]; vr[j].y &= ~b[1]; vr[j].z &= ~b[2]; vr[j].w &= ~b[3];
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            f32x4 hits = {0.f, 0.f, 0.f, 0.f};
            hits = mma(one0, see[n][0], hits);
            hits = mma(one1, see[n][1], hits);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (hits[r] > 0.f) acc[n][j][r] = __builtin_bit_cast(float, 0x7fc00000u);
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const bf16x8 v0 = codes8(vr[j].x, vr[j].y), v1 = codes8(vr[j].z, vr[j].w);
#pragma unroll
      for (int n = 0; n < NC; ++n)
#pragma unroll
        for (int q = WP - 1; q >= 0; --q) {
          acc[n][j] = mma(v0, wf[n][0][q], acc[n][j]);
          acc[n][j] = mma(v1, wf[n][1][q], acc[n][j]);
        }
    }
  };
  for (; tile < last; tile += 2 * W) {
    attend(tile, one, two);
    if (tile + W < last) attend(tile + W, two, one);
  }

  // the four lanes of a column, then all waves at once: a thread has four columns of the head of one row
  __syncthreads();                       // the queries have been read
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    l[n] += __shfl_xor(l[n], 16, 64);
    l[n] += __shfl_xor(l[n], 32, 64);
    int any = seen[n];
    any |= __shfl_xor(any, 16, 64);
    any |= __shfl_xor(any, 32, 64);
    if (any && m[n] == -INFINITY && l[n] == 0.f) l[n] = -1.f;
    if (col0 + n * 16 + i >= columns) continue;
    if (g == 0) sml[wave][n * 16 + i] = make_float2(m[n], l[n]);
#pragma unroll
    for (int j = 0; j < NJ; ++j) *reinterpret_cast<f32x4*>(&so[wave][n * 16 + i][j * 16 + g * 4]) = acc[n][j];
  }
  __syncthreads();
  const int quads = dh / 4, there = columns - col0 < width ? columns - col0 : width;
  for (int it = threadIdx.x; it < there * quads; it += 64 * W) {
    const int n = it / quads, d = (it - n * quads) * 4;
    float2 ml[W];
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < W; ++v) {
      ml[v] = sml[v][n];
      top = fmaxf(top, ml[v].x);
    }
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    bool none = false;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float f = __builtin_amdgcn_exp2f(ml[v].x - base);
      none |= ml[v].y < 0.f;
      sum += ml[v].y < 0.f ? 0.f : top == -INFINITY ? ml[v].y : ml[v].y * f;        // minus infinity: no scores but such (or NaN)
      o += *reinterpret_cast<const f32x4*>(&so[v][n][d]) * f;
    }
    if (none && top == -INFINITY && sum == 0.f) sum = -1.f;
    if (w.pieces > 1) {
      float* out = a.part + piece_at(c.B * c.Hkv * a.tiles, width, dh, w.slot);
      if (d == 0) *reinterpret_cast<float2*>(out + width * dh + n * 2) = make_float2(top, sum);
      *reinterpret_cast<f32x4*>(out + n * dh + d) = o;
    } else {
      const int t = new_of(col0 + n), head = w.h * a.G + col0 + n - t * a.G;
      const int64_t row = s.first + t;
      if (a.lse && d == 0) a.lse[row * a.H + head] = log_sum(top, sum);
      put4((T*)a.o + row * a.ldo + head * dh + d, o * over(top, sum), a.vec);
    }
  }
}

// ------------------------------------------------------------------------------------------------ many rows
// The same for calls with many columns (prompts, chunks of them): a block has 128 columns, a wave 32 of them, and tiles of 64
// tokens go through LDS, as numbers, for all its waves: keys in bf16, values in f16 (bf16 in fp32 calls), each code converted once.  Products are 32 x 32 x 16; the rows of K are dealt
// to tokens so that a lane's eight scores, and its operand of the second product, are eight tokens in order (token_of).
// In fp32 weights enter the second product in three bf16 parts, all their 24 bits; in bf16 in f16, whose eleven bits leave 2^-12 of a weight, a sixteenth of the output's own rounding: codes of 8 bits are f16 numbers too.  Neither
// has room for a weight times any scale of its values, so that they are held relative to the largest such product that the row has met (`top`), at 2^7 of which one stands; both it
// and the largest score lag by a factor of up to 2^8, so that sums are seldom rescaled.  One exponential gives a weight with its values' scale; the sum of weights takes the scale out
// again, run by run, and is of 32-bit numbers.  In f16 2^-32 of `top` is lost of small products, which a page of a larger scale may be the cause of while its numbers in a column are zeros: where `top` is
// more than 2^8 times the row's largest weight times the scale of a run of the tile, the tile's weights are two bf16 parts (2^-16 of a weight; bf16 has the range of fp32).  So of a value
// 2^-24 of the row's largest weight is lost at most, whatever the other pages hold.
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

__device__ __forceinline__ f32x16 mma32(const bf16x8& a, const bf16x8& b, const f32x16& c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(const f16x8& a, const f16x8& b, const f32x16& c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f16x8 codes8_f16(unsigned a, unsigned b) {
  const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
  const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
  f16x8 v;
  v[0] = p[0]; v[1] = p[1]; v[2] = q[0]; v[3] = q[1]; v[4] = r[0]; v[5] = r[1]; v[6] = s[0]; v[7] = s[1];
  return v;
}
template <typename V> __device__ __forceinline__ auto codes8_as(unsigned a, unsigned b) {
  if constexpr (std::is_same<V, bf16_t>::value) return codes8(a, b);
  else return codes8_f16(a, b);
}
// Codes that stand in f16, in bf16: both hold them.
__device__ __forceinline__ bf16x8 in_bf16(const bf16x8& v) { return v; }
__device__ __forceinline__ bf16x8 in_bf16(const f16x8& v) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (bf16_t)(float)v[e];
  return r;
}
// Token of a tile of 32 that row `r` of a product stands for: values 8 kk .. 8 kk + 7 of lane l are rows 16 kk + 4 (l / 32) + {0..3, 8..11}, tokens
// 16 kk + 8 (l / 32) + {0..7}.
__device__ __forceinline__ int token_of(int r) { return (r & 16) | (r & 4) << 1 | (r & 8) >> 1 | (r & 3); }
// The larger of the two halves' numbers.  (The exchange's results are copied first: a bit cast straight from a vector's element takes the first one.)
__device__ __forceinline__ float both_max(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned x = r[0], y = r[1];
  return fmaxf(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
}

constexpr int kRuns = 128;                 // of sixteen tokens, whose pages and scales are known to a block ahead of their tiles
// k, v: bytes of the pools before the run's in the block's head (where there is no page, those of page 0).
struct Runs { int64_t k[kRuns], v[kRuns]; int here[kRuns]; float ks[kRuns], lv[kRuns], rv[kRuns]; };
// Where axes are whole: block `n` in the order of the column tiles' numbers, last tiles (the longest chains of a prompt) first, through the sequences that have
// such a tile and their heads.  Numbered without gaps, so that whatever share of the blocks a compute unit gets, in turn as they come, is like the others' (8 prompts of 4096, 3584
// .. 512, 12 heads, with a place kept for every sequence and tile: 141 to 196 us by how the places fell on the units).
__device__ __forceinline__ bool find_longest(const CacheView& c, const AttnArgs& a, int width, int64_t n, Work* w) {
  w->piece = w->slot = 0;
  w->pieces = 1;
  if (c.B > 64) {
    const int pairs = c.B * c.Hkv, turn = (int)(n / pairs), pair = (int)(n - (int64_t)turn * pairs);
    w->tile = a.tiles - 1 - turn;
    w->b = pair / c.Hkv;
    w->h = pair - w->b * c.Hkv;
    return turn < a.tiles;
  }
  const int lane = threadIdx.x & 63;
  const unsigned own = lane < c.B ? ((unsigned)sequence_of(c, lane).n * a.G + width - 1) / width : 0;
  auto from = [&](unsigned t) {          // column tiles of a head from number t on
    return (unsigned)__builtin_amdgcn_readlane((int)running_sum(own > t ? own - t : 0u), 63);
  };
  const unsigned unit = (unsigned)(n / c.Hkv);
  w->h = (int)(n - (int64_t)unit * c.Hkv);
  unsigned t = 0, end = a.tiles;
  if (unit >= from(0)) return false;
  while (end - t > 1) {
    const unsigned mid = (t + end) / 2;
    if (from(mid) > unit) t = mid;
    else end = mid;
  }
  unsigned long long who = __ballot(own > t);
  for (unsigned skip = unit - from(t + 1); skip; --skip) who &= who - 1;
  w->tile = (int)t;
  w->b = __builtin_ctzll(who);
  return true;
}

// NB: head size in units of 32 columns, rounded up.  Two waves a SIMD up to heads of 128, although fp32 then keeps 26 registers in scratch memory over 96: heads of 128, chunks of 509 rows 154 us and 168 with one
// wave and none there, prompts of 2048 185 and 219.
template <typename T, int NB>
__global__ void __launch_bounds__(256, NB <= 4 ? 2 : 1) k_cache_prompt(CacheView c, AttnArgs a) {
  constexpr bool F = std::is_same<T, float>::value;
  constexpr int QP = F ? 3 : 1, WP = F ? 3 : 2, DH = 32 * NB, KLD = DH + 8, VLD = 72, kLoads = (64 * (DH / 16) + 255) / 256;
  constexpr float kTop = 7.f, kLag = 8.f, kLeast = F ? -60.f : kTop - 8.f;
  typedef typename std::conditional<F, bf16_t, _Float16>::type V;            // numbers that values are held in
  typedef __attribute__((ext_vector_type(8))) V V8;
  __shared__ __align__(16) bf16_t sk[2][64][KLD];
  __shared__ __align__(16) V sv[2][DH][VLD];
  __shared__ __align__(16) Runs runs[2];
  __shared__ __align__(8) unsigned short snan[2][DH][4];     // of a tile that not all columns see: which of a column's sixteen tokens are NaN
  const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int dh = c.dh, page = 1 << c.shift, width = 128;
  Work w;
  if (a.target) {
    if (!find_work(c, a, width, (unsigned)id, &w)) return;
    note_pieces(c, a, w);
  } else {
    if (!find_longest(c, a, width, id, &w)) return;
  }
  const Sequence s = sequence_of(c, w.b);
  const int col0 = w.tile * width, columns = s.n * a.G;
  if (col0 >= columns) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 31, half = lane >> 5, first = col0 + wave * 32;

  auto limit = [&](int t) {
    const int v = a.causal ? s.len - s.n + t + 1 : s.len;
    return v < 0 ? 0 : v;
  };
  // visible tokens: of the block's first and last column there is, of the wave's, of the lane's
  const int blo = limit(col0 / a.G), bhi = limit((col0 + width < columns ? col0 + width - 1 : columns - 1) / a.G);
  const int lo = limit(first / a.G), hi = first >= columns ? 0 : limit((first + 32 < columns ? first + 31 : columns - 1) / a.G);
  int tile, last;
  tiles_of((((a.target ? s.len : bhi) + 63) >> 6), w.piece, w.pieces, &tile, &last);
  if (last > (bhi + 63) >> 6) last = (bhi + 63) >> 6;

  const int64_t page_bytes = (int64_t)c.Hkv * dh << c.shift;
  // 32 tiles' runs from tile t on; the two sets take turns
  auto known = [&](int t) -> Runs& { return runs[(t - tile) >> 5 & 1]; };
  auto look_up = [&](int t) {
    if (tid >= kRuns) return;
    const int at = t * 64 + tid * 16, p = at < bhi ? page_of(c, w.b, at >> c.shift) : -1;
    const int64_t where = (int64_t)(p < 0 ? 0 : p) * c.Hkv + w.h;
    const float vs = p < 0 ? 1.f : c.vs[where];
    Runs& r = known(t);
    r.k[tid] = (p < 0 ? 0 : p) * page_bytes + (at & (page - 1)) * dh;
    r.v[tid] = (p < 0 ? 0 : p) * page_bytes + (at & (page - 1));
    r.here[tid] = p < 0 ? 0 : -1;
    r.ks[tid] = p < 0 ? 1.f : c.ks[where] * a.scale;
    r.lv[tid] = __builtin_amdgcn_logf(vs);
    r.rv[tid] = 1.f / vs;
  };
  if (tile < last) look_up(tile);

  int lim;
  bf16x8 qf[2 * NB][QP];
  {
    const Column col = column_of(s, a, w.h, first + i);
    lim = col.there ? limit(col.t) : 0;
#pragma unroll
    for (int k = 0; k < 2 * NB; ++k) {
      const int d = k * 16 + half * 8;
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (col.there && d < dh) {
        const T* p = (const T*)a.q + col.row * a.ldq + col.head * dh + d;
        if (a.vec) {
          load8(p, v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = to_f(p[e]);
        }
      }
      split8<QP>(v, qf[k]);
    }
  }

  f32x16 acc[NB];
  float m = -INFINITY, top = -INFINITY, l = 0.f;      // largest score; largest score plus the logarithm of its values' scale; sum of weights
  bool seen = false;
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[j][v] = 0.f;

  // A tile on its way: sixteen bytes of a token's keys, and of a column's values, a thread and load.  No load is skipped: where there is no page, page 0 is read
  // and its scores and values are taken out; keys behind the head's columns are its last ones, against zeros of the query, and what comes of values there
  // is not written.
  uint4 kr[kLoads], vr[kLoads];
  const uint8_t *kh[kLoads], *vh[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int x = tid + 256 * u, tok = x / (DH / 16), d = x % (DH / 16) * 16, e = x >> 2;
    kh[u] = c.k + ((int64_t)w.h * dh << c.shift) + (tok & 15) * dh + (d < dh ? d : dh - 16);
    vh[u] = c.v + (((int64_t)w.h * dh + (e < dh ? e : dh - 1)) << c.shift);
  }
  auto fetch = [&](int t) {
    const Runs& r = known(t);
    const int run0 = (t - tile & 31) * 4;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int x = tid + 256 * u;
      if (x >= 64 * (DH / 16)) continue;                   // whole waves
      kr[u] = *reinterpret_cast<const uint4*>(kh[u] + r.k[run0 + (x / (DH / 16) >> 4)]);
      vr[u] = *reinterpret_cast<const uint4*>(vh[u] + r.v[run0 + (x & 3)]);
    }
  };
  auto stage = [&](int t, int buf) {
    const Runs& kn = known(t);
    const int run0 = (t - tile & 31) * 4;
    const int4 here = *reinterpret_cast<const int4*>(&kn.here[run0]);
    const bool part = t * 64 + 64 > blo || (here.x & here.y & here.z & here.w) == 0;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int x = tid + 256 * u, tok = x / (DH / 16), d = x % (DH / 16);
      if (x >= 64 * (DH / 16)) continue;
      *reinterpret_cast<bf16x8*>(&sk[buf][tok][d * 16]) = codes8(kr[u].x, kr[u].y);
      *reinterpret_cast<bf16x8*>(&sk[buf][tok][d * 16 + 8]) = codes8(kr[u].z, kr[u].w);
      const int e = x >> 2, run = x & 3;
      {
        unsigned q[4] = {vr[u].x, vr[u].y, vr[u].z, vr[u].w};
        if (part) {
          // what stands behind the last visible token is no number; a NaN leaves the product, and is told to the columns that see it
          const int left = kn.here[run0 + run] ? bhi - (t * 64 + run * 16) : 0;
          unsigned bits = 0;
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const int b = left - 4 * z;
            q[z] &= b >= 4 ? 0xffffffffu : b <= 0 ? 0u : (1u << (8 * b)) - 1u;
            const unsigned bad = nan_bytes(q[z]);
            q[z] &= ~bad;
            bits |= ((bad & 1u) | (bad >> 7 & 2u) | (bad >> 14 & 4u) | (bad >> 21 & 8u)) << (4 * z);
          }
          snan[buf][e][run] = (unsigned short)bits;
        }
        *reinterpret_cast<V8*>(&sv[buf][e][run * 16]) = codes8_as<V>(q[0], q[1]);
        *reinterpret_cast<V8*>(&sv[buf][e][run * 16 + 8]) = codes8_as<V>(q[2], q[3]);
      }
    }
  };

  __syncthreads();
  if (tile < last) {
    fetch(tile);
    stage(tile, 0);
  }
  __syncthreads();
  for (int t = tile, buf = 0; t < last; ++t, buf ^= 1) {
    if (t + 1 < last) {
      if ((t + 1 - tile & 31) == 0) {
        look_up(t + 1);
        __syncthreads();
      }
      fetch(t + 1);
    }
    const int tok = t * 64;
    if (tok < hi) {
      const Runs& kn = known(t);
      const int run0 = (t - tile & 31) * 4;
      const f32x4 ks = *reinterpret_cast<const f32x4*>(&kn.ks[run0]), lv = *reinterpret_cast<const f32x4*>(&kn.lv[run0]),
                  rv = *reinterpret_cast<const f32x4*>(&kn.rv[run0]);
      const int4 pg = *reinterpret_cast<const int4*>(&kn.here[run0]);
      const bool away = (pg.x & pg.y & pg.z & pg.w) == 0, masked = tok + 64 > lo || away;
      f32x16 sc[2];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const bf16_t* kp = &sk[buf][g * 32 + token_of(i)][half * 8];
#pragma unroll
        for (int k = 0; k < 2 * NB; ++k) {
          const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kp + k * 16);
#pragma unroll
          for (int q = QP - 1; q >= 0; --q) sc[g] = mma32(kf, qf[k][q], k == 0 && q == QP - 1 ? f32x16{} : sc[g]);
        }
      }
      if (masked) {
        const int here[4] = {pg.x, pg.y, pg.z, pg.w};
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool ok = here[r] && tok + r * 16 + half * 8 + e < lim;
            sc[r >> 1][(r & 1) * 8 + e] = ok ? sc[r >> 1][(r & 1) * 8 + e] : -INFINITY;
            seen |= ok;
          }
      } else {
        seen = true;
      }
      float tm = -INFINITY, tt = -INFINITY;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x16& x = sc[r >> 1];
        const int v = (r & 1) * 8;
        const float best = fmaxf(max3(max3(x[v], x[v + 1], x[v + 2]), x[v + 3], x[v + 4]), max3(x[v + 5], x[v + 6], x[v + 7])) * ks[r];
        tm = fmaxf(tm, best);
        tt = fmaxf(tt, best + lv[r]);
      }
      tm = both_max(tm);
      tt = both_max(tt);
      if (__ballot(tm > m + kLag || tt > top + kLag)) {
        const float mn = fmaxf(m, tm), tn = fmaxf(top, tt);
        l *= mn == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        const float f = tn == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - tn);
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[j] *= f;
        m = mn;
        top = tn;
      }
      const float base = m == -INFINITY ? 0.f : m, off = kTop - (top == -INFINITY ? 0.f : top);
      // a weight with its values' scale stands at 2^(apart + lv) of the weight: where that is too little, or the way back leaves the range of 32 bits, it is taken from the weight
      const float apart = off + base, least = fminf(fminf(lv[0], lv[1]), fminf(lv[2], lv[3])) + apart;
      const bool thin = __ballot(least < kLeast || fabsf(apart) > 100.f) != 0;
      const float back = thin ? 0.f : __builtin_amdgcn_exp2f(-apart);
      auto weights = [&](int r, float up, float count, float (&p)[8]) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r >> 1][(r & 1) * 8 + e], ks[r], up));
          sum += p[e];
        }
        l = __builtin_fmaf(sum, count, l);
      };
      auto values = [&](int j, int r) { return *reinterpret_cast<const V8*>(&sv[buf][j * 32 + i][half * 8 + r * 16]); };
      if (F || thin) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p[8];
          bf16x8 wf[WP];
          if (thin) {
            const float e = fmaxf(lv[r] + apart, kTop), f = __builtin_amdgcn_exp2f(fminf(lv[r] + apart - kTop, 0.f));
            weights(r, e - base, __builtin_amdgcn_exp2f(-e), p);
#pragma unroll
            for (int q = 0; q < 8; ++q) p[q] *= f;
          } else {
            weights(r, lv[r] + off, back * rv[r], p);
          }
          split8<WP>(p, wf);
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const bf16x8 vf = in_bf16(values(j, r));
#pragma unroll
            for (int q = WP - 1; q >= 0; --q) acc[j] = mma32(vf, wf[q], acc[j]);
            if (!F) __builtin_amdgcn_sched_barrier(0);     // seldom taken: no registers beyond those of the other way
          }
        }
      }
      if constexpr (!F) {
        const float in = thin ? -INFINITY : off;           // all weights are zeros then: a way around would cost the sums their place in registers
        f16x8 wf[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p[8];
          weights(r, lv[r] + in, back * rv[r], p);
#pragma unroll
          for (int e = 0; e < 8; ++e) wf[r][e] = (_Float16)p[e];
        }
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[j] = mma32(values(j, r), wf[r], acc[j]);
      }
      if (tok + 64 > blo || away) {
        unsigned long long any = 0;
        for (int d = lane; d < DH; d += 64) any |= *reinterpret_cast<const unsigned long long*>(snan[buf][d]);
        if (__ballot(any != 0)) {
          const int left = lim - tok;                     // bits of pages that are not there are zeros
          const unsigned long long see = left >= 64 ? ~0ull : left <= 0 ? 0ull : (1ull << left) - 1;
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (*reinterpret_cast<const unsigned long long*>(snan[buf][j * 32 + 8 * (v / 4) + 4 * half + v % 4]) & see)
                acc[j][v] = __builtin_bit_cast(float, 0x7fc00000u);
        }
      }
    }
    if (t + 1 < last) stage(t + 1, buf ^ 1);
    __syncthreads();
  }

  l += __shfl_xor(l, 32, 64);
  int any = seen;
  any |= __shfl_xor(any, 32, 64);
  if (any && m == -INFINITY && l == 0.f) l = -1.f;
  const int at = first + i;
  const Column col = column_of(s, a, w.h, at);
  // from the weights' reference to the scores', in two steps of half the exponent: one may leave the range
  const float back = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(0.5f * (top - m - kTop));
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] *= back;
  if (!col.there) return;
  if (w.pieces > 1) {
    float* out = a.part + piece_at(c.B * c.Hkv * a.tiles, width, dh, w.slot);
    if (half == 0) *reinterpret_cast<float2*>(out + width * dh + (at - col0) * 2) = make_float2(m, l);
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        const int d = j * 32 + 2 * v + 4 * half;
        if (d < dh)
          *reinterpret_cast<f32x4*>(out + (at - col0) * dh + d) = f32x4{acc[j][v] * back, acc[j][v + 1] * back, acc[j][v + 2] * back, acc[j][v + 3] * back};
      }
  } else {
    const float f = over(m, l) * back;
    T* out = (T*)a.o + col.row * a.ldo + col.head * dh;
    if (a.lse && half == 0) a.lse[col.row * a.H + col.head] = log_sum(m, l);
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        const int d = j * 32 + 2 * v + 4 * half;
        if (d >= dh) continue;
        put4(out + d, f32x4{acc[j][v] * f, acc[j][v + 1] * f, acc[j][v + 2] * f, acc[j][v + 3] * f}, a.vec);
      }
  }
}

// ------------------------------------------------------------------------------------------------ divided axes
// The pieces of a divided axis, in their order.  A column belongs to a wave, or to the four of a block; a quad of its columns of the head to one lane
// for every so many pieces.
template <typename T, int WAVES>
__global__ void __launch_bounds__(256) k_cache_join(CacheView c, AttnArgs a, int width, unsigned groups) {
  __shared__ f32x4 sh[4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), dh = c.dh;
  const unsigned id = blockIdx.y * gridDim.x + blockIdx.x, pair = id / groups, pairs = c.B * c.Hkv * a.tiles;
  if (pair >= pairs) return;
  const int n = (int)(id - pair * groups) * (4 / WAVES) + (WAVES == 4 ? 0 : wave);
  const int tile = (int)(pair % a.tiles), h = (int)(pair / a.tiles % c.Hkv), b = (int)(pair / a.tiles / c.Hkv);
  const Sequence s = sequence_of(c, b);
  const Column col = column_of(s, a, h, tile * width + n);
  if (!col.there) return;                                          // with four waves a column: all of them
  const int2 which = reinterpret_cast<const int2*>(a.part)[pair];
  const int pieces = which.y;
  if (pieces < 2) return;
  const int64_t step = (int64_t)width * (dh + 2);
  const float* p = a.part + piece_at(pairs, width, dh, which.x);
  const float* ml = p + width * dh + n * 2;
  float top = -INFINITY;
  for (int i = lane; i < pieces; i += 64) top = fmaxf(top, ml[i * step]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float base = top == -INFINITY ? 0.f : top;
  float l = 0.f;
  int none = 0;
  for (int i = lane; i < pieces; i += 64) {
    const float2 x = *reinterpret_cast<const float2*>(ml + i * step);
    none |= x.y < 0.f;
    l += x.y < 0.f ? 0.f : top == -INFINITY ? x.y : x.y * __builtin_amdgcn_exp2f(x.x - base);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    l += __shfl_xor(l, o, 64);
    none |= __shfl_xor(none, o, 64);
  }
  if (none && top == -INFINITY && l == 0.f) l = -1.f;

  const int quads = dh <= 16 ? 4 : dh <= 32 ? 8 : dh <= 64 ? 16 : dh <= 128 ? 32 : 64;
  const int d = (lane & (quads - 1)) * 4, first = lane / quads + (WAVES == 4 ? wave * (64 / quads) : 0), stride = 64 / quads * WAVES;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (d < dh) {
#pragma unroll 4
    for (int i = first; i < pieces; i += stride)
      o += *reinterpret_cast<const f32x4*>(p + i * step + n * dh + d) * __builtin_amdgcn_exp2f(ml[i * step] - base);
  }
  for (int q = quads; q < 64; q <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], q, 64);
  if constexpr (WAVES == 4) {
    sh[wave][lane] = o;
    __syncthreads();
    if (wave) return;
    o = sh[0][lane] + sh[1][lane] + sh[2][lane] + sh[3][lane];
  }
  if (lane >= quads || d >= dh) return;
  if (a.lse && d == 0) a.lse[col.row * a.H + col.head] = log_sum(top, l);
  put4((T*)a.o + col.row * a.ldo + col.head * dh + d, o * over(top, l), a.vec);
}

// The kernel, the columns of a block, and the pieces that axes are cut into.
struct Shape { bool prompt; int nc, waves, width, tiles, target; };
Shape shape_of(int B, int T, int H, int Hkv, int dh, int64_t tokens) {
  Shape s;
  const int64_t columns = (int64_t)T * (H / Hkv);
  // More than 32 columns go through LDS: bf16, 16 sequences of 4000, 64 columns as four tiles of 16 or as half of one of 128: heads of 64 60 and 42 us, of 128 (as two by
  // two) 52 and 36; 32 columns: 30 and 41, 34 and 36.
  s.prompt = columns > 32;
  s.nc = !s.prompt && columns > 16 && dh <= 128 ? 2 : 1;      // more registers than two tiles of wider heads take there are not
  s.width = s.prompt ? 128 : 16 * s.nc;
  s.tiles = (int)((columns + s.width - 1) / s.width);
  const int64_t pairs = (int64_t)B * Hkv * s.tiles, longest = (tokens + 63) / 64;
  s.waves = kWaves;
  // Two blocks a compute unit: 2 contexts of 131071, 4 heads of 64, 36 us with 512 pieces, 40 with 1024 and 55 with 4096; 192 ragged ones the same to 5 %.
  s.target = 512;
  // Few short axes: eight waves side by side and no second launch (one context of 1000, 12 heads of 64: 7.3 us; in pieces 9.9 and 6.0 for joining them).
  if (!s.prompt && s.nc == 1 && dh <= 128 && longest <= 32 && pairs <= 256) {
    s.waves = 8;
    s.target = 0;
  }
  // nothing to cut: short axes, or more of them than blocks are wanted; sums are of 32 bits
  if (longest <= 2 * kWaves || pairs >= (s.prompt ? s.target : 4 * s.target) || pairs * longest >= (int64_t)1 << 31) s.target = 0;
  else if (pairs * ((longest + kWaves - 1) / kWaves) < s.target) s.target = (int)(pairs * ((longest + kWaves - 1) / kWaves));
  return s;
}

}  // namespace

bool cache_ok(const CacheView& c, int page);
bool cache_operands_ok(const CacheView& c);

bool cache_attn_ok(int B, int T, int H, int Hkv, int dh, int page, int max_pages) {
  CacheView v{};
  v.B = B; v.T = T; v.Hkv = Hkv; v.dh = dh; v.max_pages = max_pages; v.n_pages = 1; v.rows = 0x7fffffff;
  return cache_ok(v, page) && H >= Hkv && H % Hkv == 0 && H <= 1 << 16 && (int64_t)T * (H / Hkv) < (int64_t)1 << 30;
}
size_t cache_attn_scratch(int B, int T, int H, int Hkv, int dh, int page, int max_pages) {
  if (!cache_attn_ok(B, T, H, Hkv, dh, page, max_pages)) return 0;
  const Shape s = shape_of(B, T, H, Hkv, dh, (int64_t)max_pages * page);
  const int64_t pairs = (int64_t)B * Hkv * s.tiles;
  return s.target ? (size_t)((pairs * 2 + 15) & ~(int64_t)15) + (size_t)(pairs + s.target) * s.width * (dh + 2) : 0;
}

hipError_t op_cache_attn(const OpCtx& c, const CacheView& view, const void* q, int64_t ldq, void* o, int64_t ldo, float* lse, int H, int causal) {
  const int page = 1 << view.shift, dh = view.dh;
  if (!cache_attn_ok(view.B, view.T, H, view.Hkv, dh, page, view.max_pages)) return hipErrorInvalidValue;
  const int64_t width = (int64_t)H * dh, widest = (int64_t)1 << 32;
  if (ldq < width || ldo < width || ldq > widest || ldo > widest) return hipErrorInvalidValue;
  if (view.B == 0 || view.rows == 0) return hipSuccess;
  if (!q || !o || !cache_operands_ok(view)) return hipErrorInvalidValue;
  const Shape s = shape_of(view.B, view.T, H, view.Hkv, dh, (int64_t)view.max_pages * page);
  const size_t need = cache_attn_scratch(view.B, view.T, H, view.Hkv, dh, page, view.max_pages);
  if (need && (!c.partial || c.partial_elems < need || ((uintptr_t)c.partial & 15))) return hipErrorInvalidValue;
  const int G = H / view.Hkv;
  AttnArgs a{q, o, lse, c.partial, ldq, ldo, H, G, causal != 0, s.tiles, (unsigned)((((uint64_t)1 << 32) + G - 1) / G), s.target,
             ldq % 8 == 0 && ldo % 8 == 0 && (((uintptr_t)q | (uintptr_t)o) & 15) == 0, kLog2e / sqrtf((float)dh)};
  const int64_t pairs = (int64_t)view.B * view.Hkv * s.tiles;
  auto grid = [](int64_t blocks) {
    constexpr int64_t most = 1 << 21;            // a launch has less than 2^32 threads along x
    return dim3((unsigned)(blocks < most ? blocks : most), (unsigned)((blocks + most - 1) / most));
  };
  if (pairs > (int64_t)1 << 32 || (int64_t)view.B * view.Hkv > 1 << 30) return hipErrorInvalidValue;
  // with few columns a block joins one of them (there are many pieces), with many four
  auto join = [&](auto t) {
    typedef decltype(t) T;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !s.target) return e;
    const int most = view.T * G < s.width ? view.T * G : s.width;       // columns of a tile
    if (s.prompt) k_cache_join<T, 1><<<grid(pairs * (s.width / 4)), 256, 0, c.stream>>>(view, a, s.width, s.width / 4);
    else k_cache_join<T, 4><<<grid(pairs * most), 256, 0, c.stream>>>(view, a, s.width, most);
    return hipGetLastError();
  };
  auto go = [&](auto t, auto nd, auto nc) {
    typedef decltype(t) T;
    constexpr int ND = decltype(nd)::value, NC = decltype(nc)::value;
    if constexpr (NC == 1 && ND <= 2) {
      if (s.waves == 8) {
        if (page >= 64) k_cache_attn<T, ND, NC, 8, true><<<grid(pairs), 512, 0, c.stream>>>(view, a);
        else k_cache_attn<T, ND, NC, 8, false><<<grid(pairs), 512, 0, c.stream>>>(view, a);
        return join(t);
      }
    }
    if (page >= 64) k_cache_attn<T, ND, NC, kWaves, true><<<grid(pairs + s.target), 64 * kWaves, 0, c.stream>>>(view, a);
    else k_cache_attn<T, ND, NC, kWaves, false><<<grid(pairs + s.target), 64 * kWaves, 0, c.stream>>>(view, a);
    return join(t);
  };
  auto many = [&](auto t, auto nb) {
    typedef decltype(t) T;
    k_cache_prompt<T, decltype(nb)::value><<<grid(pairs + s.target), 256, 0, c.stream>>>(view, a);
    return join(t);
  };
  auto by_columns = [&](auto t, auto nd) {
    if constexpr (decltype(nd)::value <= 2) if (s.nc == 2) return go(t, nd, std::integral_constant<int, 2>());
    return go(t, nd, std::integral_constant<int, 1>());
  };
  auto by_head = [&](auto t) {
    if (s.prompt) {
      if (dh <= 32) return many(t, std::integral_constant<int, 1>());
      if (dh <= 64) return many(t, std::integral_constant<int, 2>());
      if (dh <= 96) return many(t, std::integral_constant<int, 3>());
      if (dh <= 128) return many(t, std::integral_constant<int, 4>());
      if (dh <= 192) return many(t, std::integral_constant<int, 6>());
      return many(t, std::integral_constant<int, 8>());
    }
    if (dh <= 64) return by_columns(t, std::integral_constant<int, 1>());
    if (dh <= 128) return by_columns(t, std::integral_constant<int, 2>());
    if (dh <= 192) return by_columns(t, std::integral_constant<int, 3>());
    return by_columns(t, std::integral_constant<int, 4>());
  };
  return c.dt == BF16 ? by_head(bf16_t()) : by_head(float());
}

}  // namespace lp
