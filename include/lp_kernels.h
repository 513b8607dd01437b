/*
 * lp_kernels.h -- kernel-level C ABI: the individual HIP ops the local-update step is made of,
 * callable on caller-owned DEVICE buffers.  Used by the per-kernel parity tests and by the bench's
 * per-kernel roofline measurements.  Every call enqueues on `stream` (a hipStream_t, NULL = default)
 * and returns 0 or a nonzero hipError_t code; nothing is allocated.  `dtype` is the compute dtype
 * (0 = fp32, 1 = bf16) of activations and matrix operands; gradients of parameters, statistics and
 * optimizer state are fp32.  `scratch_dev` is fp32 workspace for two-stage reductions
 * (scratch_elems floats; a call that needs more fails with hipErrorInvalidValue).
 */
#ifndef LP_KERNELS_H_
#define LP_KERNELS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* C[M,N] (+)= sum_k A(m,k) B(n,k) followed by the fused epilogue
 *   v (+= bias[n]); pre[m,n] = v; v = act(v); v *= act'(dact_src[m,n]); v += res[m,n].
 * A(m,k) = a_kc ? A[m*lda+k] : A[k*lda+m]; B(n,k) = b_kc ? B[n*ldb+k] : B[k*ldb+n]  (the forward, dgrad
 * and wgrad forms of a linear layer: paper appendix A, "MLP").  act / dact: 0 none, 1 ReLU, 2 GELU(tanh).
 * variant: 0 lets the library choose the kernel; 1 forces the fp32-arithmetic kernel; for bf16, 2 forces the
 * one-tile-per-block MFMA kernel, 3 / 4 the direct-to-LDS kernel with 256 x 128 tiles and the last partial wave
 * of tiles computed whole / cut along k, 5 / 6 the same with 256 x 256 tiles and 8 wavefronts, 7 / 8 with
 * 256 x 256 tiles and 4 wavefronts; 9 / 10 / 11 those three tile shapes in panel mode (outputs 2..8 tiles
 * wide: the tile columns of one tile row walk the same cut of the reduction together, so that the other
 * operand is fetched once per row); 20 / 21 / 22 the 8-wavefront 256 x 256 shape with 64-deep k-tiles (any
 * K from 64 on whose operand rows are whole 16-byte chunks), tail whole / cut along k / panel mode; an error if the shape does not qualify (K % 32 != 0 for 3 .. 11, no workspace for
 * a cut, an output too narrow or too wide or a reduction too short for panel mode).  splitk_ws_dev (may be NULL) is fp32 workspace of
 * splitk_ws_elems floats: with it, reductions over few output tiles are split along k and the partial sums
 * added in a fixed order (at most max(8 * M * N, 2^25) floats are used). */
int lpk_gemm(int dtype, const void* A, int64_t lda, int a_kc, const void* B, int64_t ldb, int b_kc, void* C,
             int64_t ldc, int c_f32, int M, int N, int K, const float* bias, int act, void* pre,
             const void* dact_src, int dact, int64_t ldd, const void* res, int64_t ldr, int accumulate, int variant,
             float* splitk_ws_dev, size_t splitk_ws_elems, void* stream);

/* n (2..16) independent bf16 products C_i[M_i, N_i] (+)= epilogue(sum_k A_i(m,k) B_i(n,k)) with one reduction length K
 * (a multiple of 32) and one pair of operand layouts, in ONE persistent launch: the weight gradients of the linear
 * maps of one layer, or the same-shaped products of independent blocks (section 3: blocks are trained in
 * parallel; section 6), each of which alone has too few output tiles for the chip.  Every array is a HOST array of
 * n entries holding DEVICE pointers, leading dimensions and sizes (M_i, N_i multiples of 8).  Outputs are fp32
 * (c_f32) or bf16; per problem an optional bias (fp32 [N_i]) and an optional residual (bf16 [M_i, N_i], leading
 * dimension ldc_i), `bias` and `res` may be NULL; act as in lpk_gemm, common to all.  The tiles of all products form
 * one sequence that is spread over the grid like a single product's; its last partial wave is cut along k through
 * splitk_ws_dev (at least 2^25 floats).  hipErrorInvalidValue, with nothing launched, if the set does not qualify. */
int lpk_gemm_grouped(int n, const void* const* A, const int64_t* lda, const void* const* B, const int64_t* ldb,
                     void* const* C, const int64_t* ldc, int c_f32, const int* M, const int* N, int K, int a_kc,
                     int b_kc, const float* const* bias, int act, const void* const* res, int accumulate,
                     float* splitk_ws_dev, size_t splitk_ws_elems, void* stream);

/* The same products on a chosen kernel (for tests and measurements): shape -1 is the persistent kernel of lpk_gemm_grouped, with
 * any K that its operands' 16-byte accesses allow (at least 128 if not a multiple of 32); shape 0 .. 5 is one tile per block, n
 * up to 4, tiles of 64 x 64, 128 x 64, 128 x 128 (two stages), 128 x 128 (four), 256 x 128 or 256 x 256, the reduction in
 * `pieces` equal runs of whole 64-deep k-tiles (the last may be shorter; hipErrorInvalidValue if there is no such cut) that a
 * second launch adds in order from splitk_ws_dev (pieces * sum M_i N_i floats). */
int lpk_gemm_grouped_tiles(int shape, int pieces, int n, const void* const* A, const int64_t* lda, const void* const* B,
                           const int64_t* ldb, void* const* C, const int64_t* ldc, int c_f32, const int* M, const int* N, int K,
                           int a_kc, int b_kc, const float* const* bias, int act, const void* const* res, int accumulate,
                           float* splitk_ws_dev, size_t splitk_ws_elems, void* stream);

/* The weight gradients of one layer with its bias gradients, as a step takes them: dw_i[M_i, N_i] (+)= dy_i^T x_i (bf16 dy_i
 * [rows, M_i] and x_i [rows, N_i], fp32 out) and db_i[M_i] (+)= the column sums of dy_i (a null db_i: none), and in the same
 * launch out[j] (+)= sum_b part[b, j], b < nblk, j < len (partial sums that an earlier kernel has left; len 0: none); no output
 * overlaps another.  n 2 to 5,
 * arrays as in lpk_gemm_grouped; shape and pieces as in lpk_gemm_grouped_tiles, or shape -1: chosen by the library.  Where a width
 * is no multiple of 8 or a matrix is not on a 16-byte boundary the sums go ahead of the products, through the workspace (at least
 * (rows + 127) / 128 floats for every column of the widest dy_i); a forced shape refuses such matrices. */
int lpk_weight_grads(int shape, int pieces, int n, const void* const* dy, const int64_t* ld_dy, const void* const* x,
                     const int64_t* ld_x, float* const* dw, float* const* db, const int* M, const int* N, int rows,
                     int accumulate, const float* part, float* out, int nblk, int len, float* splitk_ws_dev,
                     size_t splitk_ws_elems, void* stream);

/* Causal (or full) multi-head attention of a decoder layer (appendix B.2).  qkv [B*S, 3*H*dh]
 * (q | k | v), o [B*S, H*dh], lse [B,H,S] = log-sum-exp of the scaled scores, delta [B,H,S] scratch.  plain != 0: the
 * row-by-row kernels. */
int lpk_attention_fwd(int dtype, const void* qkv, void* o, float* lse, int B, int S, int H, int dh, int causal,
                      int plain, void* stream);
int lpk_attention_bwd(int dtype, const void* qkv, const void* o, const float* lse, const void* dout, void* dqkv,
                      float* delta, int B, int S, int H, int dh, int causal, int plain, void* stream);
/* The same in bf16 on the matrix kernels, heads of 16, 32 or 64, with a block's chain of tiles in 1, 2 or 4 parts (for tests and
 * measurements); qkv, o, dout and dqkv on 16-byte boundaries.  Anything else is refused. */
int lpk_attention_fwd_parts(const void* qkv, void* o, float* lse, int B, int S, int H, int dh, int causal, int parts, void* stream);
int lpk_attention_bwd_parts(const void* qkv, const void* o, const float* lse, const void* dout, void* dqkv, float* delta, int B,
                            int S, int H, int dh, int causal, int parts, void* stream);
/* The parts that the library chooses (needs no device); 0 for heads that are not 16, 32 or 64 wide. */
int lpk_attention_parts(int B, int S, int H, int dh, int backward);

/* Linear attention with a decay for each head: with l = exp(log_decay[h]) and a state S [dh, dh] per sequence and head,
 *   S_t = l S_{t-1} + k_t v_t^T,   o_t = dh^-1/2 q_t S_t      (S_{-1} = s0, zeros if null).
 * qkv [B*S, 3*H*dh] and o [B*S, H*dh] as in lpk_attention_fwd; log_decay fp32 [H] on the device, 0 or less (a constant: it has no
 * gradient); states fp32 [B, H, dh, dh].  dh up to 128, B*H up to 524280, 3*H*dh below 2^24, S up to 2^30.
 * lens (int32 [B] on the device, may be null: all S) are the sequences' lengths, taken as 0 .. S: positions behind them are neither
 * read nor part of a state, their rows of o and dqkv become zeros.  s_out (may be null, may be s0) receives the state after the last
 * position.  An infinity or a NaN at a position reaches, as an infinity or a NaN, the outputs of that one and later ones only (the
 * gradients: dout's those of that position and earlier ones in dk and dv, of that one alone in dq).
 * The backward call takes the same qkv, lens and s0 with the gradients dout of o and ds_out of s_out (may be null: zeros) and
 * writes dqkv and, where it is not null, the gradient ds0 of s0.  But for s_out no output overlaps an input.
 * scratch_dev: lpk_linear_attention_scratch floats (needs no device; may be 0); contents undefined on return, so that calls which
 * share it are ordered. */
int lpk_linear_attention_fwd(int dtype, const void* qkv, const float* log_decay, const int32_t* lens, const float* s0, void* o,
                             float* s_out, int B, int S, int H, int dh, float* scratch_dev, size_t scratch_elems, void* stream);
int lpk_linear_attention_bwd(int dtype, const void* qkv, const float* log_decay, const int32_t* lens, const float* s0,
                             const void* dout, const float* ds_out, void* dqkv, float* ds0, int B, int S, int H, int dh,
                             float* scratch_dev, size_t scratch_elems, void* stream);
size_t lpk_linear_attention_scratch(int B, int S, int H, int dh, int backward);
/* One position more: qkv [B, 3*H*dh], o [B, H*dh], the states are updated in place.  The same as a forward call of S = 1; B*H below
 * 2^24. */
int lpk_linear_attention_step(int dtype, const void* qkv, const float* log_decay, float* state, void* o, int B, int H, int dh,
                              void* stream);

/* Dropout of n elements: y = drop(x) (+ res, may be null); y may be x or res.  An element is kept with probability 1 - p (p in
 * [0, 1], rounded to a multiple of 2^-16) and then divided by the rounded 1 - p.  Which are kept is a function of the element's index,
 * `site` (a number the caller gives every place of a model that drops) and rng_dev, two 64-bit numbers on the device: a
 * seed and a step, which the caller changes from step to step, also under a replayed graph.  No mask is stored: the gradient is the
 * same call on dy, without res.  The generator is Philox4x32-10, counter (index / 8, site, step), key seed; element 8 i + j has the
 * j-th 16-bit half of the four words, lower half first, and is dropped where that is less than 65536 p.  n up to 2^35. */
int lpk_dropout(int dtype, const void* x, const void* res, void* y, size_t n, float p, const uint64_t* rng_dev, uint32_t site,
                void* stream);

/* Root-mean-square norm over the last dimension (d up to 16384, up to 2^30 rows, rows * d up to 2^35) behind a residual branch's
 * dropout and addition:
 *   r = drop(x) (+ res),  rstd = (mean(r^2) + eps)^-1/2,  y = r rstd g.
 * res may be null; p, rng_dev and site as in lpk_dropout (index: row * d + column; p 0: nothing is dropped).  r (may be null, may be x
 * or res) and y (compute dtype, may be null) are outputs, rstd (fp32 [rows], may be null) is kept for the backward call; the norm is
 * taken of the sum before its rounding to the compute dtype.  y8 (may be null) receives y in 8 bits, e4m3, with one scale for
 * a row: y8 = y / y8_scale[row], the fp32 quotient, y8_scale = max |y| / 448 (1 for a row of zeros, otherwise 2^-126 at least).  At least one
 * of y and y8 is wanted.
 * Backward, of r as stored (x itself where there was neither res nor dropout): dres = gradient of r (+ add, the stream's own, may be
 * null), dx = that of x where p > 0 (null where it is not wanted: with p 0 it is dres), dg (+)= sum over rows (may be null).  dres and
 * dx may be dy, r or add.  scratch_dev: lpk_rmsnorm_scratch floats where dg is wanted (needs no device). */
int lpk_rmsnorm_fwd(int dtype, const void* x, const void* res, const float* g, void* r, void* y, void* y8, float* y8_scale,
                    float* rstd, int rows, int d, float eps, float p, const uint64_t* rng_dev, uint32_t site, void* stream);
int lpk_rmsnorm_bwd(int dtype, const void* dy, const void* r, const float* rstd, const float* g, const void* add, void* dres,
                    void* dx, float* dg, int rows, int d, int accumulate, float p, const uint64_t* rng_dev, uint32_t site,
                    float* scratch_dev, size_t scratch_elems, void* stream);
size_t lpk_rmsnorm_scratch(int rows, int d);

/* Rotary positions of the heads of a matrix's rows, for training (on the q and k columns of qkv in front of lpk_attention_fwd; the
 * backward call on those of dqkv) and for single tokens: with t = pos freq[i], of the pair (a, b) = columns (i, i + rot/2) of a head, or (2 i, 2 i + 1)
 * if `interleaved`, i < rot/2,
 *   y = scale (a cos t - b sin t, a sin t + b cos t);      backward: the transpose, the gradient of x from that of y.
 * x and y: `rows` rows of heads * dh columns (dh up to 512) with leading dimensions ldx and ldy; columns rot .. dh - 1 of a head (rot even) are copied;
 * y may be x (ldy = ldx), otherwise they do not overlap.  pos int32 [rows] on the device, any number (null: row % S); freq fp64 [rot/2] on
 * the device, radians a position: the product is taken in 64 bits, its whole turns are taken off, and sine and cosine are those of the rest as a 32-bit number of half turns.
 * rows up to 2^30, heads * dh up to 2^24, leading dimensions to 2^32.
 * lpk_rotary_frequencies writes such a table to host memory: base^(-2 i / rot), stretched for contexts longer than those trained on: divided by
 * `factor` where a pair turns at most `low` times within `context` positions, kept where it turns `high` times or more, in between blended in the number of
 * turns (factor 1: kept; low = high = infinity: all divided). */
int lpk_rotary(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, const int32_t* pos, const double* freq, int rows, int S, int heads,
               int dh, int rot, int interleaved, float scale, int backward, void* stream);
int lpk_rotary_frequencies(double* freq, int rot, double base, double factor, double low, double high, double context);

/* A paged cache of keys and values in 8 bits (e4m3) with a scale for each page and head, written by lpk_cache_append, read back
 * by lpk_cache_read and attended over by lpk_cache_attention.
 * A page holds `page` tokens (16, 32, 64, 128 or 256): kpages [n_pages, Hkv, page, dh], vpages [n_pages, Hkv, dh, page] (16-byte aligned), kscale and
 * vscale fp32 [n_pages, Hkv]; dh a multiple of 16 up to 256.  table int32 [B, max_pages] (max_pages * page up to 2^30): page number of
 * each `page` positions of a sequence; a number outside 0 .. n_pages - 1 means that there is no page: nothing is written there, zeros are read, and
 * attention sees no token there.  lens int32 [B]: the sequences' lengths, those of the call's new rows included, taken as 0 .. max_pages * page.
 * The new rows of sequence b are rows starts[b] .. starts[b + 1] - 1 (starts int32 [B + 1]; null: rows b T .. b T + T - 1), and n of them stand at its
 * positions lens[b] - n .. lens[b] - 1.  T: at most so many rows a sequence; one whose rows are more, not in order or not within the `rows` rows of
 * the matrix counts as one of none.  Rows of no sequence are neither read nor written.  All of these are on the device, B up to 2^20.
 *
 * Append quantises rows of k and v (compute dtype, Hkv * dh columns, leading dimensions ldk and ldv): per page and head s' = max(s, need), need the least power
 * of two (2^-126 at least) with |x| / need <= 448 for all new finite x, s the scale of the page's earlier tokens (positions before the new rows'; none: s' =
 * need); code = e4m3(x / s'), rounded to nearest even, and where s' > s the earlier codes become e4m3(code s / s').  A NaN or an infinity is held as
 * a NaN and has no part in the scale.  The pages that one call writes are all different.
 * Read writes code * s of the same rows to k and v (zeros for positions before the first).
 *
 * Attention: o = softmax(q k^T dh^-1/2) v for the rows of q [rows, H * dh] (leading dimension ldq; H a multiple of Hkv, heads h G .. h G + G - 1 read
 * head h of the cache, G = H / Hkv), over the positions up to the row's own if `causal`, otherwise all of the sequence's.  o [rows, H * dh]; lse fp32 [rows, H]
 * (may be null) = log-sum-exp of the scaled scores.  A row that sees no token becomes zeros, its lse minus infinity.  What a row does not see does not
 * change it, a NaN there included.  Scores, largest scores and sums are of 32 bits.  Weights stand before the values with 24 bits if dtype is fp32; in bf16 they are
 * rounded, to 2^-16 of a weight where T H / Hkv is 32 or less, otherwise to 2^-12 of it or 2^-24 of the row's largest, whichever is more.  Numbers of q, and of pages with their
 * scale, that are neither zero nor within 2^-80 .. 2^80 may be beyond what 32 bits hold in between.  Scales are positive, as append leaves them.  q and o do not overlap.
 * scratch_dev: lpk_cache_attention_scratch floats (needs no device; may be 0), 16-byte aligned; contents
 * undefined on return, so that calls which share it are ordered. */
int lpk_cache_append(int dtype, const void* k, int64_t ldk, const void* v, int64_t ldv, int rows, const int32_t* starts, const int32_t* lens,
                     const int32_t* table, void* kpages, void* vpages, float* kscale, float* vscale, int B, int T, int Hkv, int dh, int page,
                     int max_pages, int n_pages, void* stream);
int lpk_cache_read(int dtype, void* k, int64_t ldk, void* v, int64_t ldv, int rows, const int32_t* starts, const int32_t* lens,
                   const int32_t* table, const void* kpages, const void* vpages, const float* kscale, const float* vscale, int B, int T, int Hkv,
                   int dh, int page, int max_pages, int n_pages, void* stream);
int lpk_cache_attention(int dtype, const void* q, int64_t ldq, int rows, const int32_t* starts, const int32_t* lens, const int32_t* table,
                        const void* kpages, const void* vpages, const float* kscale, const float* vscale, void* o, int64_t ldo, float* lse, int B,
                        int T, int H, int Hkv, int dh, int page, int max_pages, int n_pages, int causal, float* scratch_dev, size_t scratch_elems,
                        void* stream);
size_t lpk_cache_attention_scratch(int B, int T, int H, int Hkv, int dh, int page, int max_pages);

/* LayerNorm over the last dimension (eps 1e-5, biased variance); backward adds `add` to dx if given. */
int lpk_layernorm_fwd(int dtype, const void* x, const float* g, const float* b, void* y, float* mean, float* rstd,
                      int rows, int d, void* stream);
int lpk_layernorm_bwd(int dtype, const void* dy, const void* x, const float* mean, const float* rstd,
                      const float* g, const void* add, void* dx, float* dg, float* db, int rows, int d,
                      int accumulate, float* scratch_dev, size_t scratch_elems, void* stream);

/* lpk_layernorm_bwd for callers that cannot allocate device memory or bring a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments and results as
 * lpk_layernorm_bwd without the scratch pair: the partial sums of dg and db go through an array built into
 * the library (LPK_STATIC_SCRATCH_FLOATS floats = 8 MiB, held on every GPU the library runs on until the
 * process ends).  Nothing is allocated or freed.  hipErrorInvalidValue (and a line on stderr) if
 * ((rows + 7) / 8) * d * 2 exceeds LPK_STATIC_SCRATCH_FLOATS; 8192 rows of width 1024 just fit.  All calls on
 * one GPU share the array, whatever their stream: calls that overlap in time on one GPU race, so order them on
 * one stream or with events.  The array keeps the last call's partial sums; a call reads only what it wrote. */
#define LPK_STATIC_SCRATCH_FLOATS (1u << 21)
int lpk_layernorm_bwd_static(int dtype, const void* dy, const void* x, const float* mean, const float* rstd,
                             const float* g, const void* add, void* dx, float* dg, float* db, int rows, int d,
                             int accumulate, void* stream);

/* Row-wise softmax cross-entropy (the auxiliary objective, section 3): loss_rows[r] = lse(z_r) - z[r,y_r];
 * with write_grad, z is overwritten by (softmax(z_r) - onehot(y_r)) * inv_rows. */
int lpk_softmax_ce(int dtype, void* z, int64_t ld, const int32_t* y, float* loss_rows, int rows, int n,
                   int write_grad, float inv_rows, void* stream);

/* Fused optimizer update over a flat range (kind 0 SGD, 1 SGD-momentum, 2 Adam; appendix B lists the
 * optimizers); n must be a multiple of 4; p_bf16 (may be NULL) receives the bf16 working copy. */
int lpk_optimizer(int kind, float lr, float momentum, float beta1, float beta2, float eps, float weight_decay,
                  int t, float grad_scale, float* p, const float* g, float* m, float* v, void* p_bf16, size_t n,
                  void* stream);

/* Plain device-to-device copy of `bytes` bytes (a multiple of 16; both pointers 16-byte aligned), one
 * 16-byte load and store per lane.  Not part of the method: it is the kernel of known traffic against
 * which the HBM counters (FETCH_SIZE, WRITE_SIZE) are scaled when a kernel's traffic is measured. */
int lpk_copy(const void* src_dev, void* dst_dev, size_t bytes, void* stream);

/* dst[C][R] = transpose of src[R][C], bf16 (R and C multiples of 8, both pointers 16-byte aligned).  Keeps the
 * [in][out] copy of a vocabulary head's weight [out][in] with which the head's input-gradient GEMM
 * (section 3: the backward pass inside a block) has the reduction index fastest in both operands. */
int lpk_transpose_bf16(const void* src_dev, void* dst_dev, int R, int C, void* stream);

/* Embedding-table gradient: demb[v,:] (+)= sum of dh[t,:] over positions with ids[t] == v, in order of t
 * (ids outside [0, V) count as the nearest valid id, as in the forward lookup).  scratch_dev (may be NULL)
 * is device scratch of scratch_elems 4-byte words.  With at least 2 T of them (T up to 65536, V T below 2^31 - 1, d a
 * multiple of 8 up to 8192, dh and demb on 16-byte boundaries) the positions are sorted there first; otherwise, with
 * at least V, every id's positions are counted there and the rows that do not occur are skipped.  Same bits each way. */
int lpk_embed_bwd(int dtype, const int32_t* ids, const void* dh, float* demb, int T, int V, int d, int accumulate,
                  float* scratch_dev, size_t scratch_elems, void* stream);

/* NHWC convolution with [O,R,S,C] filters as implicit GEMM (appendix B.3), forward / data gradient /
 * filter gradient (fp32). */
int lpk_conv_fwd(int dtype, const void* x, const void* w, void* out, int N, int H, int W, int C, int O, int R,
                 int stride, int pad, void* stream);
int lpk_conv_bwd_data(int dtype, const void* dout, const void* w, void* dx, int N, int H, int W, int C, int O, int R,
                      int stride, int pad, void* stream);
int lpk_conv_bwd_weight(int dtype, const void* dout, const void* x, float* dw, int N, int H, int W, int C, int O,
                        int R, int stride, int pad, int accumulate, void* stream);
/* The same filter gradient with fp32 workspace (device memory, splitk_ws_elems floats, contents undefined on
 * return): with it the reduction over the N*P*Q output pixels is cut into pieces whose partial sums are added in a
 * fixed order, which is how the step computes it; a 3-channel stem with 64 output channels then takes one image per
 * block (needs N*O*R*R*C floats).  Without enough workspace the call computes the gradient uncut. */
int lpk_conv_bwd_weight_ws(int dtype, const void* dout, const void* x, float* dw, int N, int H, int W, int C, int O,
                           int R, int stride, int pad, int accumulate, float* splitk_ws_dev, size_t splitk_ws_elems,
                           void* stream);

/* The filter gradients of a stage's convolutions, as its backward pass takes them: the pieces of all wait in the workspace and
 * are added in one launch (in more where they do not fit together), with the bits of lpk_conv_bwd_weight_ws.  bf16; dims: n rows
 * of N, H, W, C, O, R, stride, pad; no dw overlaps another. */
int lpk_conv_weight_grads(int n, const void* const* dout, const void* const* x, float* const* dw, const int* dims, int accumulate,
                          float* splitk_ws_dev, size_t splitk_ws_elems, void* stream);

/* A bf16 convolution on chosen tiles of the matrix-core kernel (for tests and measurements).  dir 0: out = conv(a = x, b = w);
 * 1: out = data gradient of (a = dout, b = w), plus `add` if given; 2: out (fp32) = filter gradient of (a = dout, b = x), added to
 * what is there if `accumulate`.  shape: rows x columns 0: 64 x 64, 1: 128 x 64, 2: 128 x 128 (two stages), 3: 128 x 128 (four),
 * 4: 256 x 128, 6: 64 x 128, 7: 256 x 64, 8: 128 x 32 (outputs of at most 32 columns); pieces as in lpk_gemm_grouped_tiles.
 * dir 0 with stats_dev: where the output is whole tiles in one piece, the normalisation's sums per tile and column
 * ([3][tiles][O] floats: sum (z - p), sum (z - p)^2 and p, the tile's first row) are left there and *stats_rows is a
 * tile's rows, otherwise 0.  hipErrorInvalidValue if the kernel does not take the convolution that way. */
int lpk_conv_tile(int dir, const void* a, const void* b, void* out, const void* add, int accumulate, int N, int H, int W, int C,
                  int O, int R, int stride, int pad, int shape, int pieces, float* stats_dev, size_t stats_elems, int* stats_rows,
                  float* splitk_ws_dev, size_t splitk_ws_elems, void* stream);
/* The shape and number of pieces the library takes for such a convolution by itself, with splitk_ws_elems floats of workspace
 * (host only). */
int lpk_conv_plan(int dir, int N, int H, int W, int C, int O, int R, int stride, int pad, size_t splitk_ws_elems, int* shape,
                  int* pieces);

/* One convolution + normalisation unit of a ResNet stage, forward (appendix B.3): z = conv(x, w) as lpk_conv_fwd,
 * then y = [relu](bn(z) (+ res)) as lpk_batchnorm_fwd, with z, y, mean, rstd all written.  Where the convolution's
 * output is whole tiles of the matrix-core kernel and O / 8 divides 256, the convolution itself leaves the per-channel sums of its rounded
 * outputs in scratch_dev and the normalisation does not read z for its statistics; otherwise the two run as the
 * separate calls would.  scratch_dev: at least max(3 * (N*P*Q/32 + O), (2*1024 + 2) * O) floats. */
int lpk_conv_bn_fwd(int dtype, const void* x, const void* w, void* z, const float* g, const float* b, const void* res,
                    void* y, float* mean, float* rstd, int N, int H, int W, int C, int O, int R, int stride, int pad,
                    int relu, float* scratch_dev, size_t scratch_elems, void* stream);

/* BatchNorm with batch statistics over rows = N*H*W, fused residual add and ReLU.  scratch_dev: S * C floats forward
 * (2 * S * C where C / 8 is whole and divides 256, bf16), (2 * S + 2) * C backward, S = ceil(rows / 1024); in the bf16
 * case just named S = ceil(rows / max(ceil(rows / 1024), 8 * (256 / (C / 8)))).  (2*1024 + 2) * C floats always do
 * for at most 2^20 rows; more than needed lets more of the chip work. */
int lpk_batchnorm_fwd(int dtype, const void* z, const float* g, const float* b, const void* res, void* y,
                      float* mean, float* rstd, int rows, int C, int relu, float* scratch_dev, size_t scratch_elems,
                      void* stream);
int lpk_batchnorm_bwd(int dtype, const void* dy, const void* y, const void* z, const float* mean, const float* rstd,
                      const float* g, void* dz, void* dres, float* dg, float* db, int rows, int C, int relu,
                      int accumulate, float* scratch_dev, size_t scratch_elems, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LP_KERNELS_H_ */
