/*
 * fno.h -- C ABI of libfno: the 4D (x,y,z,t) Fourier-neural-operator spectral convolution
 * and FNO block, forward and adjoint, as hand-written HIP kernels for gfx950 (MI355X).
 *
 * What the calls compute follows the paper's statement of the layer
 * (Grady et al., "Model-Parallel Fourier Neural Operators ...", arXiv 2204.01205):
 *   - eq. (2), Sec. 1.4 and the block update of Sec. 2.4:  nu_{k+1} = sigma(W nu_k + K(phi) nu_k)
 *   - eq. (3), Sec. 1.4:  K(phi) nu = F^{-1}( R_phi . F nu ), R_phi = low-pass restriction to a
 *     user-chosen number of modes per dimension plus a learned complex weight per kept mode
 *   - eq. (4), Sec. 2.2:  y = W x + b contracted along the channel dimension
 *   - eq. (7), Sec. 2.3 and the Fig. 5 caption: F^T is the adjoint (inverse) transform, used
 *     for the backward pass
 *
 * Conventions (all calls):
 *   - Tensors are dense, row-major, layout NCXYZT (Sec. 3.1): x[b][c][nx][ny][nz][nt], t contiguous.
 *   - Every data pointer is a DEVICE pointer owned by the caller.  The library never allocates,
 *     frees or synchronises; scratch comes from the caller's workspace `ws` (device memory,
 *     256-byte aligned, at least fno_workspace_bytes() bytes).  Descriptors are host structs
 *     read during the call only.
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*, NULL = default stream) and
 *     the call returns without waiting.
 *   - Complex tensors are interleaved (re, im) float pairs.  Grid-sized and mode-sized tensors
 *     must be 16-byte aligned (FNO_EINVAL otherwise).
 *   - Return value: FNO_OK (0) or a negative FNO_E* code.  On an argument error nothing is
 *     launched and no output byte is written.
 *   - Two calls that share a workspace or an output must be ordered by the caller.
 *
 * Kept modes.  With modes = (mx, my, mz, mt) the spatial axes keep the signed frequencies
 *   rule 0:  0..m-1, -m..-1      (L = 2m)        rule 1:  0..m, -m..-1     (L = 2m+1)
 * in exactly this order along the weight tensor's mode axes, and the real-transform axis t
 * keeps 0..mt-1.  Requirements: 1 <= L <= N on x,y,z and 1 <= mt <= Nt/2 + 1.
 *
 * Forward transform is unnormalised; the inverse carries 1/(Nx Ny Nz Nt) and is a complex
 * inverse over x,y,z followed by a complex-to-real step over t, i.e.
 *   y[n] = (1/N) Re sum_k c_kt Yhat[k] exp(+i theta(k,n)),   c_kt = 1 for kt = 0 and kt = Nt/2, else 2.
 */
#ifndef FNO_H_
#define FNO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  FNO_OK = 0,
  FNO_EINVAL = -1,        /* null required pointer, non-positive size, too many modes, bad flag  */
  FNO_EUNSUPPORTED = -2,  /* valid request outside what the kernels cover (see fno_status_string) */
  FNO_ENOSPC = -3,        /* workspace too small or misaligned                                    */
  FNO_EHIP = -4           /* the HIP runtime refused a launch or copy                             */
};

/* GELU is z Phi(z) with Phi the normal distribution function (the erf form, not the tanh one).  The
 * forward epilogues evaluate the tail of Phi by a polynomial for its logarithm (z Phi(z) within 3e-7), the
 * backward kernels of a block and of the projection by such a polynomial or by the density times one; projections
 * whose weights or hidden width are off the matrix-core kernels use the float erff / expf routines.  In every case the
 * activation and its slope are within 1e-6 (absolute) of the float64 definition for every finite argument, far
 * inside the 1e-5 relative L2 the library is tested to; minus infinity gives NaN.  Where products run as sums of
 * 16-bit parts (the projection, its adjoint, the forward transform), finite values from 3.39e38 on count as
 * infinite, an infinite one gives NaN in what depends on it, and values below 1e-33 keep 8 to 24 bits. */
enum { FNO_ACT_IDENTITY = 0, FNO_ACT_GELU = 1 };

enum {
  FNO_OP_SPECTRAL_CONV_FWD = 0,
  FNO_OP_SPECTRAL_CONV_BWD = 1,
  FNO_OP_BLOCK_FWD = 2,
  FNO_OP_BLOCK_BWD = 3
};

enum {
  FNO_FLAG_MSE_TARGET = 1,       /* block_bwd: `gout` holds a target field; the upstream gradient is that of
                                    the mean squared error, 2 (sigma(z) - target) / (B Cout N)            */
  FNO_FLAG_ACCUMULATE_GRADS = 2, /* block_bwd, spectral_conv_bwd: the parameter gradients (gR, gW, gb) are
                                    added to what the output buffers hold instead of overwriting them: the
                                    gradient of a broadcast weight is a sum (Sec. 2.1), and a step made of
                                    several calls (one per sample or per shard) continues that sum.  gx is
                                    always overwritten.                                                    */
  FNO_FLAG_TABLES_READY = 4      /* every call with a workspace: the twiddle tables for this descriptor are in
                                    `ws` already (written by fno_plan_tables on the same workspace, nothing
                                    else having written there since except the library's own calls with the
                                    same grid, modes and mode rule); the call then skips the four small
                                    kernels that rebuild them                                              */
};

typedef struct {
  int32_t batch;       /* B >= 1                                                      */
  int32_t c_in;        /* input channel width                                         */
  int32_t c_out;       /* output channel width (<= 32 for the block calls)            */
  int32_t grid[4];     /* Nx, Ny, Nz, Nt                                              */
  int32_t modes[4];    /* mx, my, mz: per-side count on x,y,z ; mt: count on t        */
  int32_t mode_rule;   /* 0 or 1, see above                                           */
  int32_t activation;  /* FNO_ACT_*; used by the block calls only                     */
  int32_t flags;       /* FNO_FLAG_* bits                                             */
} fno_desc;

/* Size in bytes of the workspace the given FNO_OP_* needs for this descriptor (host-only). */
int fno_workspace_bytes(const fno_desc* desc, int op, size_t* bytes);

/* Writes the twiddle tables of the transforms (Sec. 2.3: one truncated DFT per axis; they depend on
 * the grid, the kept modes and the mode rule only) into the workspace, on `stream`.  Optional: every
 * call rebuilds them itself unless its descriptor carries FNO_FLAG_TABLES_READY.  The table region
 * sits at the same place in the workspace of every FNO_OP_*, so one plan serves all four calls on
 * that workspace.  ws, ws_bytes as for the op given. */
int fno_plan_tables(const fno_desc* desc, int op, void* ws, size_t ws_bytes, void* stream);

/* Kept signed frequencies of axis 0..3 (x,y,z,t) in weight-tensor order (host-only).
 * out_k (host, nullable) receives *out_n values; out_n (host) receives the count. */
int fno_mode_indices(const fno_desc* desc, int axis, int32_t* out_k, int32_t* out_n);

/* What the bits of a result depend on.  A call repeated with the same descriptor, values and alignment gives the same
 * bits.  An entry of a batch may differ in its last bits from the same entry in a batch of another size: kernels are
 * chosen by sizes, the batch among them (the (z,t) stages by their number of columns; small layers take the x stages and
 * the mode mix in one launch, whose sums are in double, up to four entries, or to one where c_in != c_out, and their
 * adjoint as long as all entries together are small).  The spectrum that an adjoint works out again from x has the bits
 * that the forward call saves with the same descriptor.
 *
 * Spectral convolution, eq. (3):  y = K(phi) x.
 *   x         in   float  [B][Cin][Nx][Ny][Nz][Nt]
 *   R         in   cfloat [Cin][Cout][Lx][Ly][Lz][mt]
 *   y         out  float  [B][Cout][Nx][Ny][Nz][Nt]
 *   xhat_save out  cfloat [B][Cin][Lx][Ly][Lz][mt], nullable: the kept forward spectrum F x */
int fno_spectral_conv_fwd(const fno_desc* desc, const float* x, const float* R, float* y,
                          float* xhat_save, void* ws, size_t ws_bytes, void* stream);

/* Adjoint of the spectral convolution (eq. (7): the transposed transform chain).
 *   x          in  float, used only when xhat_saved is NULL (then F x is recomputed)
 *   xhat_saved in  cfloat [B][Cin][Lx][Ly][Lz][mt], nullable
 *   gy         in  float  [B][Cout][grid]     dL/dy
 *   gx         out float  [B][Cin][grid]      dL/dx, nullable
 *   gR         out cfloat [Cin][Cout][modes]  dL/dRe R + i dL/dIm R, nullable (overwritten, or added
 *                                             to with FNO_FLAG_ACCUMULATE_GRADS) */
int fno_spectral_conv_bwd(const fno_desc* desc, const float* x, const float* xhat_saved,
                          const float* R, const float* gy, float* gx, float* gR,
                          void* ws, size_t ws_bytes, void* stream);

/* One FNO block, eq. (2):  out = sigma(W x + b + K(phi) x), Cin == Cout.
 *   W  in float [Cout][Cin]     b  in float [Cout], nullable (= 0)
 *   out        out float [B][Cout][grid]
 *   z_save     out float [B][Cout][grid], nullable: the pre-activation, needed by fno_block_bwd
 *              (one of out and z_save may be x itself, the block in place; no other overlap)
 *   xhat_save  out cfloat, nullable, as above */
int fno_block_fwd(const fno_desc* desc, const float* x, const float* R, const float* W,
                  const float* b, float* out, float* z_save, float* xhat_save,
                  void* ws, size_t ws_bytes, void* stream);

/* Adjoint of the block.  z_saved is the pre-activation from fno_block_fwd; gout is dL/dout, or
 * with FNO_FLAG_MSE_TARGET the target field of a mean-squared-error loss.
 *   gx out float [B][Cin][grid], gR out cfloat [Cin][Cout][modes], gW out float [Cout][Cin],
 *   gb out float [Cout]; each nullable, each overwritten (gR, gW, gb added to instead with
 *   FNO_FLAG_ACCUMULATE_GRADS).  gW and gb are sums over all batch
 *   entries and grid points (the adjoint of broadcasting W and b, Sec. 2.1), reduced in a fixed
 *   order so repeated calls give identical bits. */
int fno_block_bwd(const fno_desc* desc, const float* x, const float* R, const float* W,
                  const float* z_saved, const float* xhat_saved, const float* gout,
                  float* gx, float* gR, float* gW, float* gb,
                  void* ws, size_t ws_bytes, void* stream);

/* Channel lift of Sec. 2.4 (eq. (11)):  y[b][o][p] = sum_i W[o][i] x[b][i][p] + bias[o] over
 * npoints contiguous points per channel.  bias nullable.  c_out <= 32. */
int fno_pointwise_linear(int32_t batch, int32_t c_in, int32_t c_out, int64_t npoints,
                         const float* x, const float* W, const float* bias, float* y, void* stream);

/* Input lifts of Sec. 2.4 (eqs. (8)-(9)), fused: the input a [B][c_in][nspace] has a time axis of
 * length one; a_1 = Wt a + bt along time (Wt, bt: nt values each), then the channel lift
 * nu = Wc a_1 + bc (Wc [c_out][c_in], bc [c_out]) gives out [B][c_out][nspace][nt], t contiguous.
 * All pointers are device pointers owned by the caller; bt and bc nullable; out 16-byte aligned
 * when nt is a multiple of 4; c_out <= 32.  Asynchronous on `stream`; nothing is launched on an
 * argument error. */
int fno_time_lift(int32_t batch, int32_t c_in, int32_t c_out, int64_t nspace, int32_t nt, const float* a,
                  const float* Wt, const float* bt, const float* Wc, const float* bc, float* out,
                  void* stream);

/* Adjoint of fno_time_lift (Sec. 2.4, eqs. (8)-(9); sums over broadcast axes, Sec. 2.1) with
 * respect to its parameters, for a cotangent g [B][c_out][nspace][nt] of its output:
 *   gbc[o] = sum g,  gWc[o][i] = sum g (Wt[t] a[b][i][s] + bt[t]),
 *   gWt[t] = sum g Wc[o][i] a[b][i][s],  gbt[t] = sum g Wc[o][i]
 * (each over every index not on the left).  The input a is data: its gradient is not formed.
 * Every output is nullable and overwritten; fixed summation order, the same bits on every run.
 * ws: device scratch of fno_time_lift_bwd_workspace_bytes(c_in, c_out, nt) bytes, 8-byte aligned,
 * owned by the caller.  c_in <= 8, batch <= 1024.  Asynchronous on `stream`; nothing is
 * launched on an argument error. */
int fno_time_lift_bwd_workspace_bytes(int32_t c_in, int32_t c_out, int32_t nt, size_t* bytes);
int fno_time_lift_bwd(int32_t batch, int32_t c_in, int32_t c_out, int64_t nspace, int32_t nt, const float* a,
                      const float* Wt, const float* bt, const float* Wc, const float* g, float* gWt,
                      float* gbt, float* gWc, float* gbc, void* ws, size_t ws_bytes, void* stream);

/* Adjoints of fno_pointwise_linear and fno_pointwise_mlp2 (what the backward of a whole network
 * needs around its blocks).  For a cotangent g of the output:
 *   linear:  gx = W^T g  [B][c_in][npoints];  gW[o][i] = sum g[b][o][p] x[b][i][p];  gb[o] = sum g
 *   mlp2:    with h = W1 x + b1:  gW2[o][k] = sum g_o gelu(h_k), gb2 = sum g,
 *            gh = (W2^T g) gelu'(h), gW1[k][i] = sum gh_k x_i, gb1 = sum gh, gx = W1^T gh.
 * The sums run over all batch entries and points (the adjoint of broadcasting the weights,
 * Sec. 2.1) in a fixed order: the same bits on every run.  Every output is nullable and
 * overwritten.  ws: device scratch of fno_pointwise_bwd_workspace_bytes(c_in, hidden, c_out)
 * bytes (hidden = 0 for the linear map), 8-byte aligned, owned by the caller.  Widths: c_in,
 * c_out <= 32 (linear); c_in <= 32, c_out <= 4, hidden <= 1024 (mlp2). */
int fno_pointwise_bwd_workspace_bytes(int32_t c_in, int32_t hidden, int32_t c_out, size_t* bytes);
int fno_pointwise_linear_bwd(int32_t batch, int32_t c_in, int32_t c_out, int64_t npoints, const float* x,
                             const float* W, const float* g, float* gx, float* gW, float* gb, void* ws,
                             size_t ws_bytes, void* stream);
int fno_pointwise_mlp2_bwd(int32_t batch, int32_t c_in, int32_t hidden, int32_t c_out, int64_t npoints,
                           const float* x, const float* W1, const float* b1, const float* W2, const float* g,
                           float* gx, float* gW1, float* gb1, float* gW2, float* gb2, void* ws,
                           size_t ws_bytes, void* stream);

/* Relative L2 misfit of Sec. 4 over n floats:  loss = ||pred - target||_2 / ||target||_2, written to
 * the device scalar `loss` (nullable), and its gradient with respect to pred,
 * (pred - target) / (||pred - target||_2 ||target||_2), written to grad (nullable, n floats; all
 * zero when pred equals target).  The sums are accumulated in double in a fixed order: the same
 * bits on every run.  ws: device scratch of fno_rel_l2_workspace_bytes() bytes, 8-byte aligned,
 * owned by the caller.  A zero target gives the IEEE result of the division.  Asynchronous on
 * `stream`; nothing is launched on an argument error. */
int fno_rel_l2_workspace_bytes(size_t* bytes);
int fno_rel_l2_loss(int64_t n, const float* pred, const float* target, float* loss, float* grad,
                    void* ws, size_t ws_bytes, void* stream);

/* One step of Adam (the optimiser of Sec. 4; Kingma & Ba, Algorithm 1) in place on n floats:
 *   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2;
 *   param -= lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps).
 * step counts from 1.  Complex parameters (the spectral weights) are passed as 2n floats: real
 * and imaginary parts are updated as separate reals.  All pointers are device pointers owned by
 * the caller. */
int fno_adam_step(int64_t n, float* param, const float* grad, float* m, float* v, double lr, double beta1,
                  double beta2, double eps, int32_t step, void* stream);

/* Group norm with an activation over a field of C = channels and P = npoints points, for the C / groups channels and all
 * points of every (batch entry, group) together:
 *   mean, var = sum (x - mean)^2 / n, n = P C / groups;  rstd = 1 / sqrt(var + eps);  xh = (x - mean) rstd;
 *   y = act(gamma xh + beta), gamma and beta [C], one value a channel.
 * layout FNO_LAYOUT_CHANNELS_FIRST: [B][C][P], the layout of every other call here; FNO_LAYOUT_CHANNELS_LAST: [B][P][C].
 * dtype is that of x, y, gy and gx: float, or bf16 (16 bits, each the upper half of a float).  Everything else is float.
 * Statistics are formed in double; the adjoint's sums in double, over a few values in float, whatever the dtype; bf16 results are
 * rounded once, to nearest even.  Range: x to 1e36 in size and sqrt(var + eps) from 1e-36 to 1e36, any mean beside any spread; in
 * the adjoint gy, and gy (x - mean) where it counts in the sums, from 1e-30 to 1e36.  (The adjoint starts from the saved mean, a
 * float: its xh is off by up to 2^-24 |mean| rstd, the forward call's is not.)
 * activation: FNO_ACT_IDENTITY, FNO_ACT_GELU or FNO_ACT_SILU (z / (1 + exp(-z))). */
enum { FNO_ACT_SILU = 2 };       /* the group norm's and the layer norm's calls only */
enum { FNO_LAYOUT_CHANNELS_FIRST = 0, FNO_LAYOUT_CHANNELS_LAST = 1 };
enum { FNO_DTYPE_F32 = 0, FNO_DTYPE_BF16 = 1 };
typedef struct {
  int64_t npoints;     /* P >= 0                                                      */
  double eps;          /* >= 0, finite                                                */
  int32_t batch;       /* B, 1 .. 65535, B C <= 2^23                                  */
  int32_t channels;    /* C, 1 .. 1024                                                */
  int32_t groups;      /* divides C                                                   */
  int32_t layout;      /* FNO_LAYOUT_*                                                */
  int32_t dtype;       /* FNO_DTYPE_*                                                 */
  int32_t activation;  /* FNO_ACT_*                                                   */
  int32_t flags;       /* FNO_FLAG_ACCUMULATE_GRADS (of the backward call) or 0       */
} fno_norm_desc;

/* Bytes of device scratch that both calls need for this descriptor (host-only). */
int fno_group_norm_workspace_bytes(const fno_norm_desc* desc, size_t* bytes);

/* Forward.  gamma, beta nullable (1 and 0); mean, rstd out float [B][groups], nullable: what the backward call needs.
 * y may be x itself; no other overlap.  x and y 16-byte aligned, ws 256-byte aligned.  npoints = 0 gives mean 0 and
 * rstd 1 / sqrt(eps); x and y (below x and gy) may then be null.  An infinity or a NaN in a group makes the whole group NaN.
 * Fixed summation order: the same bits on every run. */
int fno_group_norm_fwd(const fno_norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y,
                       float* mean, float* rstd, void* ws, size_t ws_bytes, void* stream);

/* Adjoint, from the statistics that the forward call saved and the cotangent gy of y; with gz = gy act'(gamma xh + beta):
 *   gbeta[c] = sum gz,  ggamma[c] = sum gz xh  (over batch entries and points, Sec. 2.1),
 *   gx = rstd (gamma gz - S1 / n - xh S2 / n),  S1 = sum gamma gz, S2 = sum gamma gz xh over the group.
 * gx, ggamma, gbeta nullable; gx is overwritten and may be gy or x itself (no other overlap); ggamma and gbeta are
 * overwritten, or added to with FNO_FLAG_ACCUMULATE_GRADS.  gamma and beta as in the forward call. */
int fno_group_norm_bwd(const fno_norm_desc* desc, const void* x, const float* gamma, const float* beta,
                       const float* mean, const float* rstd, const void* gy, void* gx, float* ggamma, float* gbeta,
                       void* ws, size_t ws_bytes, void* stream);

/* Layer norm with an activation: the statistics of every (batch entry, point) over its C channels,
 *   mean = sum_c x / C, var = sum_c (x - mean)^2 / C;  rstd = 1 / sqrt(var + eps);  xh = (x - mean) rstd;
 *   y = act(gamma xh + beta), gamma and beta [C], one value a channel.
 * Layouts, dtypes and activations as for the group norm above (rows of any other model are FNO_LAYOUT_CHANNELS_LAST).
 * Statistics and sums over channels are in float, about a mean of their own, so that a point's values may lie anywhere beside
 * their spread; bf16 results are rounded once, to nearest even.  Range: x to 5e16 in size (1e18 with up to 32 channels); squares of deviations below
 * 1e-38 are lost, which shows where eps is as small.  A NaN or an infinity makes all channels of its point NaN, and no other
 * point.  One channel gives xh = 0; so do equal channels of any value v, within 1e-11 |v| / sqrt(eps). */
typedef struct {
  int64_t npoints;     /* P >= 0                                                      */
  double eps;          /* >= 0, finite; with 0 equal channels have no value: NaN, or rounding */
  int32_t batch;       /* B, 1 .. 65535                                               */
  int32_t channels;    /* C, 1 .. 1024 channels first, 1 .. 16384 channels last       */
  int32_t layout;      /* FNO_LAYOUT_*                                                */
  int32_t dtype;       /* FNO_DTYPE_*, of x, y, gy and gx                             */
  int32_t activation;  /* FNO_ACT_*                                                   */
  int32_t flags;       /* FNO_FLAG_ACCUMULATE_GRADS (of the backward call) or 0       */
} fno_layer_norm_desc;

/* Forward.  gamma, beta nullable (1 and 0).  y may be x itself; no other overlap.  x and y 16-byte aligned; they may be null
 * where npoints is 0.  Needs no workspace, and saves nothing: the adjoint has x's statistics at hand when it has x. */
int fno_layer_norm_fwd(const fno_layer_norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y,
                       void* stream);

/* Adjoint for the cotangent gy of y, with gz = gy act'(gamma xh + beta) and h = gamma gz:
 *   gbeta[c] = sum gz,  ggamma[c] = sum gz xh  (over batch entries and points, Sec. 2.1),
 *   gx = rstd (h - sum_c h / C - xh sum_c h xh / C).
 * gx, ggamma, gbeta nullable; gx is overwritten and may be gy or x itself (no other overlap); ggamma and gbeta are
 * overwritten, or added to with FNO_FLAG_ACCUMULATE_GRADS; npoints = 0 gives gradients of zero.  Sums over points: floats in a fixed
 * order within a block, then double; the same bits on every run.  ws: device scratch of fno_layer_norm_workspace_bytes() bytes
 * (host-only call), 256-byte aligned. */
int fno_layer_norm_workspace_bytes(const fno_layer_norm_desc* desc, size_t* bytes);
int fno_layer_norm_bwd(const fno_layer_norm_desc* desc, const void* x, const float* gamma, const float* beta, const void* gy,
                       void* gx, float* ggamma, float* gbeta, void* ws, size_t ws_bytes, void* stream);

/* One AdamW step over many tensors (Loshchilov & Hutter, Algorithm 2: Adam, Sec. 4, with the decay apart from the
 * gradient), in place, in as few launches as the tensors' addresses fit (64 tensors each).  For every value
 *   g' = s g;  m = beta1 m + (1 - beta1) g';  v = beta2 v + (1 - beta2) g'^2;
 *   param = param (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps),
 * s = min(1, max_norm / *grad_norm), or 1 where grad_norm is null.  grad_norm is a device scalar (of fno_grad_norm): where
 * it is not finite the step writes nothing at all.  Complex parameters are passed as 2n floats.  step counts from 1.
 *
 * state_bits 32: m and v are float [n], exps is not used.
 * state_bits 8: m and v are bytes [n] and exps bytes [ceil(n / 256)][2], the exponents that the 256 consecutive values of
 * a block share, m's and v's.  With E the exponent, a code's lower three bits f and the bits e above them stand for
 * (1 + f / 8) 2^(e + E - 127 - K), code 0 for zero: v has no sign, five bits e and K = 31; m has its sign in bit 7, four bits
 * e and K = 15.  All bytes zero are moments of zero.  E = 255 (its codes are 0): a value of the block was not finite, and every
 * one of it is NaN from then on.  The update uses the new moments before they are rounded.  They are rounded up or down at
 * random with the odds that keep the mean (a decay of 0.1 % a step would never move a code otherwise), by a hash of seed, step,
 * the tensor's place in the list and the value's place in it: the same bits on every run.  A v that is not zero is at least the smallest
 * code, so that no step is divided by a vanished v.
 *
 * tensors: host array, read during the call only; every pointer in it is a device pointer, param, grad, m and v 4-byte
 * aligned, exps 2-byte.  Tensors must not overlap.  n = 0 and count = 0 are allowed. */
typedef struct {
  float* param;
  const float* grad;
  void* m;
  void* v;
  void* exps;            /* state_bits 8 only, else ignored */
  int64_t n;
  double weight_decay;
} fno_adamw_tensor;
int fno_adamw_step(int32_t count, const fno_adamw_tensor* tensors, int32_t state_bits, double lr, double beta1,
                   double beta2, double eps, int32_t step, const float* grad_norm, double max_norm, uint32_t seed,
                   void* stream);

/* The Euclidean norm of all gradients of the list together, to the device scalar `norm`; sums in double in a fixed order,
 * the same bits on every run.  param, m, v and exps of the tensors are not used.  ws: device scratch of
 * fno_grad_norm_workspace_bytes() bytes (host-only call), 8-byte aligned. */
int fno_grad_norm_workspace_bytes(int32_t count, const fno_adamw_tensor* tensors, size_t* bytes);
int fno_grad_norm(int32_t count, const fno_adamw_tensor* tensors, float* norm, void* ws, size_t ws_bytes, void* stream);

/* The values that moments in 8 bits stand for, as bf16, which every code is exactly: m_out[k], v_out[k] (host arrays of
 * `count` device pointers, 4-byte aligned, null only where n = 0) receive n bf16 values of tensor k.  param and grad are not
 * used. */
int fno_adamw_state_read(int32_t count, const fno_adamw_tensor* tensors, void* const* m_out, void* const* v_out,
                         void* stream);

/* One Muon step over many tensors of matrices, in place: the momentum of every matrix, made orthogonal by Newton-Schulz
 * products (Higham, Functions of Matrices, ch. 8), is what moves it (Jordan et al., 2024: Muon, an optimizer for the hidden layers of neural
 * networks, whose coefficients a, b, c = 3.4445, -4.7750, 2.0315 are the binding's).  For every matrix on its own
 *   g' = s g;  m = momentum m + g';  u = g' + momentum m where nesterov is set, else m;  X = u / (||u||_F + eps);
 *   `iterations` times:  X = a X + (b A + c A A) X,  A = X X^H;
 *   param = param (1 - lr weight_decay) - lr scale X,
 * s from grad_norm and max_norm as in fno_adamw_step: where *grad_norm is not finite nothing is written at all.  A matrix of
 * zeros stays one (X = 0), one that holds a NaN or an infinity becomes NaN, and no other matrix of the list does.
 *
 * kind FNO_MUON_MATRICES: float [batch][rows][cols], a stack of real matrices (batch 1: one).
 * kind FNO_MUON_MODES: complex [rows][cols][batch], the layout of the spectral weights R [Cin][Cout][modes]: one complex matrix
 * for every kept mode, the map that the mode mix applies there.  rows, cols <= 32 (FNO_EUNSUPPORTED beyond).
 *
 * Products: single precision for spectral weights and for real matrices with up to 32 on their shorter side and 16384 values;
 * for the others sums of products of 16-bit parts that carry 22 bits of a value, none of them below 2^-35 in X, 2^-33 in A and
 * 2^-31 in b A + c A A, as long as X stays within 64, A within 256 and b A + c A A within 1024 (singular values of X up to 1.2,
 * which the usual coefficients keep, are far from that; what leaves these ranges becomes infinite or NaN).  Sums in float in a
 * fixed order: the same bits on every run of the same list.  Norms: squares in double, those of spectral matrices in float where it
 * holds them (sums between 1e-28 and 1e30).
 *
 * tensors, options: host memory, read during the call only; pointers in tensors are device pointers, param, grad and momentum
 * 4-byte aligned (8-byte: complex ones).  Tensors must not overlap.  Empty tensors (batch, rows or cols 0) and count = 0 are
 * allowed.  ws: device scratch of fno_muon_workspace_bytes() bytes (host-only call), 256-byte aligned; null where that is 0. */
enum { FNO_MUON_MATRICES = 0, FNO_MUON_MODES = 1 };
typedef struct {
  float* param;
  const float* grad;
  float* momentum;
  int64_t batch;         /* matrices, 0 .. 2^31 - 1                                   */
  int32_t rows, cols;    /* 0 .. 32768                                                */
  int32_t kind;          /* FNO_MUON_*                                                */
  double scale;          /* of the step; finite                                       */
  double weight_decay;   /* finite                                                    */
} fno_muon_tensor;
typedef struct {
  double lr, momentum;   /* finite; 0 <= momentum < 1                                 */
  double eps;            /* >= 0                                                      */
  double a, b, c;        /* finite                                                    */
  int32_t iterations;    /* 0 .. 64                                                   */
  int32_t nesterov;      /* 0 or 1                                                    */
} fno_muon_options;
int fno_muon_workspace_bytes(int32_t count, const fno_muon_tensor* tensors, size_t* bytes);
int fno_muon_step(int32_t count, const fno_muon_tensor* tensors, const fno_muon_options* options, const float* grad_norm,
                  double max_norm, void* ws, size_t ws_bytes, void* stream);

/* Projection to the output channels (end of Sec. 2.4) through one hidden layer, fused per point:
 *   y = W2 gelu(W1 x + b1) + b2,  W1 [hidden][c_in], W2 [c_out][hidden].  The hidden tensor is
 * never stored.  c_in <= 32, c_out <= 4. */
int fno_pointwise_mlp2(int32_t batch, int32_t c_in, int32_t hidden, int32_t c_out, int64_t npoints,
                       const float* x, const float* W1, const float* b1, const float* W2,
                       const float* b2, float* y, void* stream);

/* For callers that cannot allocate device memory or bring a workspace (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): fno_spectral_conv_fwd with the
 * workspace taken from a fixed array of FNO_STATIC_SCRATCH_BYTES bytes of device memory (and 5 MiB
 * for tables) that the library owns (one copy per GPU it runs on, held until the process ends).  Arguments, layout,
 * results and error codes are those of fno_spectral_conv_fwd; the call allocates and frees
 * nothing.  Shapes whose fno_workspace_bytes(FNO_OP_SPECTRAL_CONV_FWD) exceeds the array are
 * refused with FNO_ENOSPC and nothing is launched.  The first call on a device looks up the
 * array's address there (make that call outside any capture).  All calls on one GPU share the
 * array: every byte a call reads from it is written earlier by the same call, so leftovers of the
 * previous call do no harm, but two calls that overlap in time on one GPU (different streams or
 * threads) race; order them. */
#define FNO_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
int fno_spectral_conv_fwd_static(const fno_desc* desc, const float* x, const float* R, float* y,
                                 float* xhat_save, void* stream);

/* Benchmark hooks, outside the paper's layer: per-stage timing.  While enabled, every library call brackets each kernel it
 * launches with a pair of HIP events on the call's stream (events are created on first use and
 * kept).  fno_timing_enable takes a mask of stages, bit (1 << FNO_STAGE_*) per stage, FNO_TIMING_ALL
 * for every stage, 0 to switch timing off: an event pair costs a few microseconds of idle time
 * between kernels, so a caller that times a whole step and wants one kernel's duration from the
 * same run enables that stage alone.  fno_timing_read waits for the recorded events, returns up to `capacity` records in
 * launch order (stage id FNO_STAGE_*, elapsed milliseconds; host arrays) and clears the log.  Small layers run the
 * x stage, the mode mix and the x stage back as one launch, recorded under FNO_STAGE_MIX or FNO_STAGE_MIX_BWD: these
 * stages then hold the x transforms, and no record has an x stage's id (but for an adjoint that works the spectrum of x
 * out again: its x stage keeps FNO_STAGE_X_FWD).
 * This log is the library's only process-wide state and is not thread-safe; leave it disabled
 * under graph capture.  At most 8192 records are kept between reads. */
enum {
  FNO_STAGE_TZ_FWD = 0, FNO_STAGE_Y_FWD = 1, FNO_STAGE_X_FWD = 2, FNO_STAGE_MIX = 3,
  FNO_STAGE_X_INV = 4, FNO_STAGE_Y_INV = 5, FNO_STAGE_ZT_INV = 6, FNO_STAGE_MIX_BWD = 7,
  FNO_STAGE_BWD_POINTWISE = 8
};
#define FNO_TIMING_ALL (-1)
int fno_timing_enable(int stage_mask);
int fno_timing_read(int32_t* stages, float* ms, int32_t capacity, int32_t* count);

/* Text for a status code; for FNO_EHIP / FNO_EUNSUPPORTED the calling thread's last detail. */
const char* fno_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* FNO_H_ */
