/*
 * auvnet.h -- C ABI of the network operators in libauvenv.so: what a policy
 * or critic with memory, or one with dropout and normalisation, needs next to
 * the dense products (auv_gemm).
 *
 *  - net_gate_scan: a gated linear recurrence along a trajectory, with the
 *    episode ends of the rollout (hidden currents and randomised parameters,
 *    paper §IV-C, are not in the observation: a network that is to know them
 *    has to remember), its backward pass, and with T = 1 its single step.
 *  - net_group_norm: group norm with an activation, channels last, and its
 *    backward pass; one group and one position is the layer norm of DroQ's
 *    critic (paper §III-A; Hiraoka et al. 2022).
 *  - net_dropout: dropout whose mask is drawn where it is used and never
 *    stored, optionally added to a residual; the backward pass is the same
 *    call on the gradient.
 *  - net_causal_conv and net_select_scan: a memory with many states a channel,
 *    whose decays and inputs are chosen by the input (a selective state space
 *    layer), and the short convolution in front of it; both with the rollout's
 *    episode ends, their backward passes and, with T = 1, their single steps.
 *  - net_orthogonalise: weight matrices' updates with their singular values
 *    moved towards 1 by Newton-Schulz products.
 *
 * Conventions
 *  - Return value: AUV_OK (0) or a negative AUV_ERR_* code (auvenv.h);
 *    net_last_error() gives the calling thread's reason for its last failure.
 *    No entry point aborts, traps or throws.
 *  - Asynchrony: every call only enqueues work on `stream` (a cudaStream_t;
 *    NULL = the legacy default stream).  No call synchronises, allocates or
 *    keeps anything: calls can be captured in a CUDA graph.
 *  - Memory: every array is device memory (AUV_ERR_SIZE otherwise) of the
 *    current device (AUV_ERR_INVALID otherwise), owned by the caller.  Activations are fp32, bf16 or fp16 (all
 *    of a call the same); states, statistics, weights and their gradients are
 *    fp32, and so is all arithmetic: a 16-bit result is rounded once (to
 *    nearest even) when it is stored.
 *  - Layout: an activation is a net_rows: rows of contiguous channels, row
 *    (i, j) anywhere.  Inputs may repeat rows (stride 0); rows of an output
 *    must not overlap (AUV_ERR_SIZE), and an output must not overlap another
 *    array of the call, except where a call says so.
 *  - Sizes of 0 are valid: nothing is read, sums over nothing are 0.
 *  - Reproducible: every sum has a fixed order, which follows from the sizes,
 *    the strides and how the data pointers are aligned (up to 16 bytes): a call
 *    repeated with the same of these and the same inputs gives the same bits.
 *  - Workspaces: a query takes the argument block as the call will get it.
 *    Where an array's data is still NULL, the answer serves any alignment and
 *    any strides that it may come to have, and every output.
 */
#ifndef AUVNET_H
#define AUVNET_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* types of activations */
#define NET_FP32 0
#define NET_BF16 1
#define NET_FP16 2

/* activations of net_group_norm */
#define NET_ACT_NONE 0
#define NET_ACT_RELU 1
#define NET_ACT_SILU 2
#define NET_ACT_TANH 3

/* Rows of channels: element (i, j, k) is data[i * outer + j * inner + k],
 * strides in elements, not negative. */
typedef struct net_rows {
  void* data;
  int64_t outer, inner;
} net_rows;

/*
 * net_gate_scan: for every env n and channel d, along the steps t
 *
 *   a = sigmoid(f[t]),  h[t] = a c[t] + (1 - a) v[t],   y[t] = h[t] rounded,
 *   c[t] = 0 where an episode ended before step t, else h[t - 1];  h[-1] = h0,
 *
 * hT = h[T - 1].  An episode ended before step t where done[t - 1][n] is
 * nonzero (the rollout's array), before step 0 where done_prev[n] is: the
 * last step's flags of the call before.  Whatever the ended episode's state
 * held, infinities and NaN too, nothing of it passes.  Without an end a state
 * that is infinite stays so until a gate is 0 in fp32 (f below -87), after
 * which it is infinite or NaN.  In a rollout T = 1:
 * done_prev = the env's last flags, hT = h0 for a state updated in place.
 *
 * f, v, y (i = t, j = n) and done, done_prev, h0, hT; the others are not read.
 * h0, done, done_prev, hT may be NULL: zeros, no ends, not wanted.  h0 = hT is
 * allowed.
 *
 * net_gate_scan_backward: the gradients df, dv (and dh0 unless NULL) from dy,
 * dhT (NULL: zeros), the same f, v, h0, done, done_prev, and y as the forward
 * call stored it.  With d[t] the gradient of h[t] and g[T] = dhT,
 *
 *   d[t] = dy[t] + g[t + 1],   dv[t] = (1 - a) d[t],
 *   df[t] = a (1 - a) (c[t] - v[t]) d[t],
 *   g[t] = 0 where an episode ended before step t, else a d[t];   dh0 = g[0].
 *
 * c is taken from y: with 16-bit activations its rounding is the one
 * difference from the gradient of the unrounded recurrence (2^-9 of a state
 * for bf16, as much as v's own), and it saves a second array of states.
 * hT is not read.  dh0 = dhT is allowed.
 *
 * workspace: net_gate_scan_workspace_bytes(a, backward) bytes, 16-byte
 * aligned (AUV_ERR_SIZE if there is less): 0 below 32 steps, and wherever the
 * sequence need not be split into pieces; rows that follow each other in
 * memory and rows that do not may differ in that.
 */
typedef struct net_scan {
  uint32_t struct_size;           /* sizeof(net_scan): version guard          */
  uint32_t dtype;                 /* NET_*: type of f, v, y, dy, df, dv       */
  int64_t T, N, D;                /* steps, envs, channels                    */
  net_rows f, v, y, dy, df, dv;   /* [T][N][D]                                */
  const float* h0;                /* [N][D]                                   */
  float* hT;                      /* [N][D]                                   */
  const float* dhT;               /* [N][D]                                   */
  float* dh0;                     /* [N][D]                                   */
  const uint8_t* done;            /* [T][N]                                   */
  const uint8_t* done_prev;       /* [N]                                      */
  void* workspace;
  size_t workspace_bytes;
} net_scan;
size_t net_gate_scan_workspace_bytes(const net_scan* a, int backward);
int net_gate_scan(const net_scan* a, void* stream);
int net_gate_scan_backward(const net_scan* a, void* stream);

/*
 * net_group_norm: x [B][S][C] (i = b, j = s), channels in G groups of C / G.
 * With mean and var the mean and the (biased) variance of group g of instance
 * b over its S positions and C / G channels,
 *
 *   xh = (x - mean) rstd,  rstd = 1 / sqrt(var + eps),
 *   y = act(gamma xh + beta),
 *
 * mean and rstd [B][G] are outputs.  gamma, beta [C]; NULL: ones, zeros.  Where
 * the sum of squared deviations passes fp32's range (deviations of some 10^19
 * and more), rstd is 0 and y = act(beta).
 *
 * net_group_norm_backward: dx, and dgamma, dbeta [C] (each NULL: not wanted)
 * from dy, and x, gamma, beta, mean, rstd as in the forward call.  With
 * dz = dy act'(gamma xh + beta), w = gamma dz and averages over the group:
 *
 *   dbeta = sum dz,  dgamma = sum dz xh  (over b and s),
 *   dx = rstd (w - avg(w) - xh avg(w xh)).
 *
 * workspace: net_group_norm_workspace_bytes(a, backward) bytes, 16-byte
 * aligned (AUV_ERR_SIZE if there is less): 0 forward where a group has at most
 * 2,048 values and there are at most 32,768 groups, and often otherwise; the
 * alignment of rows and data, and whether dgamma or dbeta is wanted, count.
 */
typedef struct net_norm {
  uint32_t struct_size;           /* sizeof(net_norm): version guard          */
  uint32_t dtype;                 /* NET_*: type of x, y, dy, dx              */
  uint32_t act;                   /* NET_ACT_*                                */
  float eps;                      /* >= 0                                     */
  int64_t B, S, C, G;
  net_rows x, y, dy, dx;          /* [B][S][C]                                */
  const float *gamma, *beta;      /* [C]                                      */
  float *mean, *rstd;             /* [B][G]                                   */
  float *dgamma, *dbeta;          /* [C]                                      */
  void* workspace;
  size_t workspace_bytes;
} net_norm;
size_t net_group_norm_workspace_bytes(const net_norm* a, int backward);
int net_group_norm(const net_norm* a, void* stream);
int net_group_norm_backward(const net_norm* a, void* stream);

/*
 * net_dropout: y = residual + (dropped ? 0 : x / (1 - p)), elements of
 * x [T][N][D] (i = t, j = n) dropped with probability p, in steps of 2^-16:
 * with e = (t N + n) D + d, or n D + d if shared (one mask for all t), element
 * e is dropped where u < round(65536 p), u the 16 bits number e % 8 (word by
 * word, low half first) of Philox4x32-10 at counter (e / 8 low, e / 8 high,
 * draw low, draw high) with key (seed low, seed high).  1 - p is that of the
 * rounded p; at p = 1 all are dropped.  A dropped element passes nothing of x,
 * infinities and NaN neither.  residual.data = NULL: none.  The gradient by x
 * is the same call on dy without the residual; that by the residual is dy.
 * y may be x, or the residual, itself (same pointer and strides).
 */
typedef struct net_drop {
  uint32_t struct_size;           /* sizeof(net_drop): version guard          */
  uint32_t dtype;                 /* NET_*: type of x, residual, y            */
  uint32_t shared;                /* 0 or 1                                   */
  uint32_t reserved;              /* 0                                        */
  int64_t T, N, D;
  net_rows x, residual, y;        /* [T][N][D]                                */
  double p;                       /* 0 <= p <= 1                              */
  uint64_t seed, draw;
} net_drop;
int net_dropout(const net_drop* a, void* stream);

/*
 * net_causal_conv: for every env n and channel d, along the steps t
 *
 *   y[t] = act(b + sum over k < K of w[k] x[t - (K - 1) + k]),
 *
 * with x[-j] = state[K - 1 - j], and in the place of rows behind an episode end
 * zeros: what an ended episode's rows held, infinities and NaN too, passes
 * nothing on.  new_state: the last K - 1 rows of (state, x), zeros where an
 * episode has ended ahead of the last step; the next call's state, together
 * with its done_prev.  done, done_prev as in net_gate_scan.  state and
 * new_state are of the activations' type; new_state may be state.  bias,
 * state, new_state, done, done_prev may be NULL: zeros, zeros, not wanted, no
 * ends.  act: NET_ACT_NONE or NET_ACT_SILU.  K <= 8 (AUV_ERR_UNSUPPORTED).
 *
 * net_causal_conv_backward: dx, dw, dbias and dstate (each of the last three
 * unless NULL) from dy, dnew_state (NULL: zeros) and what the forward call had.
 * With p the sums in front of act and dp = dy act'(p),
 *
 *   dx[s] = sum over j of w[K - 1 - j] dp[s + j], j < K, of the steps s + j
 *           that see row s, + dnew_state where row s is left in the state,
 *   dw[k] = sum of dp[t] x[t - (K - 1) + k],   dbias = sum of dp,
 *
 * dstate as dx, for the rows ahead of the first.
 *
 * workspace: net_causal_conv_workspace_bytes(a, backward) bytes, 16-byte
 * aligned: 0 forward, and backward where neither dw nor dbias is wanted.
 */
typedef struct net_conv {
  uint32_t struct_size;           /* sizeof(net_conv): version guard          */
  uint32_t dtype;                 /* NET_*: type of x, y, dy, dx, the states  */
  uint32_t act;                   /* NET_ACT_NONE or NET_ACT_SILU             */
  uint32_t reserved;              /* 0                                        */
  int64_t T, N, D, K;             /* steps, envs, channels, taps              */
  net_rows x, y, dy, dx;          /* [T][N][D]                                */
  const float *w, *bias;          /* [K][D], [D]                              */
  const void* state;              /* [K - 1][N][D]                            */
  void* new_state;                /* [K - 1][N][D]                            */
  const void* dnew_state;         /* [K - 1][N][D]                            */
  void* dstate;                   /* [K - 1][N][D]                            */
  float *dw, *dbias;              /* [K][D], [D]                              */
  const uint8_t* done;            /* [T][N]                                   */
  const uint8_t* done_prev;       /* [N]                                      */
  void* workspace;
  size_t workspace_bytes;
} net_conv;
size_t net_causal_conv_workspace_bytes(const net_conv* a, int backward);
int net_causal_conv(const net_conv* a, void* stream);
int net_causal_conv_backward(const net_conv* a, void* stream);

/*
 * net_select_scan: a state space layer whose step sizes, inputs and outputs are
 * functions of the input.  For every env n, channel d with S states, and g the
 * group of D / G channels that d is in, along the steps t
 *
 *   e = softplus(dt[t] + dt_bias),
 *   h[t][s] = exp(e A[d][s]) c[t][s] + e B[t][g][s] x[t],
 *   y[t] = (sum over s of C[t][g][s] h[t][s] + skip x[t]) silu(gate[t]),
 *
 * c[t] = 0 where an episode ended before step t (done, done_prev as in
 * net_gate_scan), else h[t - 1]; h[-1] = h0, hT = h[T - 1].  Nothing of an
 * ended episode's state passes.  A state that has become infinite is infinite
 * or NaN until its episode ends.  In a rollout T = 1, done_prev = the env's
 * last flags and hT = h0 for states updated in place.
 *
 * B and C have rows of G S channels.  h0, hT and kept are fp32.  kept
 * [(T + 15) / 16][N][D][S]: h before steps 0, 16, 32, ..., from which the
 * backward pass starts again.  gate.data, skip, dt_bias, h0, done, done_prev
 * may be NULL: no gate, zeros, zeros, zeros, no ends; hT, kept: not wanted.
 * S <= 128 (AUV_ERR_UNSUPPORTED).
 *
 * net_select_scan_backward: gradients from dy, dhT (NULL: zeros), kept as the
 * forward call wrote it, and the other arguments of that call (h0 is kept's
 * first state).  With p = dy silu(gate), f the gradient of h[t], G' = that of
 * c[t + 1] (dhT after the last step), and sums over the s of a channel, the d
 * of a group, or all t and n, as the output's indices say,
 *
 *   f = C p + G',   dC = sum p h,   dB = sum e x f,   dA = sum f a c e,
 *   dx = skip p + e sum B f,   de = sum f (a c A + B x),   dskip = sum p x,
 *   ddt = de sigmoid(dt + dt_bias),   ddt_bias = sum ddt,
 *   dgate = dy silu'(gate) (y in front of the gate),
 *   gradient of c[t] = a f, or 0 where an episode ended before step t;
 *   dh0 that of c[0],
 *
 * a = exp(e A).  dA, dskip, ddt_bias, dgate.data, dh0 may be NULL: not wanted;
 * dgate has no use without a gate.  dh0 = dhT is allowed.
 *
 * workspace: net_select_scan_workspace_bytes(a, backward) bytes, 16-byte
 * aligned; forward 0 unless envs and channels are few and steps many.
 */
typedef struct net_select {
  uint32_t struct_size;           /* sizeof(net_select): version guard        */
  uint32_t dtype;                 /* NET_*: type of the rows                  */
  int64_t T, N, D, S, G;          /* steps, envs, channels, states, groups    */
  net_rows x, dt, gate, y;        /* [T][N][D]                                */
  net_rows B, C;                  /* [T][N][G S]                              */
  net_rows dy, dx, ddt, dgate;    /* [T][N][D]                                */
  net_rows dB, dC;                /* [T][N][G S]                              */
  const float* A;                 /* [D][S]                                   */
  const float *skip, *dt_bias;    /* [D]                                      */
  const float* h0;                /* [N][D][S]                                */
  float* hT;                      /* [N][D][S]                                */
  float* kept;                    /* [(T + 15) / 16][N][D][S]                 */
  const float* dhT;               /* [N][D][S]                                */
  float* dh0;                     /* [N][D][S]                                */
  float* dA;                      /* [D][S]                                   */
  float *dskip, *ddt_bias;        /* [D]                                      */
  const uint8_t* done;            /* [T][N]                                   */
  const uint8_t* done_prev;       /* [N]                                      */
  void* workspace;
  size_t workspace_bytes;
} net_select;
size_t net_select_scan_workspace_bytes(const net_select* a, int backward);
int net_select_scan(const net_select* a, void* stream);
int net_select_scan_backward(const net_select* a, void* stream);

/*
 * net_orthogonalise: y = p(p(...(x / (|x| + eps)))), `steps` times, of each of
 * the L matrices x [M][N] (i = the matrix, j = the row), |x| its Frobenius
 * norm, with
 *
 *   p(x) = a x + (b P + c P P) x,   P = x x^T,
 *
 * which takes each singular value v to a v + b v^3 + c v^5 and leaves the
 * singular vectors: with coef (a, b, c) = (3.4445, -4.775, 2.0315) and five
 * steps an update's singular values come to lie about 1.  Where M > N the
 * products are x (b P + c P P) with P = x^T x, the same polynomial.  Norms are
 * taken in range whatever the scale of x, from the smallest subnormal to the
 * largest number.  steps = 0: y = x / (|x| + eps).  y may be x.  A matrix with a
 * value that is not finite comes out as NaN, whatever the steps; so does one of
 * zeros with eps = 0.
 *
 * The products are taken of two fp16 pieces of every value (22 bits, and not
 * below 2^-37 for a value of x / (|x| + eps): where |x| is far below eps, that is
 * less) with sums in fp32, so the coefficients have to keep what is between them in fp16's
 * range: from v in [0, 1] no singular value may come above 8, nor
 * |a| + |b| v^2 + |c| v^4 above 1000 (AUV_ERR_UNSUPPORTED; the usual ones reach 1.3 and 15).
 *
 * workspace: net_orthogonalise_workspace_bytes(a) bytes, 256-byte aligned.  Its
 * first 32-bit word is AUV_OK after the call has run, or AUV_ERR_TIMEOUT where
 * a wait inside a kernel gave up (2 s); y then holds NaN in the place of every
 * value that finished products have not come to.
 *
 * net_orthogonalise_selftest_timeout: failure-detection self-test.  The same
 * call, but that behind the product-th of its 3 * steps products (1 on, ahead
 * of the last) one block waits for something that never comes, and all waits
 * give up after limit_us microseconds (1 .. 5e6).  Matrices of one tile
 * (M, N <= 128) have no such wait: the call is then net_orthogonalise.
 */
typedef struct net_ortho {
  uint32_t struct_size;           /* sizeof(net_ortho): version guard         */
  uint32_t dtype;                 /* NET_*: type of x and y                   */
  uint32_t steps;                 /* <= 64                                    */
  float eps;                      /* >= 0                                     */
  float coef[3];
  uint32_t reserved;              /* 0                                        */
  int64_t L, M, N;
  net_rows x, y;                  /* [L][M][N]                                */
  void* workspace;
  size_t workspace_bytes;
} net_ortho;
size_t net_orthogonalise_workspace_bytes(const net_ortho* a);
int net_orthogonalise(const net_ortho* a, void* stream);
int net_orthogonalise_selftest_timeout(const net_ortho* a, uint32_t product, uint32_t limit_us, void* stream);

const char* net_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* AUVNET_H */
