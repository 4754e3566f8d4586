/*
 * qd_seq.h -- C ABI of libqdseq.so: the layers of a sequence policy over
 * episodes, for MI355X (gfx950).
 *
 * An archive's elites act for episodes of up to some thousand steps.  A
 * sequence policy fitted to those episodes, or rolled out in their place, is
 * told the wanted descriptor in its first tokens and then reads one token per
 * step.  This library has the operators of its blocks:
 *
 *   - root-mean-square norm with the residual's addition, with its gradient,
 *     and with an output in 8 bits (e4m3) and scales;
 *   - attention over a sliding window whose first tokens ("sinks", here the
 *     descriptor's) stay visible, with its gradient, and its single-token form
 *     over a ring cache;
 *   - linear attention with a decay for each head, by chunks, with its
 *     gradient, and its recurrent form for single tokens.
 *
 * Conventions for every entry point (those of qd.h):
 *   - Plain C types only.  `stream` is a hipStream_t passed as void*; work is
 *     enqueued on it and nothing waits for the GPU.
 *   - Every call returns a qds_status; nothing throws across the ABI.
 *     Arguments are checked before any launch.
 *   - The caller owns all device memory.  A call that needs scratch memory
 *     takes a workspace (256-byte aligned) of the size that its *_workspace
 *     function gives; its content means nothing before or after the call.
 *   - Calls keep no state: they may run on any streams and threads, as long
 *     as calls that run at the same time have workspaces of their own.
 *   - Results do not depend on timing: no sum is formed by atomics.
 *   - Empty tensors (no rows, batch 0, length 0) are valid and launch nothing,
 *     except that outputs that are sums over them are still written.
 */
#ifndef QD_SEQ_H
#define QD_SEQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define QDS_ABI_VERSION 1u

/* The numbers of qd_status, as far as they occur here. */
typedef enum {
  QDS_OK = 0,
  QDS_ERR_INVALID_ARG = 1,          /* bad config field, null or misaligned pointer */
  QDS_ERR_WORKSPACE_TOO_SMALL = 2,  /* workspace shorter than needed                */
  QDS_ERR_UNSUPPORTED = 4,          /* valid but not built (e.g. head dimension), or */
                                    /*   a launch of 2^32 threads or more            */
  QDS_ERR_HIP = 5                   /* a HIP runtime or launch error                */
} qds_status;

/* Types of tensors. */
enum { QDS_F32 = 0, QDS_BF16 = 1, QDS_F16 = 2 };

/* A tensor of rows per batch element and head: element (b, t, h, d) is
 * data[b * stride[0] + t * stride[1] + h * stride[2] + d].  Strides are in
 * elements; any sign or order, also 0; multiples of 8, as data is of 16 bytes.
 * Rows that are read by tiles (keys and values, and all inputs of a backward pass
 * or of the decay attention) are less than 2^23 elements apart; others are
 * QDS_ERR_UNSUPPORTED. */
typedef struct {
  void* data;
  int64_t stride[3];
} qds_view;

/* ------------------------------------------------------------------------
 * Root-mean-square norm with the residual's addition
 *
 *   h = x + residual;  rstd = (mean(h^2) + eps)^(-1/2);  y = h rstd weight
 *
 * over rows of `width` elements.  Sums are in fp32 and y comes from the sum
 * before it is rounded to the stored h.  residual may be null (h = x).
 * ------------------------------------------------------------------------ */
typedef struct {
  uint32_t abi_version;   /* QDS_ABI_VERSION                                        */
  int32_t dtype;          /* QDS_*: x, residual, h, y, dy, dh, dx                   */
  int32_t weight_dtype;   /* QDS_F32 or dtype: weight, dweight                      */
  int32_t width;          /* elements per row, 1 .. 2^20                            */
  int64_t rows;           /* >= 0                                                   */
  float eps;              /* >= 0                                                   */
  int32_t group;          /* 8-bit output: columns per scale; 0 = the whole row,    */
                          /*   else 128, which must divide width.  0 elsewhere.     */
} qds_norm_config;

/* y, h [rows][width] of dtype and rstd [rows] fp32, contiguous.  Inputs have a
 * row stride in elements. */
qds_status qds_residual_norm(const qds_norm_config* c, const void* x, int64_t x_stride,
                             const void* residual, int64_t residual_stride, const void* weight,
                             void* y, void* h, float* rstd, void* stream);

/* The same with y in e4m3 (OCP): q [rows][width] bytes and scale
 * [rows][width / group or 1] fp32, y ~ q * scale, scale = max |y| of its
 * columns / 448.  Columns that are all zero get scale 1; a maximum below 2^-100
 * counts as 2^-100.  Not-a-number stays so; an infinite row is 0 or
 * not-a-number, as y is.  dtype is 16 bits or fp32. */
qds_status qds_residual_norm_fp8(const qds_norm_config* c, const void* x, int64_t x_stride,
                                 const void* residual, int64_t residual_stride, const void* weight,
                                 void* q, float* scale, void* h, void* stream);

/* dx [rows][width] (the gradient of x and of residual alike) and dweight
 * [width] from dy, dh (the gradient that reaches h by other ways; may be null),
 * the stored h and rstd. */
qds_status qds_residual_norm_backward_workspace(const qds_norm_config* c, uint64_t* bytes);
qds_status qds_residual_norm_backward(const qds_norm_config* c, const void* dy, int64_t dy_stride,
                                      const void* dh, int64_t dh_stride, const void* h,
                                      int64_t h_stride, const float* rstd, const void* weight,
                                      void* dx, void* dweight, void* workspace,
                                      uint64_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Attention over a sliding window whose first tokens stay visible
 *
 * Row i of an episode of n rows sees row j where  j <= i < n  and
 * (i - j < window or j < sinks);  o_i = sum_j softmax_j(scale q_i k_j) v_j.
 * Query head h reads key head h / (heads / kv_heads).
 * ------------------------------------------------------------------------ */
typedef struct {
  uint32_t abi_version;   /* QDS_ABI_VERSION                                        */
  int32_t dtype;          /* QDS_BF16 or QDS_F16                                    */
  int32_t batch;          /* >= 0                                                   */
  int32_t length;         /* rows per batch element, >= 0; unused by the step       */
  int32_t heads;          /* a multiple of kv_heads                                 */
  int32_t kv_heads;       /* >= 1                                                   */
  int32_t dim;            /* a multiple of 8, 8 .. 128                              */
  int32_t window;         /* >= 1                                                   */
  int32_t sinks;          /* >= 0; window + sinks < 2^30                            */
  float scale;
} qds_window_config;

/* o [batch][length][heads][dim] and lse [batch][heads][length] fp32 (natural
 * logarithm of each row's sum of exponentials; -infinity where i >= n).
 * lengths [batch] int32 gives n (clamped to 0 .. length; null: all `length`);
 * rows from n on are not read and get o = 0.  Rows must be 16-byte aligned. */
qds_status qds_window_forward(const qds_window_config* c, qds_view q, qds_view k, qds_view v,
                              const int32_t* lengths, qds_view o, float* lse, void* stream);

/* dq, dk, dv (rows from n on get 0) from do and what the forward call saw and
 * gave. */
qds_status qds_window_backward_workspace(const qds_window_config* c, uint64_t* bytes);
qds_status qds_window_backward(const qds_window_config* c, qds_view dout, qds_view q, qds_view k,
                               qds_view v, qds_view o, const float* lse, const int32_t* lengths,
                               qds_view dq, qds_view dk, qds_view dv, void* workspace,
                               uint64_t workspace_bytes, void* stream);

/* The ring cache: k_cache, v_cache [batch][kv_heads][sinks + window][dim],
 * contiguous.  Position p is kept in slot p (p < sinks) or
 * sinks + (p - sinks) mod window.
 *
 * One token: writes k and v of position pos[b] into their slots, then attends
 * with q to what the token sees.  Positions 0 .. pos[b] - 1 (as far as still
 * kept) must have been written before.  pos[b] < 0: the cache is left alone
 * and o is 0.  q, k, v, o have no rows (stride[1] unused). */
qds_status qds_window_step_workspace(const qds_window_config* c, uint64_t* bytes);
qds_status qds_window_step(const qds_window_config* c, qds_view q, qds_view k, qds_view v,
                           void* k_cache, void* v_cache, const int32_t* pos, qds_view o,
                           void* workspace, uint64_t workspace_bytes, void* stream);

/* Writes the rows of a prompt that are still kept after its n rows into the
 * cache (slots without one are left alone). */
qds_status qds_window_cache_fill(const qds_window_config* c, qds_view k, qds_view v,
                                 const int32_t* lengths, void* k_cache, void* v_cache,
                                 void* stream);

/* ------------------------------------------------------------------------
 * Linear attention with a decay for each head
 *
 *   S_t = a_h S_{t-1} + k_t v_t^T;  o_t = scale q_t S_t;  a_h = exp(log_decay_h)
 *
 * State S is [dim_k][dim_v] fp32 for each batch element and head.
 * ------------------------------------------------------------------------ */
typedef struct {
  uint32_t abi_version;   /* QDS_ABI_VERSION                                        */
  int32_t dtype;          /* QDS_BF16 or QDS_F16                                    */
  int32_t batch;          /* >= 0                                                   */
  int32_t length;         /* rows per batch element, >= 0; unused by the step       */
  int32_t heads;          /* >= 1                                                   */
  int32_t dim_k, dim_v;   /* multiples of 8, 8 .. 128                               */
  float scale;
} qds_decay_config;

/* o [batch][length][heads][dim_v] and the state after the last row, from the
 * state before the first (null: 0).  log_decay [heads] fp32, <= 0.  lengths as
 * for the window: rows from n on are not read and get o = 0, and the state is
 * the one after n rows.  state_out may be null, or the same as state_in. */
qds_status qds_decay_forward_workspace(const qds_decay_config* c, uint64_t* bytes);
qds_status qds_decay_forward(const qds_decay_config* c, qds_view q, qds_view k, qds_view v,
                             const float* log_decay, const float* state_in,
                             const int32_t* lengths, qds_view o, float* state_out,
                             void* workspace, uint64_t workspace_bytes, void* stream);

/* Gradients of q, k, v and of state_in (dstate_in; may be null) from do and
 * from the gradient of state_out (dstate_out; null: 0). */
qds_status qds_decay_backward_workspace(const qds_decay_config* c, uint64_t* bytes);
qds_status qds_decay_backward(const qds_decay_config* c, qds_view dout, qds_view q, qds_view k,
                              qds_view v, const float* log_decay, const float* state_in,
                              const float* dstate_out, const int32_t* lengths, qds_view dq,
                              qds_view dk, qds_view dv, float* dstate_in, void* workspace,
                              uint64_t workspace_bytes, void* stream);

/* One token; state_out may be the same as state_in.  q, k, v, o have no rows
 * (stride[1] unused). */
qds_status qds_decay_step(const qds_decay_config* c, qds_view q, qds_view k, qds_view v,
                          const float* log_decay, const float* state_in, qds_view o,
                          float* state_out, void* stream);

const char* qds_status_str(qds_status status);

#ifdef __cplusplus
}
#endif
#endif /* QD_SEQ_H */
