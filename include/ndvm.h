/*
 * ndvm.h -- C ABI of the NDVM tape-replay library (GB300, sm_103a).
 *
 * The library builds the realized numeric trace ("tape") of a program run by a
 * fixed evaluator and replays it on the GPU across a population of B parameter
 * lanes: a forward sweep over a lane-major value buffer, an exact reverse-mode
 * adjoint sweep back to per-lane parameter gradients, and the per-lane loss.
 *
 * Problem statement (paper section 2): a fixed evaluator E walks a program P given
 * as runtime data with numeric parameters theta, y = E(P, theta), and we want
 * dy/dtheta.  Section 3.4: the tape records one node per differentiable numeric
 * primitive of the realized trace and is replayed in reverse to accumulate
 * adjoints; section 3.5: one walk serves a batch axis of B lanes; Appendix C lists
 * the primitives and their adjoints.
 *
 * Conventions for every entry point:
 *   - No exception or C++ type crosses this boundary; every function returns an
 *     ndvm_status (or a plain value documented below).  On a non-OK status,
 *     ndvm_last_error() returns a message for the calling thread.
 *   - Pointers documented "device" are CUDA device pointers on the current device;
 *     "host" pointers are ordinary CPU memory.  The caller owns every buffer it
 *     passes; the library owns tapes and their cached device copies.
 *   - Argument errors are detected on the host and return a status before any
 *     launch.  Compute calls are asynchronous and ordered on the given CUDA stream
 *     (NULL = legacy default stream), except that the first call for a tape on a
 *     device uploads the tape synchronously (make that call before any stream
 *     capture).
 *   - Non-finite lane results are data, not errors.
 *   - dtype NDVM_F64 means every buffer holds double; NDVM_F32 means float.
 *   - The network operators at the end take no tape; their element types and layouts
 *     are stated there.
 */
#ifndef NDVM_H
#define NDVM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  NDVM_OK = 0,
  NDVM_E_INVALID_ARG = 1,  /* null pointer, bad size, too small a buffer */
  NDVM_E_PARSE = 2,        /* program text is not well formed */
  NDVM_E_UNSUPPORTED = 3,  /* well formed but outside the supported surface */
  NDVM_E_SHAPE = 4,        /* matrix shape mismatch in the program */
  NDVM_E_OOM = 5,          /* host or device allocation failed */
  NDVM_E_CUDA = 6,         /* a CUDA runtime call failed */
  NDVM_E_DEVICE_CHECK = 7  /* a device-side consistency check fired */
} ndvm_status;

typedef enum { NDVM_FE_SCHEME = 0, NDVM_FE_BYTECODE = 1 } ndvm_frontend;
/* NDVM_F16 and NDVM_BF16 are element types of the network operators alone; the replays take F64 and F32. */
typedef enum { NDVM_F64 = 0, NDVM_F32 = 1, NDVM_F16 = 2, NDVM_BF16 = 3 } ndvm_dtype;

typedef struct ndvm_tape ndvm_tape; /* opaque; immutable once built */

/*
 * ndvm_trace_build -- walk the program once on the host and record its tape
 * (sections 3.3-3.4: control is the exact realized trace; only numeric
 * primitives are recorded; structural work records nothing).
 *   program, len : program text (host); not NUL-terminated necessarily
 *   fe           : NDVM_FE_SCHEME (Scheme-style evaluator) or NDVM_FE_BYTECODE
 *                  (stack-bytecode VM, section 7's second client)
 *   out          : receives a new tape; free it with ndvm_tape_free
 * The tape is a deterministic function of the text: byte-identical across runs,
 * threads and hosts (constants are parsed correctly rounded and stored as bits).
 * Errors: NDVM_E_INVALID_ARG, NDVM_E_PARSE, NDVM_E_UNSUPPORTED, NDVM_E_SHAPE, NDVM_E_OOM.
 */
ndvm_status ndvm_trace_build(const char* program, size_t len, ndvm_frontend fe, ndvm_tape** out);

/*
 * ndvm_tape_info -- sizes of a tape (any output pointer may be NULL).
 *   n_nodes : tape nodes; n_params : P (parameters per lane);
 *   n_obs   : observations the program reads (the obs buffer must hold at least this many);
 *   n_slots : per-lane value/adjoint slots of the gradient replay plan;
 *   hash    : FNV-1a 64 of the serialized tape.
 */
ndvm_status ndvm_tape_info(const ndvm_tape* tape, int64_t* n_nodes, int32_t* n_params, int64_t* n_obs,
                           int64_t* n_slots, uint64_t* hash);

/*
 * ndvm_tape_serialize -- write the tape's canonical byte form into buf (host).
 * *len receives the full size; if cap < size nothing is written and
 * NDVM_E_INVALID_ARG is returned (call with buf = NULL, cap = 0 to query).
 */
ndvm_status ndvm_tape_serialize(const ndvm_tape* tape, void* buf, size_t cap, size_t* len);

/* ndvm_tape_free -- release a tape and its device copies (NULL is ignored). */
void ndvm_tape_free(ndvm_tape* tape);

/*
 * ndvm_workspace_bytes -- device workspace needed by ndvm_value_and_grad to run all
 * B lanes in one launch (forward intermediates that the reverse sweep reads, stored
 * lane-contiguous).  A smaller workspace is accepted: lanes then run in chunks
 * sized to fit; 0 is returned when the tape needs no workspace.
 */
size_t ndvm_workspace_bytes(const ndvm_tape* tape, int64_t B, ndvm_dtype dtype);

/*
 * ndvm_forward -- per-lane loss only (no reverse sweep, no workspace).
 *   B      : lanes (0 is allowed and does nothing)
 *   params : device, B x P row-major (lane b's parameters at params[b*P .. b*P+P-1])
 *   obs    : device, n_obs values shared by every lane (may be NULL if the tape reads none)
 *   n_obs  : length of obs; must be >= the tape's n_obs
 *   loss   : device, B outputs
 *   stream : cudaStream_t or NULL
 */
ndvm_status ndvm_forward(const ndvm_tape* tape, ndvm_dtype dtype, int64_t B, const void* params,
                         const void* obs, int64_t n_obs, void* loss, void* stream);

/*
 * ndvm_value_and_grad -- per-lane loss and exact gradient along the realized trace
 * (Property 1, section 4; Appendix C adjoints).  Arguments as ndvm_forward, plus
 *   grad      : device, B x P row-major outputs
 *   workspace : device scratch of ws_bytes bytes (may be NULL when ws_bytes = 0);
 *               contents are overwritten; it must not be used concurrently by
 *               another call.
 * Returns NDVM_E_INVALID_ARG if the tape needs workspace and ws_bytes cannot hold
 * even one block of lanes.
 */
ndvm_status ndvm_value_and_grad(const ndvm_tape* tape, ndvm_dtype dtype, int64_t B, const void* params,
                                const void* obs, int64_t n_obs, void* loss, void* grad, void* workspace,
                                size_t ws_bytes, void* stream);

/*
 * ndvm_workspace_bytes_multi -- device workspace that ndvm_value_and_grad_multi needs
 * for the batch (tapes[k] with B[k] lanes): per tape, its shared per-point values and
 * all of its lanes' saved forward values, each tape's region 256-byte aligned.  0 when
 * the batch needs none (or an argument is invalid).
 */
size_t ndvm_workspace_bytes_multi(const ndvm_tape* const* tapes, int32_t n_tapes, const int64_t* B,
                                  ndvm_dtype dtype);

/*
 * ndvm_value_and_grad_multi -- ndvm_value_and_grad for a batch of tapes in as few
 * launches as possible (the optional multi-tape extension of the boundary; the paper's
 * setting of many candidate programs evaluated together, sections 5-6).  Tape k replays
 * B[k] lanes with its own params[k] (device, B[k] x P_k), obs[k] (device, n_obs[k]
 * values), loss[k] (device, B[k]) and grad[k] (device, B[k] x P_k); the results are
 * those of n_tapes separate ndvm_value_and_grad calls.  Replays of the same kernel
 * variant, block size and threads per lane share one launch (up to 240 tapes each)
 * while they have the same occupancy or the launch stays small; a batch with shared
 * per-point values adds launches of derive plans in front and, for tapes on the
 * general kernel, one of observation copies.
 *   tapes, B, params, obs, n_obs, loss, grad : host arrays of n_tapes entries
 *   workspace : device, 256-byte aligned, at least ndvm_workspace_bytes_multi bytes
 *               (NULL if that is 0); overwritten; not to be shared with a concurrent call
 * Tapes with B[k] = 0 are skipped.  Returns NDVM_E_INVALID_ARG before any launch when an
 * entry is invalid (the message names the tape) or the workspace is too small; the
 * first call for a tape uploads it synchronously, as for ndvm_value_and_grad.
 */
ndvm_status ndvm_value_and_grad_multi(const ndvm_tape* const* tapes, int32_t n_tapes, ndvm_dtype dtype,
                                      const int64_t* B, const void* const* params, const void* const* obs,
                                      const int64_t* n_obs, void* const* loss, void* const* grad, void* workspace,
                                      size_t ws_bytes, void* stream);

/*
 * ndvm_value_and_grad_host -- the same computation through host buffers: copies
 * params and obs to the device, runs ndvm_value_and_grad, copies loss and grad
 * back, and synchronizes the stream.  Device buffers are cached per tape and
 * reused across calls.
 *   params, obs, loss, grad : host pointers (grad may be NULL for value only)
 */
ndvm_status ndvm_value_and_grad_host(const ndvm_tape* tape, ndvm_dtype dtype, int64_t B, const void* params,
                                     const void* obs, int64_t n_obs, void* loss, void* grad, void* stream);

/*
 * ndvm_value_and_grad_host_async -- ndvm_value_and_grad_host without the final
 * synchronization: the copies and the replay are queued on `stream` and the call
 * returns.  loss and grad hold the results once the caller has synchronized the
 * stream; params and obs must stay unchanged until then.  Host buffers should be
 * page-locked (cudaHostAlloc / pinned), else the copies are not asynchronous.
 * The tape's cached device buffers are shared by its calls, so two calls on the
 * same tape must be ordered (same stream, or a synchronization between them);
 * calls on different tapes may overlap on different streams.  The paper has no
 * counterpart; it lets a host-driven population of programs overlap its copies
 * and replays.
 */
ndvm_status ndvm_value_and_grad_host_async(const ndvm_tape* tape, ndvm_dtype dtype, int64_t B, const void* params,
                                           const void* obs, int64_t n_obs, void* loss, void* grad, void* stream);

/*
 * ndvm_value_and_grad_noalloc -- ndvm_value_and_grad for callers that may not
 * allocate device memory while they run (their device memory is planned up front
 * and must not grow).  The paper has no counterpart; this is a deployment variant.
 * Arguments as ndvm_value_and_grad, without a workspace: the forward values that
 * the reverse sweep reads go to a fixed scratch array of 32 MiB inside the
 * library, held by every GPU that loads the library until the process exits.
 * The call allocates nothing: it makes no cudaMalloc, cudaFree or other allocating
 * call.  Therefore:
 *   - the tape must already be resident on the current device: one earlier
 *     ndvm_forward or ndvm_value_and_grad call for this tape uploads it (that
 *     call allocates); otherwise NDVM_E_INVALID_ARG;
 *   - the first call on a device looks up the scratch array's device address
 *     (once per device); make that first call before any stream capture;
 *   - lanes run in chunks that fit the scratch; a tape whose workspace for one
 *     block of lanes exceeds 32 MiB is rejected with NDVM_E_INVALID_ARG;
 *   - every call shares the one array, so calls whose work overlaps on the GPU
 *     race; nothing in the array needs clearing (each saved value is written
 *     before it is read).
 */
ndvm_status ndvm_value_and_grad_noalloc(const ndvm_tape* tape, ndvm_dtype dtype, int64_t B, const void* params,
                                        const void* obs, int64_t n_obs, void* loss, void* grad, void* stream);

/*
 * ndvm_check_device -- synchronize and report whether any kernel of this tape
 * on the current device recorded a consistency failure (NDVM_E_DEVICE_CHECK);
 * clears the flag.
 */
ndvm_status ndvm_check_device(const ndvm_tape* tape);

/*
 * ndvm_tape_cost -- algorithmic cost of one lane's value-and-gradient replay (any
 * output may be NULL): FP64 work of the forward and reverse sweeps in
 * DFMA-equivalents, workspace elements per lane, and flags (bit 0: the tape has
 * data-axis regions; bit 1: the reverse sweep reads the workspace).
 */
ndvm_status ndvm_tape_cost(const ndvm_tape* tape, double* work_fwd, double* work_rev, int64_t* save_elems,
                           int32_t* flags);

/*
 * ndvm_tape_shared_work -- FP64 work (DFMA-equivalents) per value-and-gradient call
 * that does not scale with the lanes: the shared per-point values of data-axis regions
 * (section 3.5: values that depend on the data point but on no parameter are the same
 * on every lane, so they are computed once per call).  0 when there are none.
 */
ndvm_status ndvm_tape_shared_work(const ndvm_tape* tape, double* work_per_call);

/*
 * ndvm_measure_fp64_peak -- measure the device's FP64 fused multiply-add rate
 * (flop/s, two per FMA) with a dependent-chain microbenchmark on all SMs.  On GB300
 * a saturated DFMA stream issues one warp instruction per 19 cycles per SM, 84 % of
 * the FP64 pipe's unit-count peak (2 per clock per SM); the benchmark reports it
 * beside that peak.  The paper has no counterpart.  Synchronous.
 */
ndvm_status ndvm_measure_fp64_peak(double* flops_per_s, void* stream);

/* Functions that ndvm_measure_op_cost times (the replay's own exp, log, sin, cos and
 * sincos; CUDA's other functions, and CUDA's log, exp, sin and sincos for comparison;
 * DFMA as the unit). */
enum {
  NDVM_PROBE_DFMA = 0, NDVM_PROBE_EXP = 1, NDVM_PROBE_LOG = 2, NDVM_PROBE_SIN = 3, NDVM_PROBE_COS = 4,
  NDVM_PROBE_SINCOS = 5, NDVM_PROBE_TANH = 6, NDVM_PROBE_SQRT = 7, NDVM_PROBE_DIV = 8, NDVM_PROBE_RCP = 9,
  NDVM_PROBE_POW = 10, NDVM_PROBE_LOGLIB = 11, NDVM_PROBE_EXPLIB = 12, NDVM_PROBE_SINLIB = 13,
  NDVM_PROBE_SINCOSLIB = 14, NDVM_PROBE_COUNT = 15
};

/*
 * ndvm_measure_op_cost -- device time per call (ns, every SM busy with four
 * independent chains per thread, 1024 threads per SM) of the function `fn`
 * (NDVM_PROBE_*), each call followed by one FP64 add.  Dividing by the DFMA probe's
 * time gives the function's throughput cost in DFMA-equivalents; an ncu capture of
 * the probe launch gives its FP64-pipe instructions per call (calls = 4 x iters x
 * threads).  The paper has no counterpart: it measures the denominators of the
 * roofline.  Synchronous; NDVM_E_INVALID_ARG for an unknown fn or iters < 1.
 */
ndvm_status ndvm_measure_op_cost(int fn, int iters, double* ns_per_call, void* stream);

/*
 * Network operators: the parts of a residual block whose output is the lanes' parameters (the
 * paper's section 2 makes the evaluator an operator that gradients pass through, so what proposes
 * theta can be trained through a replay; the paper names no operator of that network).
 *   - A matrix argument is `rows` rows of contiguous elements, `*_stride` elements from one row to
 *     the next (at least a row's length, or 0 for an input whose rows are all the same memory).
 *     Pointers are aligned to their element type; other alignments only cost speed.
 *   - Everything is computed in binary32 and rounded to the output's type once, except where said.
 *   - Sums are added up in an order that depends on the sizes, strides and alignment alone: the same
 *     call gives the same bits again.
 *   - The first call of an operator on a device loads its kernels: make it before any stream capture.
 *   - Errors: NDVM_E_INVALID_ARG for null pointers, sizes, strides, alignment or a workspace that
 *     is too small; NDVM_E_UNSUPPORTED for a type the operator does not take.  Outputs may not
 *     overlap inputs, except ndvm_dropout's y, which may be x or residual itself (address and stride).
 */

/*
 * ndvm_layer_norm_forward -- y = (x - mean) * rstd * weight + bias over each row of `cols` elements,
 * mean and variance (of the differences, not of the squares) over the row, rstd = 1 / sqrt(variance + eps).
 *   dtype  : x and y (F32, F16, BF16);  wtype : weight and bias, dtype or F32
 *   rows   : 0 is allowed and does nothing, below 2^31;  cols : at least 1
 *   weight, bias : device, cols values, or NULL for 1 and 0
 *   eps    : not negative, finite
 *   stats  : device, 2 x rows floats for the backward pass (all means, then all rstd), or NULL
 */
ndvm_status ndvm_layer_norm_forward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* x,
                                    int64_t x_stride, const void* weight, const void* bias, double eps, void* y,
                                    int64_t y_stride, float* stats, void* stream);

/* ndvm_layer_norm_workspace_bytes -- device workspace that ndvm_layer_norm_backward needs for dweight or dbias. */
size_t ndvm_layer_norm_workspace_bytes(int64_t rows, int64_t cols);

/*
 * ndvm_layer_norm_backward -- gradients of ndvm_layer_norm_forward under the cotangent dy.
 *   x, weight, stats : as the forward pass had and wrote them
 *   dx, dweight, dbias : outputs (dweight and dbias of wtype, cols values), each NULL if not wanted;
 *                        rows = 0 sets dweight and dbias to 0
 *   workspace : device, 16-byte aligned; may be NULL when dweight and dbias are
 */
ndvm_status ndvm_layer_norm_backward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* dy,
                                     int64_t dy_stride, const void* x, int64_t x_stride, const void* weight,
                                     const float* stats, void* dx, int64_t dx_stride, void* dweight, void* dbias,
                                     void* workspace, size_t ws_bytes, void* stream);

/*
 * ndvm_dropout -- y = residual + (kept ? x / (1 - p) : 0); element i (row-major index, whatever the
 * strides) is kept if word offset + i of the generator's sequence is at least round(p 2^32), so nothing
 * is stored for the backward pass: that is the same call on the cotangent with the same p, seed and
 * offset and no residual.  The sequence: Philox4x32, 10 rounds (Salmon, Moraes, Dror, Shaw, 2011), word
 * w being word w % 4 of the block of counter (w / 4 as 64 bits, 0, 0) under the key `seed`.
 *   dtype    : x, residual and y (F32, F16, BF16)
 *   residual : device, or NULL for none (a dropped x contributes an exact 0, also where it is not finite)
 *   p        : 0 <= p <= 1 - 2^-32
 *   offset   : a multiple of 4; calls of one seed draw apart where their [offset, offset + rows * cols) are
 */
ndvm_status ndvm_dropout(ndvm_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                         const void* residual, int64_t r_stride, double p, uint64_t seed, uint64_t offset, void* y,
                         int64_t y_stride, void* stream);

/* NDVM_ACT_NONE (act(z) = z) is for the dense layers alone. */
typedef enum { NDVM_ACT_SILU = 0, NDVM_ACT_GELU = 1, NDVM_ACT_RELU = 2, NDVM_ACT_SIGMOID = 3, NDVM_ACT_NONE = 4 } ndvm_activation;

/*
 * ndvm_gated_forward -- h = act(x Wg^T) * (x Wu^T), both products, the activation and the product in
 * one kernel: x is rows x k, w_gate and w_up are n x k, h is rows x n.
 *   dtype : every matrix (F16, BF16; sums in binary32)
 *   act   : silu g / (1 + e^-g), gelu g (1 + erf(g / sqrt 2)) / 2, relu, or sigmoid
 *   rows  : 0 is allowed and does nothing;  k, n : at least 1; rows, k and n at most 2^28
 *   workspace : device, 256-byte aligned, ndvm_gated_workspace_bytes(..., 0, ...) bytes (NULL if that is 0)
 */
ndvm_status ndvm_gated_forward(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n, const void* x,
                               int64_t x_stride, const void* w_gate, int64_t g_stride, const void* w_up,
                               int64_t u_stride, void* h, int64_t h_stride, void* workspace, size_t ws_bytes,
                               void* stream);

/*
 * ndvm_gated_workspace_bytes -- device workspace of a forward (backward = 0) or backward (1) call.
 * aligned = 1: x, w_gate, w_up (and dh) start on 16 bytes and their row strides are multiples of 8 elements
 * and not 0; otherwise 0, which adds room for copies that are.  0 on invalid sizes.
 */
size_t ndvm_gated_workspace_bytes(int64_t rows, int64_t k, int64_t n, int backward, int aligned);

/*
 * ndvm_gated_backward -- gradients of ndvm_gated_forward under the cotangent dh (rows x n).  The two
 * products are computed again; dG and dU are rounded to dtype before the products that make dx (rows x k)
 * and dw_gate, dw_up (n x k, contiguous), or, where there are few of them (rows * min(n, k) up to 16384 or
 * n * k up to 2048), split into two halves of dtype that together lose next to nothing.  In F16 they are
 * infinite beyond 65504 and lose digits below 6e-5, as a stored half does (scale dh accordingly).  Each output may be
 * NULL if not wanted; rows = 0 sets dw_gate and dw_up to 0.
 */
ndvm_status ndvm_gated_backward(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                const void* dh, int64_t dh_stride, const void* x, int64_t x_stride, const void* w_gate,
                                int64_t g_stride, const void* w_up, int64_t u_stride, void* dx, int64_t dx_stride,
                                void* dw_gate, void* dw_up, void* workspace, size_t ws_bytes, void* stream);

/*
 * ndvm_gated_forward_keep, ndvm_gated_backward_kept -- the same pair with the pre-activations G = x Wg^T and
 * U = x Wu^T kept in between instead of computed again.
 *   kept : device, 16-byte aligned floats, 2 x rows rows (G's, then U's) of ndvm_gated_kept_stride(n), written by
 *          the one and read by the other; NULL: nothing is kept, as above
 * Keeping costs 8 bytes an element of h and saves a third of the backward pass's operations: it pays from about
 * k = 1536 on, and where h has up to about 2^21 elements.
 */
int64_t ndvm_gated_kept_stride(int64_t n);
ndvm_status ndvm_gated_forward_keep(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                    const void* x, int64_t x_stride, const void* w_gate, int64_t g_stride,
                                    const void* w_up, int64_t u_stride, void* h, int64_t h_stride, float* kept,
                                    void* workspace, size_t ws_bytes, void* stream);
ndvm_status ndvm_gated_backward_kept(ndvm_dtype dtype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                     const void* dh, int64_t dh_stride, const void* x, int64_t x_stride,
                                     const void* w_gate, int64_t g_stride, const void* w_up, int64_t u_stride,
                                     const float* kept, void* dx, int64_t dx_stride, void* dw_gate, void* dw_up,
                                     void* workspace, size_t ws_bytes, void* stream);

/*
 * ndvm_rms_norm_forward -- y = s * rstd * weight over each row of `cols` elements, s = x + residual rounded to
 * dtype (x where residual is NULL), rstd = 1 / sqrt(mean(s^2) + eps).
 *   dtype  : x, residual, y and sum (F32, F16, BF16);  wtype : weight, dtype or F32
 *   rows   : 0 is allowed and does nothing, below 2^31 - 128;  cols : at least 1
 *   weight : device, cols values, or NULL for 1
 *   sum    : receives s (it may be x or residual; y may be either where sum is not), or NULL; only with a residual
 *   rstd   : device, rows floats for the backward pass, or NULL
 */
ndvm_status ndvm_rms_norm_forward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* x,
                                  int64_t x_stride, const void* residual, int64_t r_stride, const void* weight, double eps,
                                  void* y, int64_t y_stride, void* sum, int64_t sum_stride, float* rstd, void* stream);

/* ndvm_rms_norm_workspace_bytes -- device workspace that ndvm_rms_norm_backward needs for dweight. */
size_t ndvm_rms_norm_workspace_bytes(int64_t rows, int64_t cols);

/*
 * ndvm_rms_norm_backward -- gradients of ndvm_rms_norm_forward under the cotangents dy and dsum (NULL: 0).
 *   s, weight, rstd : as the forward pass had and wrote them (s: its sum, or x)
 *   dx      : the gradient of x and of the residual;  dweight : of wtype; each NULL if not wanted; rows = 0 sets dweight to 0
 *   workspace : device, 16-byte aligned; may be NULL when dweight is
 */
ndvm_status ndvm_rms_norm_backward(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* dy,
                                   int64_t dy_stride, const void* dsum, int64_t dsum_stride, const void* s, int64_t s_stride,
                                   const void* weight, const float* rstd, void* dx, int64_t dx_stride, void* dweight,
                                   void* workspace, size_t ws_bytes, void* stream);

/*
 * 8-bit blocks -- 32 consecutive elements of a row (the last block may be shorter) share a scale 2^e, the least from
 * e = -127 on with which none is over 448 in size; an element is the nearest e4m3 value to v / 2^e, ties to even.  A block
 * with an infinity or a NaN is NaN throughout.
 *   values : device, 16-byte aligned, a byte an element; row stride a multiple of 16 that holds a row.  Bytes of a row
 *            behind its last element, up to a multiple of 16, are written as 0.
 *   scales : device, 16-byte aligned, ndvm_quantized_scale_bytes: e + 127 (255: NaN) as bytes
 *            [row / 128][column / 128][row % 32][row / 32 % 4][column / 32 % 4]; those of no block are written as 0, and
 *            are not read.
 *
 * ndvm_quantize makes them of rows (F32, F16, BF16).  ndvm_dequantize writes what they stand for, rounded to dtype; what
 * rounding lifts beyond dtype's largest finite value becomes that value.  ndvm_rms_norm_quantized makes them of
 * ndvm_rms_norm_forward's y, which is not rounded in between.
 */
size_t ndvm_quantized_scale_bytes(int64_t rows, int64_t cols);
ndvm_status ndvm_quantize(ndvm_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, uint8_t* values,
                          int64_t v_stride, uint8_t* scales, void* stream);
ndvm_status ndvm_dequantize(ndvm_dtype dtype, int64_t rows, int64_t cols, const uint8_t* values, int64_t v_stride,
                            const uint8_t* scales, void* x, int64_t x_stride, void* stream);
ndvm_status ndvm_rms_norm_quantized(ndvm_dtype dtype, ndvm_dtype wtype, int64_t rows, int64_t cols, const void* x,
                                    int64_t x_stride, const void* residual, int64_t r_stride, const void* weight, double eps,
                                    uint8_t* values, int64_t v_stride, uint8_t* scales, void* sum, int64_t sum_stride,
                                    void* stream);

/*
 * ndvm_linear_forward -- y = act(z) + residual with z = x w^T + bias, in one kernel (two where a long contraction is
 * split): x is rows x k, w is n x k, y and residual are rows x n.
 *   dtype    : every matrix (F16, BF16; sums in binary32, which tensor cores cut off where others round: z is off towards 0 by
 *              some 1e-9 k of its size, so one that close to relu's 0 or to an 8-bit step may fall on its other side);
 *              btype : bias, dtype or F32
 *   act      : as the gated projection's, or NDVM_ACT_NONE
 *   rows     : 0 is allowed and does nothing;  k, n : at least 1; rows, k and n at most 2^28
 *   bias     : device, n values, or NULL;  residual : or NULL; y may be residual
 *   z        : receives z for the backward pass, which needs it if act is not NDVM_ACT_NONE: device, 16-byte aligned floats,
 *              rows rows of ndvm_linear_kept_stride(n); or z_values and z_scales: z as 8-bit blocks whose row stride is n
 *              up to a multiple of 16 (scales of no block are left as they are); or all NULL
 *   workspace : device, 256-byte aligned, ndvm_linear_workspace_bytes bytes (NULL if that is 0)
 */
int64_t ndvm_linear_kept_stride(int64_t n);
ndvm_status ndvm_linear_forward(ndvm_dtype dtype, ndvm_dtype btype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                const void* x, int64_t x_stride, const void* w, int64_t w_stride, const void* bias,
                                const void* residual, int64_t r_stride, void* y, int64_t y_stride, float* z,
                                uint8_t* z_values, uint8_t* z_scales, void* workspace, size_t ws_bytes, void* stream);

/*
 * ndvm_linear_workspace_bytes -- device workspace of a forward (backward = 0) or backward (1) call.  aligned = 1: x, w (and
 * dy) start on 16 bytes and their row strides are multiples of 8 elements that hold a row; otherwise 0, which adds room
 * for copies that are.  held = 1: the backward call has x as 8-bit blocks.  0 on invalid sizes.  A forward call of one row
 * that keeps no z_values needs none, whatever this says for its sizes.
 */
size_t ndvm_linear_workspace_bytes(ndvm_activation act, int64_t rows, int64_t k, int64_t n, int backward, int aligned, int held);

/*
 * ndvm_linear_backward -- gradients of ndvm_linear_forward under the cotangent dy (which is the residual's gradient).
 * dz = dy act'(z) is rounded to dtype before the products that make dx (rows x k) and dw (n x k, contiguous), or, where there
 * are few elements (rows * min(n, k) up to 16384 or n * k up to 2048), split into two halves of dtype that together lose next
 * to nothing; dbias (btype) sums it unrounded.  In F16 dz is infinite beyond 65504 and loses digits below 6e-5.
 *   x        : as the forward call had it, or NULL and x_values, x_scales: as 8-bit blocks, rounded to dtype (neither is read
 *              without dw);  w is not read without dx
 *   z, z_values, z_scales : as the forward call wrote them
 *   dx, dw, dbias : each NULL if not wanted; rows = 0 sets dw and dbias to 0
 */
ndvm_status ndvm_linear_backward(ndvm_dtype dtype, ndvm_dtype btype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                 const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const uint8_t* x_values,
                                 int64_t xv_stride, const uint8_t* x_scales, const void* w, int64_t w_stride, const float* z,
                                 const uint8_t* z_values, const uint8_t* z_scales, void* dx, int64_t dx_stride, void* dw,
                                 void* dbias, void* workspace, size_t ws_bytes, void* stream);

/*
 * ndvm_linear_quantized -- ndvm_linear_forward of x and w in 8-bit blocks (dtype: y and residual, F16 or BF16): the products
 * of what the blocks stand for, sums in binary32.
 */
size_t ndvm_linear_quantized_workspace_bytes(int64_t rows, int64_t k, int64_t n);
ndvm_status ndvm_linear_quantized(ndvm_dtype dtype, ndvm_dtype btype, ndvm_activation act, int64_t rows, int64_t k, int64_t n,
                                  const uint8_t* x_values, int64_t xv_stride, const uint8_t* x_scales,
                                  const uint8_t* w_values, int64_t wv_stride, const uint8_t* w_scales, const void* bias,
                                  const void* residual, int64_t r_stride, void* y, int64_t y_stride, void* workspace,
                                  size_t ws_bytes, void* stream);

/*
 * ndvm_check_operators -- synchronize and report whether a kernel of the network operators gave up a wait on
 * the current device since the last check (NDVM_E_DEVICE_CHECK: its outputs are not valid); clears the flag.
 */
ndvm_status ndvm_check_operators(void);

/* ndvm_launch_count -- replay kernels launched by this process so far. */
unsigned long long ndvm_launch_count(void);

/* ndvm_last_error -- message for the last non-OK status on this thread ("" if none). */
const char* ndvm_last_error(void);

/* ndvm_version -- library version string. */
const char* ndvm_version(void);

#ifdef __cplusplus
}
#endif

#endif /* NDVM_H */
