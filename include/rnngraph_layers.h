/*
 * rnngraph_layers -- layers that need no step loop, on tensors of the caller's own: linear
 * attention with a decay for each head (a recurrent layer whose state is a matrix), the residual
 * sum with dropout and root-mean-square norm, and dropout.  Networks have the same layers as node
 * kinds (RNN_NODE_ATTENTION, RNN_NODE_NORM, RNN_NODE_DROPOUT of rnngraph.h, in fp32); the functions
 * here take other types, strides and lengths too, and need no graph.
 *
 * Conventions
 *  - As in rnngraph.h: 0 or a negative rnn_status, rnn_last_error() for the message, "d_" pointers
 *    are DEVICE pointers of the caller's, work is queued on hip_stream (NULL = the default stream)
 *    of the current device, nothing throws.  The functions keep nothing between calls, allocate
 *    nothing, do not synchronise and can be captured into a HIP graph.
 *  - Where a function takes a workspace, rnn_*_workspace_bytes tells its size (0: none is needed
 *    and d_workspace may be NULL); 256-byte aligned.  Calls whose work may overlap need workspaces
 *    of their own: two streams, or two captured graphs that are replayed at the same time.
 *  - Frames x streams tensors are given as rnn_frames: element (t, n, h, i) lies at
 *    data[t * stride_t + n * stride_n + h * stride_h + i], strides in elements, of any sign and size.
 *    Inputs may overlap each other; an output may overlap nothing (where it begins at an input or another
 *    output the call is refused), and two of its elements may not share a place (strides with which neighbours along one or
 *    two axes do are refused).  Alignment: that of the element type.
 *  - Sums, statistics and states are fp32 whatever the type of the tensors, and what is stored is rounded once, to
 *    nearest.  Attention on RNN_BF16 tensors multiplies with the matrix instructions for bf16: the scores between frames of
 *    a chunk and, for outputs and gradients, the state that the chunk starts from go there in two bf16 numbers each, which
 *    lose at most 2^-16 of a term of the result's sum (the state that is handed on loses nothing by it).
 */
#ifndef RNNGRAPH_LAYERS_H
#define RNNGRAPH_LAYERS_H

#include "rnngraph.h"

#ifdef __cplusplus
extern "C" {
#endif

enum rnn_dtype { RNN_F32 = 0, RNN_BF16 = 1, RNN_F16 = 2 };

/* ---- linear attention with a decay for each head ------------------------------------------
 * Head h of stream n keeps a state S [dim_k][dim_v], and for every frame
 *     S(t) = exp(log_decay[h]) S(t - 1) + k(t) v(t)^T          o(t) = scale S(t)^T q(t)
 * that is o(t) = scale sum_{s <= t} exp((t - s) log_decay[h]) (q(t) . k(s)) v(s) + the part of
 * the state before the window.  Frames are worked on together, in chunks (Section 3.1's aim for
 * a recurrence that has no nonlinearity); few frames (up to 4; up to 8 of heads of less than 16 bytes) one after another.  An infinity or NaN in a
 * frame reaches what the formulas make of that frame, where an infinity may become NaN: outputs and dq of it
 * and later frames, dk and dv of it and earlier ones, of its stream and head.
 *   T, N        frames and streams; T = 0 and N = 0 are allowed
 *   heads       heads of q and o; kv_heads heads of k and v, heads = kv_heads * group: head h reads
 *               key / value head h / group
 *   dim_k, dim_v  1 .. 256 units of a head
 *   dtype       of q, k, v, o and their gradients: RNN_F32 or RNN_BF16
 * d_log_decay: float [heads], at most 0 (0: nothing is forgotten, -inf: everything; positive values
 * count as 0; a head whose decay is NaN has NaN wherever its state has passed a frame).  It has no gradient: the decays are constants of the layer.
 * d_lengths: int32 [N] or NULL.  Stream n has its first d_lengths[n] frames (values outside [0, T]
 * count as the nearer end); what lies behind them is not read, outputs there stay as they were.
 * d_state_in: float [N][heads][dim_k][dim_v] or NULL (zero).  d_state_out: the state after the
 * stream's last frame, or NULL; may be d_state_in. */
typedef struct { int32_t T, N, heads, kv_heads, dim_k, dim_v, dtype; float scale; } rnn_linear_attention_desc;
typedef struct { void* data; int64_t stride_t, stride_n, stride_h; } rnn_frames;

/* Bytes of workspace of the forward (backward = 0) or backward call; negative rnn_status on error. */
int64_t rnn_linear_attention_workspace_bytes(const rnn_linear_attention_desc* desc, int32_t backward);

/* o may be NULL: then only the state is advanced (q may be NULL too). */
int rnn_linear_attention_forward(const rnn_linear_attention_desc* desc, const rnn_frames* q, const rnn_frames* k,
                                 const rnn_frames* v, const float* d_log_decay, const int32_t* d_lengths,
                                 const float* d_state_in, float* d_state_out, const rnn_frames* o,
                                 void* d_workspace, int64_t ws_bytes, void* hip_stream);

/* Gradients from d_o = dE/do and d_dstate_out = dE/d state_out (float, or NULL: zero).  dq, dk, dv and
 * d_dstate_in (dE/d state_in, float) are overwritten; any of them may be NULL.  d_dstate_in may be neither
 * d_dstate_out nor, if dq is asked for, d_state_in.  dk and dv are sums over
 * the heads that share a key / value head, in a fixed order: same bits from call to call.  Frames behind
 * a stream's length stay as they were. */
int rnn_linear_attention_backward(const rnn_linear_attention_desc* desc, const rnn_frames* q, const rnn_frames* k,
                                  const rnn_frames* v, const float* d_log_decay, const int32_t* d_lengths,
                                  const float* d_state_in, const rnn_frames* d_o, const float* d_dstate_out,
                                  const rnn_frames* dq, const rnn_frames* dk, const rnn_frames* dv, float* d_dstate_in,
                                  void* d_workspace, int64_t ws_bytes, void* hip_stream);

/* ---- residual sum, dropout and root-mean-square norm ----------------------------------------
 * For every row of dim units
 *     h = residual + drop(x)        y = gain h / sqrt(mean(h^2) + eps)
 * Element (r, i) of a tensor lies at data[r * ld + i], ld >= dim; an output may be the input of the
 * same call that it replaces (h: residual or x; y: x or residual; dx and dresidual: dy, dh or h), with the same ld (another one is
 * refused, and so are two outputs in one place).
 *   rows >= 0, dim 1 .. 16384; dtype of x, residual, h, y: any of rnn_dtype
 *   dropout, seed, offset, d_offset: as in rnn_dropout; dropout = 0: none
 *   d_residual, d_gain (float [dim]) may be NULL: zero, one
 *   d_h may be NULL: the sum is not stored;  d_rstd: float [rows], 1 / sqrt(mean(h^2) + eps), or NULL
 * Statistics are taken from the sum before it is rounded to its type. */
typedef struct {
    int64_t rows;
    int32_t dim, dtype;
    float eps, dropout;
    uint64_t seed, offset;
    const uint64_t* d_offset;
} rnn_add_norm_desc;
int rnn_add_norm_forward(const rnn_add_norm_desc* desc, const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual,
                         const float* d_gain, void* d_h, int64_t ld_h, void* d_y, int64_t ld_y, float* d_rstd, void* hip_stream);

/* The same with y in 8 bits (e4m3: four exponent and three mantissa bits, largest value 448) and float scales: y = scale * y8.
 * A scale for every row (group = 0, d_scales [rows]) or for every 128 units of a row (group = 128, d_scales [rows][ceil(dim / 128)]):
 * the largest |y| / 448, or 1 where all are zero.  y8 may not be an input. */
int rnn_add_norm_e4m3(const rnn_add_norm_desc* desc, const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual,
                      const float* d_gain, void* d_h, int64_t ld_h, uint8_t* d_y8, int64_t ld_y8, float* d_scales, int32_t group,
                      float* d_rstd, void* hip_stream);

/* Gradients: d_dy = dE/dy, d_dh = dE/dh from what reads the sum besides the norm (or NULL: zero), d_h and d_rstd as the forward call
 * stored them.  With n = h rstd:  s = dh + rstd (gain dy - n mean(gain dy n)) is stored to d_dresidual, and drop(s) (the forward
 * call's mask again) to d_dx; dgain = sum over the rows of dy n, always in the same order.  Each may be NULL, dgain needs the
 * workspace.  Without dropout dx = dresidual: one of the two need not be stored. */
int64_t rnn_add_norm_workspace_bytes(const rnn_add_norm_desc* desc);
int rnn_add_norm_backward(const rnn_add_norm_desc* desc, const void* d_dy, int64_t ld_dy, const void* d_dh, int64_t ld_dh,
                          const void* d_h, int64_t ld_h, const float* d_rstd, const float* d_gain, void* d_dx, int64_t ld_dx,
                          void* d_dresidual, int64_t ld_dresidual, float* d_dgain, void* d_workspace, int64_t ws_bytes, void* hip_stream);

/* ---- dropout -----------------------------------------------------------------------------------
 * y = x / (1 - p) where an element is kept, 0 where it is dropped; the gradient is the same call on dy.  Nothing is stored: element
 * (r, i) takes the 16-bit number i % 8 (low half of a word first) of Philox4x32 with seven rounds (Salmon, Moraes, Dror, Shaw: "Parallel
 * random numbers: as easy as 1, 2, 3", 2011), counter { r * ceil(dim / 8) + i / 8, offset } as two 64-bit halves, key seed, and is
 * kept if that number is at least round(65536 p): p is taken in steps of 1 / 65536, and the factor is that p's.
 *   p in [0, 1] (1: all are dropped);  d_offset: DEVICE uint64 added to offset when the call runs, or NULL: a captured
 *   call draws other numbers in each replay if something advances it.
 * y may be x (with the same ld). */
typedef struct {
    int64_t rows;
    int32_t dim, dtype;
    float p;
    uint64_t seed, offset;
    const uint64_t* d_offset;
} rnn_dropout_desc;
int rnn_dropout(const rnn_dropout_desc* desc, const void* d_x, int64_t ld_x, void* d_y, int64_t ld_y, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RNNGRAPH_LAYERS_H */
