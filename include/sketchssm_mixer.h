/*
 * sketchssm_mixer.h -- C ABI of the operators around the recurrence of a
 * Mamba-2 mixer layer on MI355X (gfx950): the short causal convolution and the
 * selective scan of prompts, the single token that goes into the decode path's
 * replay buffer, root-mean-square norms that end in 8 bits, and products of
 * 8-bit matrices with block scales.  Same library, statuses, error texts and
 * conventions as sketchssm.h: device pointers owned by the caller and 16-byte
 * aligned, checks on the host before any launch, no allocation and no
 * synchronisation, every launch on `stream`.
 *
 * Packed sequences.  The tokens of a batch's prompts lie one sequence after
 * the other, T in all; sequence b is rows offsets[b] .. offsets[b+1]-1, with
 * offsets[0] = 0 and offsets[batch] = T, non-decreasing (device memory, int32;
 * an empty sequence is allowed).  The host cannot see the values: the kernels
 * hold every access inside the arrays whatever they are, and results are
 * unspecified where they break that rule.  NULL: sequences of T / batch tokens.
 *
 * Row strides (ld*) are in elements, multiples of 16 bytes, and at least the
 * row's length, so that the parts of a projection's output are read where they
 * lie.  "io" is skssm_dtype F32 or BF16.
 */
#ifndef SKETCHSSM_MIXER_H
#define SKETCHSSM_MIXER_H

#include "sketchssm.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SKSSM_E4M3 = 2 }; /* skssm_dtype of a norm's 8-bit output: OCP e4m3, largest value 448 */

/* A depthwise causal convolution over `channels` channels with `width` taps. */
typedef struct {
  int32_t channels; /* a multiple of 16 bytes of io                              */
  int32_t width;    /* 2..4                                                      */
  int32_t io_dtype; /* skssm_dtype of x, y and the states                        */
  int32_t silu;     /* 1: y = z sigmoid(z) of the sum z, 0: y = z                */
} skssm_conv_config;

/*
 * sketchssm_conv -- the convolution over packed prompts:
 *     y[t][c] = act(bias[c] + sum_j taps[c][j] x[t - (width-1) + j][c])
 * where positions before the sequence's first token are rows of its state:
 * state[b][width-1][channels], the width-1 inputs before it, oldest first.
 * state_in NULL: zeros.  state_out (NULL: not wanted) receives the last
 * width-1 inputs of state and sequence together, so an empty sequence keeps
 * its state; it may be state_in itself.  taps [channels][width] and bias
 * [channels] (may be NULL) are fp32; sums are fp32.  y may not overlap x or
 * the states, and neither y nor state_out taps, bias or offsets.
 */
int sketchssm_conv(const skssm_conv_config* cfg, int32_t batch, int64_t tokens, const int32_t* offsets, const void* x,
                   int64_t ldx, const float* taps, const float* bias, const void* state_in, void* state_out, void* y,
                   int64_t ldy, void* stream);

/*
 * sketchssm_conv_token -- one token of every request, from the projection's
 * output into slot n_buffered (0..window-1) of the replay buffer, ready for
 * sketchssm_decode / sketchssm_update of that slot (cfg as there, kind
 * SKSSM_MAMBA2).  x [batch][heads*dv + 2*groups*dk] holds the channels of x, B
 * and C in this order (row stride ldx); the convolution with `width` taps and
 * SiLU runs over all of them, its state [batch][width-1][channels] moves on by
 * one token in place.  Then
 *     ring.v slot = x of the head, ring.k slot = B and q = C of the head's group
 *     (heads / groups consecutive heads each),
 *     ring.beta = softplus(dt + dt_bias), ring.log_decay = beta A
 * with dt [batch][heads] (io, row stride lddt, aligned to its element only) and
 * dt_bias, A [heads] fp32 (dt_bias may be NULL).  No input but the state may overlap what is written.
 */
int sketchssm_conv_token(const skssm_config* cfg, int32_t groups, int32_t width, const void* x, int64_t ldx,
                         const float* taps, const float* bias, void* state, const void* dt, int64_t lddt,
                         const float* dt_bias, const float* A, const skssm_ring* ring, int32_t n_buffered, void* q,
                         void* stream);

/*
 * sketchssm_scan -- the selective scan of packed prompts.  Per sequence and head,
 *     dt_t = softplus(dt[t][h] + dt_bias[h]),   S_t = exp(dt_t A_h) S_{t-1} + dt_t x_t B_t^T,
 *     y_t = S_t C_t + D_h x_t
 * with x [T][heads*dv], b and c [T][groups*dk] (heads / groups consecutive heads
 * share a group), dt [T][heads] (aligned to its element only), all io;
 * dt_bias, A, D [heads] fp32 (dt_bias and D may be NULL; A <= 0).  cfg gives
 * batch, heads, dk, dv and io_dtype (kind SKSSM_MAMBA2; its rank is not used).
 * S_in (NULL: zero) and S_out are states in the tile-major layout of
 * sketchssm.h, S_out may be S_in; an empty sequence's state is passed on, so
 * sketchssm_update(q = NULL) can follow.  y [T][heads*dv] io, S_out and the
 * workspace may not overlap the inputs (but S_in).  The state and every sum are fp32; with bf16 io the products
 * inside a chunk of tokens take bf16 operands (the decayed scores and the state
 * as read by C_t are rounded to nearest), while what enters the state keeps 24 bits and D x_t
 * is fp32.
 * Row strides of x, b, c and y are less than 2^24.  A value that is not finite stays in its
 * head (x, dt) or group (b, c) and its sequence; within its chunk of 64 tokens it may
 * reach the outputs of tokens before it.
 *
 * workspace: sketchssm_scan_workspace bytes (may be 0), used where a sequence's
 * scan is split over workgroups; its contents need not be kept.
 */
int sketchssm_scan(const skssm_config* cfg, int32_t groups, int64_t tokens, const int32_t* offsets, const void* x,
                   int64_t ldx, const void* b, int64_t ldb, const void* c, int64_t ldc, const void* dt, int64_t lddt,
                   const float* dt_bias, const float* A, const float* D, const float* S_in, float* S_out, void* y,
                   int64_t ldy, void* workspace, size_t workspace_bytes, void* stream);
size_t sketchssm_scan_workspace(const skssm_config* cfg, int32_t groups, int64_t tokens);

/*
 * sketchssm_norm -- root-mean-square norm over groups of columns:
 *     u = x                       residual = gate = NULL
 *     u = x + residual            residual != NULL (residual_out, if given, receives u)
 *     u = (x + D skip) silu(gate) gate != NULL (skip optional: skip and D together)
 *     y = u / sqrt(mean of u^2 over its group + eps) * weight
 * rows x columns; `group` columns share a mean (a divisor of columns; `columns`
 * for an ordinary norm).  x is x_dtype (F32, or the io dtype); residual,
 * residual_out, gate and skip are io_dtype; weight [columns] fp32.  skip is
 * [rows][columns / skip_width] heads of skip_width columns, ld_skip apart between
 * rows and skip_head apart between heads (a slot of the replay buffer is read
 * where it lies), D [columns / skip_width] fp32.  Statistics are fp32, over the
 * unrounded u.
 * out_dtype F32 or BF16 (the io dtype), or SKSSM_E4M3: blocks of 128 columns
 * (the last may be shorter; `group` is then `columns` or a multiple of 128) are
 * stored over their scale, scales[block][row] = max(largest |y| / 448, 2^-64), rows
 * ld_scales apart -- what sketchssm_matmul_fp8 reads.  A NaN makes its block's scale NaN.
 * columns and skip_width are multiples of 8, group at most 32768.  residual_out may be x or residual
 * (same type and stride); out overlaps no input.
 */
typedef struct {
  int64_t rows;
  int32_t columns, group;
  int32_t x_dtype, io_dtype, out_dtype;
  int32_t skip_width;
  float eps;
  const void* x;
  int64_t ldx;
  const void* residual;
  int64_t ld_residual;
  void* residual_out;
  int64_t ld_residual_out;
  const void* gate;
  int64_t ld_gate;
  const void* skip;
  int64_t ld_skip, skip_head;
  const float* D;
  const float* weight;
  void* out;
  int64_t ld_out;
  float* scales;
  int64_t ld_scales;
} skssm_norm_args;
int sketchssm_norm(const skssm_norm_args* args, void* stream);

/*
 * sketchssm_matmul_fp8 -- y = a w^T of e4m3 matrices with block scales:
 *     y[m][n] = sum_kb a_scale[kb][m] w_scale[n / 128][kb] sum_{k in block kb} a[m][k] w[n][k]
 * a [M][K] (row stride lda), w [N][K] (row stride ldw), a_scale [ceil(K/128)][M] (rows
 * ld_ascale apart), w_scale [ceil(N/128)][ceil(K/128)] fp32; y [M][N] of
 * out_dtype F32 or BF16, row stride ldy (any, >= N).  K is a multiple of 16, lda and ldw are
 * less than 2^24.  Sums are fp32; for a BF16 output the 8-bit matrix instructions, which keep
 * 2^-11 of the largest product they add, for F32 those of 16 bits, which keep fp32's.
 * workspace: sketchssm_matmul_fp8_workspace bytes (may be 0), for products
 * whose K axis is split over workgroups; its contents need not be kept.
 */
int sketchssm_matmul_fp8(int64_t M, int32_t N, int32_t K, const void* a, int64_t lda, const float* a_scale,
                         int64_t ld_ascale, const void* w, int64_t ldw, const float* w_scale, int32_t out_dtype, void* y,
                         int64_t ldy, void* workspace, size_t workspace_bytes, void* stream);
size_t sketchssm_matmul_fp8_workspace(int64_t M, int32_t N, int32_t K);

#ifdef __cplusplus
}
#endif
#endif /* SKETCHSSM_MIXER_H */
