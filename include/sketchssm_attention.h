/*
 * sketchssm_attention.h -- C ABI of the operators of a softmax attention layer
 * between the linear-attention layers of a hybrid model, on MI355X (gfx950):
 * rotary positions, a paged cache of keys and values in 4 bits with its append
 * and read, and attention over it for prompts and single tokens.  Same library, statuses,
 * error texts and conventions as sketchssm.h and sketchssm_mixer.h: device
 * pointers owned by the caller and 16-byte aligned, checks on the host before
 * any launch, no allocation and no synchronisation, every launch on `stream`,
 * nothing kept between calls.  "io" is skssm_dtype F32 or BF16.
 *
 * Heads.  x [tokens][heads][dim] arrays have a token stride (ld*) and a head
 * stride (*_head) in elements, both multiples of 16 bytes and at least what
 * they step over, so that the parts of a projection's output are read where
 * they lie.  An array that is written may share no byte with one that is read
 * but where it is named as the same; it may lie between its rows.
 */
#ifndef SKETCHSSM_ATTENTION_H
#define SKETCHSSM_ATTENTION_H

#include "sketchssm_mixer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The cache: `pages` pages of `page` tokens (a power of two, 16..1024) for
 * kv_heads heads of dim channels (64, 96, 128, 192 or 256) --
 *     data [pages][kv_heads][page / 16][17 dim] bytes (sketchssm_cache_bytes).
 * A value is a 4-bit number (e2m1: sign, 0 .5 1 1.5 2 3 4 6) times a power of
 * two that 32 consecutive channels of a token and head share: the smallest 2^e, e >= -64, with
 * the largest magnitude <= 7 2^e, so that no value is off by more than half the
 * distance of the two numbers around it, or 2^e past 6 2^e.  Rounding is to nearest, ties
 * to the even code.  A block with a value that is not finite or past 7 2^124
 * reads as NaN.  A record of 16 tokens holds
 *     keys      [16][dim / 2]                  channel 2 i in the low half of byte i
 *     values    [4][16][dim / 32][4]           token 4 a + d of the record, byte c of block g at [a][c][g][d]:
 *                                              channel 32 g + c in its low half, 32 g + c + 16 above
 *     exponents [16][dim / 32] of the keys (e + 127; 255: NaN), then of the values
 * A page is contiguous, so that a page is moved or shared by one copy.
 */
typedef struct {
  void* data;
  int32_t pages, kv_heads, page, dim;
} skssm_cache;
size_t sketchssm_cache_bytes(const skssm_cache* cache); /* 0: not a cache (sketchssm_last_error) */

/*
 * A batch's new tokens.  They lie packed, T = `tokens` in all, sequence b's at rows
 * offsets[b] .. offsets[b+1]-1 (as in sketchssm_mixer.h; NULL: T / batch each).
 * lengths [batch]: tokens of the sequence with the new ones, so that its i-th of n new
 * tokens has the place lengths[b] - n + i; a token at a place below 0 is a
 * padding row: it is not appended and its attention is 0.  table [batch][columns] (rows ld_table
 * apart): the page that holds places page j .. page (j + 1) - 1 of sequence b at [b][j]; entries that lengths do not reach may
 * hold anything.  All int32, on the device.  A place whose page
 * is not in 0..pages-1 or past `columns` is not written by the append and reads as NaN.
 */
typedef struct {
  int64_t tokens;
  const int32_t* offsets;
  const int32_t* lengths;
  const int32_t* table;
  int64_t ld_table;
  int32_t batch, columns;
} skssm_new_tokens;

/*
 * The rotation: angles [places][rotated] fp32, row p the cosines of place p's
 * rotated / 2 angles and then their sines (times any factor a scaled rotation
 * has).  Channels c < rotated (even, at most dim) of a head turn in pairs,
 *     y_a = x_a cos - x_b sin,  y_b = x_b cos + x_a sin,
 * in fp32 with each product and sum rounded: (a, b) = (i, i + rotated / 2), or
 * (2 i, 2 i + 1) if interleaved.  Other channels are copied.  A place outside 0..places-1
 * turns into NaN.
 */
typedef struct {
  const float* angles;      /* NULL: nothing is rotated */
  const int32_t* positions; /* [T] row of each token; NULL: its place in its sequence (append), t (sketchssm_rotary) */
  int32_t places, rotated, interleaved;
} skssm_rotation;

/* sketchssm_rotary -- y = x rotated, x and y [T][heads][dim] io (dim a multiple of 8, up to 512).  y may be x (with its strides). */
int sketchssm_rotary(int32_t io_dtype, int64_t tokens, int32_t heads, int32_t dim, const skssm_rotation* rotation,
                     const void* x, int64_t ldx, int64_t x_head, void* y, int64_t ldy, int64_t y_head, void* stream);

/*
 * sketchssm_cache_append -- the new tokens' keys, rotated, and values into the
 * cache; rotates their queries in the same launch where q is given (q_out may be q).
 * k, v [T][kv_heads][dim], q [T][heads][dim] io.  Keys are rounded to 4 bits
 * from fp32.  A page that is written is one sequence's, and stands in its row of the table once.
 */
typedef struct {
  int32_t io_dtype, heads;
  const void* k;
  int64_t ldk, k_head;
  const void* v;
  int64_t ldv, v_head;
  const void* q;
  int64_t ldq, q_head;
  void* q_out;
  int64_t ld_qout, qout_head;
} skssm_append_args;
int sketchssm_cache_append(const skssm_cache* cache, const skssm_new_tokens* seq, const skssm_rotation* rotation,
                           const skssm_append_args* args, void* stream);

/* sketchssm_cache_read -- the values that the cache holds for the new tokens, k and v [T][kv_heads][dim] io,
 * contiguous (either may be NULL).  bf16 holds them exactly.  Padding rows are 0. */
int sketchssm_cache_read(const skssm_cache* cache, const skssm_new_tokens* seq, int32_t io_dtype, void* k, void* v,
                         void* stream);

/*
 * sketchssm_attention -- the new tokens' attention over the cache: with p the place of
 * token t of sequence b and g = h / (heads / kv_heads),
 *     out[t][h] = sum_{j <= p} softmax_j(scale q[t][h] . k[b][j][g]) v[b][j][g]
 * q [T][heads][dim] io.  out [T][heads][dim], contiguous heads, tokens ld_out
 * apart, of out_dtype io, or SKSSM_E4M3 over scales [heads dim / 128][T] (rows ld_scales
 * apart) = max(largest |out| of a row's 128 columns / 448, 2^-64): what
 * sketchssm_matmul_fp8 reads (dim 64 with an even number of heads a key head, 128 or 256).
 * A padding row is 0.  Rows of `out` past the last sequence keep their values.
 * Scores, softmax statistics and sums are fp32; keys and values enter the products as they are, and with F32 io queries with 24 bits.
 * Weights e^(s - m) are taken over a maximum m that may be an earlier one of the row's (they are up to 2^16 then) and keep
 *     24 bits with F32 io,
 *     at least 16 bits with bf16 io where out is E4M3 (scales are fp32), or where the call's sequences have at most 16 rows
 *         (new tokens times heads a key head) on average: single tokens of up to 16 heads a key head,
 *     8 bits at least, bf16's, otherwise: prompts with bf16 io and out;
 * their sum is that of the rounded ones.  scale is from 2^-96 to 2^96.  Scores and scale times them are in fp32's range, up to 2^126,
 * but for scores that fall below it, which weigh nothing; values up to 2^80 leave the sums in it whatever the number of
 * keys.  A NaN reaches only outputs of its head whose token sees it.
 *
 * Equal calls give equal bits.  A token's may differ in their last places with the sequences beside it: keys are split elsewhere.
 * The form is one for the whole call, by the rows that a sequence has on average, and long contexts are split over workgroups only
 * in that of few rows: prompts and single tokens over long contexts are faster as two calls (a prompt of 4096 tokens and one
 * token over 131072 keys, 32 heads on 8 of 128 channels: 175 and 35 us, as one call 4.1 ms).
 *
 * workspace: sketchssm_attention_workspace bytes (may be 0), where a sequence
 * is split over workgroups; its contents need not be kept, and calls that may run at the same time need one each.
 */
typedef struct {
  int32_t io_dtype, out_dtype, heads;
  float scale;
  const void* q;
  int64_t ldq, q_head;
  void* out;
  int64_t ld_out;
  float* scales;
  int64_t ld_scales;
  void* workspace;
  size_t workspace_bytes;
} skssm_attention_args;
int sketchssm_attention(const skssm_cache* cache, const skssm_new_tokens* seq, const skssm_attention_args* args,
                        void* stream);
size_t sketchssm_attention_workspace(const skssm_cache* cache, int32_t heads, int32_t batch, int64_t tokens, int32_t columns);

#ifdef __cplusplus
}
#endif
#endif /* SKETCHSSM_ATTENTION_H */
