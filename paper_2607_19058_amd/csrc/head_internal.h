// head_internal.h -- what the kernels of the head's loss share.
#pragma once

#include "../../include/skew_loss.h"
#include "moe_internal.h"

namespace moe {

// A token as the gradients' kernels take it: the base-2 exponent of its sum, the logits' gradient's factors (times the power
// of two that its row of G is kept with), and its target (-1: no token).
struct HeadRow {
  float l2, both, one;
  int32_t target;
};

// One product of the head on the tiles of product_tiles.h. Operands are padded to chunks of 8 where a chunk may pass their end: rows and cols say
// where the result ends, pad_rows and pad_cols where its operands do.
struct HeadProduct {
  const void *a, *b;          // kForward: a rows, b [K x cols]; kBackward: b [cols x K]; kOuter: a [K x rows], b [K x cols]
  int64_t lda, ldb;
  int64_t rows, cols, K;      // of the result, and the contraction
  int64_t pad_rows, pad_cols; // kOuter: a's columns; b's columns or rows
};

// Tiles of the head's products, and about how long they take (us, contraction 2048): `full` a round with work-groups on all slots of the
// chip, `lone` one with a work-group on each compute unit at most. Both grow with the contraction. Measured with each tile forced:
//   logits of 4096 rows, 16384 words of width 2048 (forward | tied): 226 231 286 339 | 223 261 287 310;  of 1024 rows and 1152 words: 56 46
//   30 26 | 57 47 33 28.  Rows' gradient, 4096 x 4096 from 4096 words (untied, tied): 127 142 - 164, 117 123 - 181, weights' 122 122 - 183
struct HeadTile {
  int rows, cols, slots;
  double full, lone;
};
constexpr int kHeadTiles = 4;
inline HeadTile head_tile(bool backward, int i) {
  static const HeadTile tiles[2][kHeadTiles] = {{{256, 256, 256, 54, 54}, {128, 256, 512, 58, 40}, {64, 256, 512, 36, 24}, {64, 128, 768, 33, 20}},
                                                {{256, 256, 256, 56, 56}, {128, 256, 512, 70, 46}, {64, 256, 512, 36, 25}, {64, 128, 768, 32, 21}}};
  return tiles[backward ? 1 : 0][i];
}
inline int64_t head_count(const HeadTile &t, int64_t rows, int64_t cols) {
  return ((rows + t.rows - 1) / t.rows) * ((cols + t.cols - 1) / t.cols);
}
// of n tiles with contractions of K, and their launch
inline double head_time(const HeadTile &t, int64_t n, int64_t K) {
  constexpr int64_t kUnits = 256;
  const int64_t left = n % t.slots;
  const double more = left > kUnits ? (double)(left - kUnits) / (t.slots - kUnits) : 0.0;
  return ((double)(n / t.slots) * t.full + (left ? t.lone + (t.full - t.lone) * more : 0.0)) * (double)(K + 128) / 2176 + 4;
}

// Forward: of each row and each run of 128 (or 64) columns that a wave has, the largest base-2 exponent and the sum
// of the powers relative to it; the product of the row and its target's word.
struct alignas(8) HeadPair {
  float top, sum;
};
struct HeadForward {
  float c;                    // scale log2(e)
  const void *targets;
  int32_t target_bytes;
  int64_t vocab, col0;        // of the whole; the first column of this product
  HeadPair *part;             // [rows x part_ld], runs of this product from part_at on
  int64_t part_ld, part_at;
  float *target_sum;          // [rows]: <x, w_y>
};
int launch_head_forward(int mode, const HeadProduct &p, const HeadForward &f, void *stream);

// The same (kForward) for up to 16 rows: any position and alignment, K and cols as they are (no padding); 32 rows of b lie within 2^31
// bytes. One pair a row and work-group.
constexpr int64_t kFewRows = 16;
inline int64_t head_few_parts(int64_t cols) { return (cols + 127) / 128; }
int launch_head_few(const HeadProduct &p, const HeadForward &f, void *stream);

// Backward: G of this product's columns, float16 [rows x ldg]; or, split, as the sum of two bf16 numbers, [2 rows x ldg]: all rows of the
// upper halves, then all of the rests.
struct HeadGrad {
  float c;
  const HeadRow *row;
  int64_t vocab, col0;
  uint16_t *g;
  int64_t ldg;
  uint32_t *word_top;         // of each word of the vocabulary, bits of the largest magnitude in G as it is kept (split: not wanted)
};
int launch_head_grad(int mode, const HeadProduct &p, const HeadGrad &g, bool split, void *stream);

// result = 2^e (a b) + prev, of float16 operands. e is the sum of the exponents that they are kept with: of the result's rows or columns (top:
// bits of their largest magnitudes), and of G: of each row (row_exponent), or the largest of all (coef), which the rows of x then make up for.
// split: the operands are bf16, e is 0; and with `fold` the result's rows are twice as many, of which row t and the one half of them further on
// are added.
struct HeadResult {
  void *y;
  int64_t ldy;
  int32_t y_dtype;
  const float *prev;          // NULL, or float [rows x ldprev] that is added
  int64_t ldprev;
  const uint32_t *top;        // per column, or per row
  int32_t by_row;
  const int32_t *row_exponent;   // NULL: *coef
  const uint32_t *coef;
  int32_t split, fold;
  const HeadRow *token;       // NULL, or of each row: one that is no token gets zeros, whatever b holds
};
int launch_head_result(int mode, const HeadProduct &p, const HeadResult &r, char *ws, void *stream);

// Exponents of what is kept in float16: a value whose largest magnitude has the bits `top` is kept times 2^-exponent, so
// that the largest lies in [2^14, 2^15).
constexpr int kHalfTop = 14;
constexpr int half_exponent(uint32_t top) { return (int)(top >> 23) - 127 - kHalfTop; }
// The same of a row of G, from its larger factor: an entry is at most twice it.
constexpr int factor_exponent(uint32_t top) { return half_exponent(top) + 1; }

// Float16 has no room for a word that is rare for every token: beside the tokens' factors its entries of G are below the smallest normal
// number, and at last 0. A piece's words whose largest entry is below rare_top() are computed a second time, with a power of two of
// their own (head_rare.hip). Below the normal numbers an entry is off by 2^-25.8 on average (2^-24 / sqrt(12)): the tokens together by
// 2^-25.8 sqrt(tokens), which is 2^-8.8 of rare_top(), about a rounding to bf16 of the word's largest entry.
inline float rare_top(int64_t tokens) { return 7.62939453125e-06f * __builtin_sqrtf((float)tokens); }   // 2^-17 sqrt(tokens)
struct HeadRare {
  const void *x, *x16;        // x as it is [tokens x d8], and as the gradients take it
  int64_t ldx, ldx16, tokens, d, d8;
  const void *w;              // bf16, the piece's words, anywhere
  int64_t ldw, words;         // and how many
  int32_t tied;
  float c;
  const HeadRow *row;
  const uint32_t *word_top, *x_top, *coef;   // of the piece's words, ..
  int64_t word0;              // the piece's first word
  int32_t *list;              // [1 + words]: how many are rare, and which, in order
  void *copy;                 // their words in w's layout, rows of d8 values, or d8 rows
  int64_t ldcopy;
  uint16_t *g;                // and their G
  int64_t ldg;
  void *dw;                   // the piece's first word in dw
  int64_t lddw;
};
int launch_head_rare(const HeadRare &r, void *stream);

// The calls of skew_loss.h, after their checks.
size_t head_forward_scratch(const skew_head_desc &h);
size_t head_backward_scratch(const skew_head_desc &h);
int launch_fill_zero(void *dw, int64_t rows, int64_t cols, int64_t ld, void *stream);   // bf16
int launch_head_loss(const skew_head_desc &h, float *loss, float *lse, char *ws, void *stream);
int launch_head_loss_backward(const skew_head_desc &h, const float *lse, const float *dloss, const float *dlse, void *dx, int dx_dtype,
                              int64_t lddx, void *dw, int64_t lddw, char *ws, void *stream);

}  // namespace moe
