// head_plan.h -- host arithmetic of the head's loss: tiles and remainders of its products, pieces of the vocabulary, the workspace.
#pragma once

#include <algorithm>

#include "head_internal.h"

namespace moe {

// ---- the logits' products ----------------------------------------------------------------------
// Which tile: the one that takes the least time. Where the last round of large tiles would be nearly empty, the columns past the whole
// rounds (first to last) get tiles of their own.
struct LogitsChoice {
  int tile;
  int64_t first;   // columns that `tile` takes; the rest has `rest`
  int rest;
};
inline double logits_best(int mode, int64_t rows, int64_t cols, int64_t K, int *tile) {
  double least = 1e300;
  for (int i = 0; i < kHeadTiles; i++) {
    const HeadTile t = head_tile(mode == kBackward, i);
    const double time = head_time(t, head_count(t, rows, cols), K);
    if (time < least) {
      least = time;
      *tile = i;
    }
  }
  return least;
}
inline LogitsChoice choose_logits(int mode, const HeadProduct &p) {
  LogitsChoice c = {0, p.cols, 0};
  const double all = logits_best(mode, p.rows, p.cols, p.K, &c.tile);
  const HeadTile large = head_tile(mode == kBackward, 0);
  const int64_t down = (p.rows + large.rows - 1) / large.rows;
  const int64_t first = head_count(large, p.rows, p.cols) / large.slots * large.slots / down * large.cols;
  if (first > 0 && first < p.cols) {
    int rest = 0;
    const double time = head_time(large, first / large.cols * down, p.K) + logits_best(mode, p.rows, p.cols - first, p.K, &rest);
    if (time < 0.97 * all) c = {0, first, rest};
  }
  return c;
}
inline int head_runs(int mode, int tile, int64_t cols) {   // of a wave's columns
  const int w = head_tile(mode == kBackward, tile).cols;
  return (int)((cols + w - 1) / w) * 2;
}
// runs that a row's columns fall into
inline int head_parts(int mode, const HeadProduct &p) {
  const LogitsChoice c = choose_logits(mode, p);
  return head_runs(mode, c.tile, c.first) + (c.first < p.cols ? head_runs(mode, c.rest, p.cols - c.first) : 0);
}

// ---- the gradients' products -------------------------------------------------------------------
// Which tile, and how many work-groups share a contraction (their parts go through memory, and join_kernel adds them up: a launch, and
// the bytes at some 4 TB/s).
struct ResultChoice {
  int tile, parts;
};
inline double result_best(int mode, int64_t rows, int64_t cols, int64_t K, ResultChoice *c) {
  double least = 1e300;
  for (const int tile : {0, 1, 3}) {
    const HeadTile t = head_tile(mode == kBackward, tile);
    const int64_t n = head_count(t, rows, cols);
    for (const int parts : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
      if (parts > 1 && (K / parts < 128 || n * parts > 2 * t.slots)) break;
      const double time = head_time(t, n * parts, K / parts) + (parts > 1 ? 4 + (double)parts * rows * cols * 4 * 2 / 4e6 : 0);
      if (time < least) {
        least = time;
        *c = {tile, parts};
      }
    }
  }
  return least;
}
// Where the last round of large tiles would be nearly empty, or the last row or column of them, what lies past the whole ones is
// a product of its own.
struct ResultPlan {
  ResultChoice main, rest;
  int64_t rows, cols;   // of main
};
inline ResultPlan plan_result(int mode, const HeadProduct &p, bool fold) {
  ResultPlan s = {{0, 1}, {0, 0}, p.rows, p.cols};
  double least = 0.97 * result_best(mode, p.rows, p.cols, p.K, &s.main);
  const HeadTile t = head_tile(mode == kBackward, 0);
  const int64_t down = (p.rows + t.rows - 1) / t.rows, across = (p.cols + t.cols - 1) / t.cols, whole = down * across / t.slots * t.slots;
  auto cut = [&](int64_t rows, int64_t cols) {   // (one of them all)
    if (rows == 0 || cols == 0 || (rows >= p.rows && cols >= p.cols) || (fold && rows < p.rows)) return;
    ResultPlan c = {{0, 1}, {0, 1}, rows, cols};
    const double time = result_best(mode, rows, cols, p.K, &c.main) +
                        result_best(mode, rows < p.rows ? p.rows - rows : rows, rows < p.rows ? cols : p.cols - cols, p.K, &c.rest);
    if (time < least) {
      least = time;
      s = c;
    }
  };
  cut(whole / across * t.rows, p.cols);
  cut(p.rows, whole / down * t.cols);
  cut(p.rows / t.rows * t.rows, p.cols);
  cut(p.rows, p.cols / t.cols * t.cols);
  return s;
}
inline int64_t part_ld(int64_t cols) { return (cols + 7) / 8 * 8; }

inline size_t scratch_of(const ResultChoice &c, int64_t rows, int64_t cols, bool fold) {
  return c.parts > 1 || fold ? pad256((size_t)c.parts * (size_t)rows * (size_t)part_ld(cols) * 4) : 0;
}

inline size_t head_result_scratch(int mode, const HeadProduct &p, bool fold) {
  const ResultPlan s = plan_result(mode, p, fold);
  const size_t main = scratch_of(s.main, s.rows, s.cols, fold);
  if (s.rest.parts == 0) return main;
  const size_t rest = scratch_of(s.rest, s.rows < p.rows ? p.rows - s.rows : p.rows, s.rows < p.rows ? p.cols : p.cols - s.cols, fold);
  return main > rest ? main : rest;
}

// ---- the calls ---------------------------------------------------------------------------------
inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
// The row stride of an operand in the workspace: whole 128-byte lines (3001 tokens, 32003 words of width 1031, a pass: 1067 us with chunks of 8,
// 1000 with lines), and one more where rows would be multiples of 1024 bytes apart, on the same memory channels (8192 tokens, 16384 words of
// width 1024, backward: 839 | 824, tied 855 | 822).
inline int64_t lines(int64_t cols) { return up(cols, 64) + (up(cols, 64) % 512 == 0 ? 64 : 0); }
inline bool chunks(const void *p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }
inline bool tied(const skew_head_desc &h) { return (h.flags & SKEW_TRANSPOSE) != 0; }

// What is the same in both calls: which operands the tiles take as they are, and pieces of the vocabulary (of kPieceStep columns,
// the last one of what is left).
constexpr int64_t kTileRows = 256, kPieceStep = 256, kMaxPiece = 1 << 21;
constexpr int64_t kPieceBytes = (int64_t)512 << 20;   // of G, and of a copy of w (8192 tokens, 50304 words: 128 MiB 5.91 ms, 256 6.02, 512 5.72, 1024 5.71)
constexpr int64_t kRun = 16384;                       // rows of a forward launch, whose pairs are held
// Whether G is split (see BackwardPlan).
inline bool splits(const skew_head_desc &h) {
  constexpr int64_t kRows = 512, kSmall = (int64_t)1 << 29;   // (tokens * d is below 2^42)
  return h.tokens <= kRows || h.tokens * h.d <= kSmall / h.vocab;
}
struct HeadPlan {
  bool x_as_is, w_as_is;
  int64_t d8, v8, ldd, piece, run;   // ldd: stride of rows of d in the workspace
};
inline HeadPlan head_plan(const skew_head_desc &h, bool backward) {
  HeadPlan p;
  p.d8 = up(h.d, 8);
  p.v8 = up(h.vocab, 8);
  p.ldd = lines(h.d);
  p.x_as_is = chunks(h.x, h.ldx) && h.d % 8 == 0 && short_rows(kTileRows, h.ldx);
  p.w_as_is = chunks(h.w, h.ldw) && h.d % 8 == 0 && (tied(h) || h.vocab % 8 == 0) && short_rows(kTileRows, h.ldw);
  p.run = std::min(h.tokens, kRun);
  if (!backward && p.w_as_is) {
    p.piece = h.vocab;
  } else {
    const int64_t wide = std::max(p.d8, backward ? h.tokens * (splits(h) ? 2 : 1) : 0);   // rows of G, columns of w
    int64_t most = std::min(std::max(kPieceBytes / (2 * wide), kPieceStep), kMaxPiece);
    const int64_t n = (h.vocab + most - 1) / most;
    p.piece = std::min(up((h.vocab + n - 1) / n, kPieceStep), p.v8);
  }
  return p;
}
inline int64_t pieces(const skew_head_desc &h, const HeadPlan &p) { return (h.vocab + p.piece - 1) / p.piece; }
inline int64_t piece_cols(const skew_head_desc &h, const HeadPlan &p, int64_t v0) { return std::min(p.piece, h.vocab - v0); }

// bytes of a piece of w in the workspace
inline size_t words_bytes(const skew_head_desc &h, const HeadPlan &p) {
  return 2 * (size_t)(tied(h) ? up(p.piece, 8) * p.ldd : p.d8 * lines(p.piece));
}
// w from word v0 on, as it is
inline const uint16_t *words(const skew_head_desc &h, int64_t v0) {
  return static_cast<const uint16_t *>(h.w) + (tied(h) ? v0 * h.ldw : v0);
}
// x w of rows `rows` and the piece at v0 of `cols` words: from (a, lda) and w or its copy
inline HeadProduct logits_of(const skew_head_desc &h, const HeadPlan &p, const void *a, int64_t lda, int64_t rows, int64_t v0, const void *copy) {
  const int64_t cols = piece_cols(h, p, v0), cols8 = tied(h) && !copy ? cols : up(cols, 8);   // (words in rows need no padding)
  HeadProduct q = {a, copy ? copy : words(h, v0), lda, copy ? (tied(h) ? p.ldd : lines(cols)) : h.ldw, rows, cols, p.d8, 0, cols8};
  return q;
}
// (shapes alone)
inline int mode_of(const skew_head_desc &h) { return tied(h) ? kBackward : kForward; }

// a region of the workspace
struct Regions {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t here = at;
    at += pad256(bytes);
    return here;
  }
};

struct ForwardPlan : HeadPlan {
  bool few;
  int64_t part_ld;
  size_t part, sum, x, w, bytes;
};
inline ForwardPlan forward_plan(const skew_head_desc &h) {
  ForwardPlan f;
  static_cast<HeadPlan &>(f) = head_plan(h, false);
  // One row and words at odd positions, in pieces copied for the tiles | as they are (us): width 2048, 8001 words 34 | 46, 16001 47 | 44,
  // 24001 59 | 52, 50257 117 | 77; width 512, 50257 36 | 26; width 4096, 16001 79 | 78.
  f.few = !f.w_as_is && !tied(h) && h.tokens <= kFewRows && h.vocab >= 16384 && (h.d == 1 || short_rows(kTileRows, h.ldw));
  if (f.few) f.x_as_is = f.w_as_is = true;   // (whatever their alignment)
  // rows of the last run may be fewer, and their tiles narrower
  f.part_ld = f.few ? head_few_parts(h.vocab) : 0;
  const int64_t last = h.tokens % f.run ? h.tokens % f.run : f.run;
  for (const int64_t rows : {f.run, last}) {
    if (f.few) break;
    int64_t ld = 0;
    for (int64_t v0 = 0; v0 < h.vocab; v0 += f.piece) ld += head_parts(mode_of(h), logits_of(h, f, nullptr, 0, rows, v0, nullptr));
    f.part_ld = std::max(f.part_ld, ld);
  }
  Regions r;
  f.part = r.take((size_t)f.run * f.part_ld * sizeof(HeadPair));
  f.sum = r.take((size_t)f.run * 4);
  f.x = f.x_as_is ? 0 : r.take((size_t)f.run * f.ldd * 2);
  f.w = f.w_as_is ? 0 : r.take(words_bytes(h, f));
  f.bytes = r.at;
  return f;
}

// Up to 512 tokens the bytes of w decide. Then G is the sum of two bf16 numbers, and w enters its product as it is; with more,
// where the products decide, w is converted to float16, which takes its bytes four times more, and rare words take four launches. Where
// tokens, width and words together are few, these launches decide. Backward calls, us, float16 | two bf16 numbers (the rule goes by
// tokens alone; a few percent are lost on either side of it):
//   tokens                             1           64          256         512         768          1024
//   50304 words of width 2048          364 | 205   402 | 241   517 | 398   616 | 599   743 | 848    848 | 1031
//   the same, tied                     398 | 198   427 | 235   512 | 389   639 | 615   761 | 838    879 | 1035
//   32003 words of width 1031          138 |  97   156 | 117   213 | 207   299 | 289   339 | 378    384 | 472
//   8192 words of width 1024            69 |  48    73 |  49    81 |  64    95 |  95   118 | 120    130 | 138
//   tokens x width x words             2048x128x512   1024x512x1024   2048x256x1024   4096x128x1024   1024x1024x1024   1024x256x4096
//     (2^27, 2^29, .., 2^30)           51 | 38        62 | 48         61 | 49         66 | 59         66 | 56          67 | 62
//     tied                             58 | 38        66 | 50         65 | 49         71 | 59         75 | 58          75 | 64
struct BackwardPlan : HeadPlan {
  bool split;
  int64_t rows;   // of G
  int64_t top_count;   // bits of largest magnitudes: of G's factors, x's columns, w's; of each word's G
  size_t tops, row, exponent, list, x16, x, w16, w, g, dx, rest, bytes;
  int64_t ldg;
};
// the three products of a piece
inline HeadProduct dx_of(const skew_head_desc &h, const BackwardPlan &b, const void *g, const void *w16, int64_t v0) {
  const int64_t cols = piece_cols(h, b, v0), cols8 = up(cols, 8);
  if (!b.split || !b.w_as_is) return {g, w16, b.ldg, tied(h) ? b.ldd : lines(cols), b.rows, h.d, cols8, 0, b.d8};
  return {g, words(h, v0), b.ldg, h.ldw, b.rows, h.d, tied(h) ? cols : cols8, 0, b.d8};   // (words in rows end with the contraction)
}
inline HeadProduct dw_of(const skew_head_desc &h, const BackwardPlan &b, const void *x16, const void *g, int64_t v0) {
  const int64_t cols = piece_cols(h, b, v0), cols8 = up(cols, 8);
  if (tied(h)) return {g, x16, b.ldg, b.ldd, cols, h.d, b.rows, cols8, b.d8};
  return {x16, g, b.ldd, b.ldg, h.d, cols, b.rows, b.d8, cols8};
}
inline int dx_mode(const skew_head_desc &h) { return tied(h) ? kForward : kBackward; }

inline BackwardPlan backward_plan(const skew_head_desc &h) {
  BackwardPlan b;
  static_cast<HeadPlan &>(b) = head_plan(h, true);
  b.ldg = lines(b.piece);
  b.split = splits(h);
  b.rows = b.split ? 2 * h.tokens : h.tokens;
  const size_t x = (size_t)h.tokens * b.ldd * 2, w = words_bytes(h, b);
  Regions r;
  b.top_count = b.split ? 0 : 1 + 2 * b.d8 + b.v8;
  b.tops = r.take((size_t)b.top_count * 4);
  b.row = r.take((size_t)h.tokens * sizeof(HeadRow));
  b.exponent = r.take((size_t)h.tokens * 4);
  b.list = b.split ? 0 : r.take((size_t)(1 + b.piece) * 4);
  b.x16 = r.take((size_t)b.rows * b.ldd * 2);   // split: x twice, as it is
  b.x = b.x_as_is || b.split ? b.x16 : r.take(x);
  b.w16 = b.split ? 0 : r.take(w);
  b.w = b.w_as_is ? 0 : r.take(w);
  b.g = r.take((size_t)b.rows * b.ldg * 2);
  b.dx = pieces(h, b) > 1 ? r.take((size_t)h.tokens * b.d8 * 4) : 0;
  size_t rest = 0;
  for (int64_t v0 = 0; v0 < h.vocab; v0 += b.piece) {
    rest = std::max(rest, head_result_scratch(dx_mode(h), dx_of(h, b, nullptr, nullptr, v0), b.split));
    rest = std::max(rest, head_result_scratch(kOuter, dw_of(h, b, nullptr, nullptr, v0), false));
  }
  b.rest = r.take(rest);
  b.bytes = r.at;
  return b;
}

}  // namespace moe
