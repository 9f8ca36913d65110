// Which tiles a product gets, into how many parts its contraction is cut, and what the calls' workspaces hold: arithmetic of the host
// alone, by types of 2 (bf16) and 4 bytes (fp32).
//
// A caller keeps the workspace of its most rows and makes calls of fewer with it, so what a workspace call reports must hold what
// any smaller number of rows needs, although shape and cut go up and down with the rows.  Each plan therefore has an allowance that grows
// with the rows: the choice is made among what fits into it, and it is the allowance that is reported.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "hpd.h"

namespace {

enum { BY_ROWS = 0, BY_COLUMNS = 1 };
enum { LARGE = 0, MIDDLE = 1, SMALL = 2, FEW64 = 3, FEW32 = 4, FEW128 = 5, WIDE = 6 };
constexpr int SHAPE_SUMS[] = {1, 2, 4, 4, 4, 2, 1};  // that a block's contraction is added up in

template <typename T>
constexpr int CHUNK = 16 / (int)sizeof(T);  // elements of a 16-byte chunk
template <typename T>
constexpr int STAGE_K = 8 * CHUNK<T>;       // of the contracted index in a stage

constexpr int LEAST_STAGES = 4;  // of a part
// how many parts a contraction of k elements can have, of `most`; 0: it is never cut
template <typename T>
int64_t most_parts(int64_t k, int64_t most) {
  const int64_t parts = std::min(most, (k + STAGE_K<T> - 1) / STAGE_K<T> / LEAST_STAGES);
  return parts > 1 ? parts : 0;
}

struct Plan {
  int shape, splits;
  int64_t bm() const { return shape == LARGE ? 256 : shape == WIDE ? 192 : shape == MIDDLE ? 128 : 64; }
  int64_t bn() const { return shape == FEW32 ? 32 : shape == FEW128 ? 128 : shape == WIDE ? 256 : bm(); }
};
// The least time by a simple account, in us: workgroups go in rounds of as many as run at a time.  Each takes `fixed` for its start and
// end, and for a stage stage[n - 1] where n run on its CU, `uneven` times that where contracted rows do not begin at multiples of 128 bytes
// (a row's part of a stage is then in two lines).  What is read comes at `rate` TB/s at most; each workgroup has `flight` KB of it on the
// way, about 1 us, and a CU takes a third more than its share of the rate.  Parts are written and read, and take a launch.  (Fitted to
// random products of 1 to 9000 rows, weights from memory, in all shapes and cuts: of 460 in bf16 and 240 in fp32 the choice takes 1.01 times
// the best one's time in the geometric mean, 1.2 at worst.)
struct ShapeCost {
  int on_cu;
  double stage[3], uneven, fixed, flight, rate;
};
constexpr int CUS = 256;
template <typename T>
ShapeCost shape_cost(int shape) {
  constexpr ShapeCost BF16[] = {{1, {1.55}, 1.0, 7.0, 64, 5.2},              {2, {0.78, 0.97}, 1.15, 4.0, 32, 5.0},
                                {3, {0.28, 0.46, 0.68}, 1.2, 2.7, 16, 5.2}, {2, {0.25, 0.39}, 1.15, 3.5, 24, 5.7},
                                {3, {0.24, 0.3, 0.4}, 1.1, 2.5, 24, 5.8},   {2, {0.39, 0.76}, 1.2, 4.0, 24, 5.5},
                                {1, {1.22}, 1.1, 6.0, 56, 5.2}};
  constexpr ShapeCost F32[] = {{}, {}, {3, {0.56, 1.05, 1.45}, 1.1, 2.5, 16, 5.2}, {2, {0.47, 1.03}, 1.2, 3.0, 24, 4.5},
                               {3, {0.46, 1.0, 1.1}, 1.0, 3.3, 24, 5.9}};
  return sizeof(T) == 4 ? F32[shape] : BF16[shape];
}
// k: contracted elements, of all segments; cut: us that parts cost besides being written and read; fits(p): p is allowed
template <typename T, int FA, int FB, typename Fits>
Plan plan_product(int64_t features, int64_t rows, int64_t k, bool dual, int most_splits, double cut, Fits fits) {
  const int64_t stages = (k + STAGE_K<T> - 1) / STAGE_K<T>;
  const double bytes = (double)((dual ? 2 : 1) * features + rows) * k * sizeof(T);
  Plan best = {SMALL, 1};
  double least = 1e30;
  for (int shape = sizeof(T) == 4 ? SMALL : LARGE; shape <= (sizeof(T) == 4 ? FEW32 : WIDE); ++shape) {
    Plan p = {shape, 1};
    if (shape == WIDE ? FA != BY_ROWS : shape >= FEW64 && (FB != BY_ROWS || rows > p.bn())) continue;
    const ShapeCost c = shape_cost<T>(shape);
    const double uneven = FA == BY_ROWS && FB == BY_ROWS && k * sizeof(T) % 128 ? c.uneven : 1.0;
    const int64_t bm = dual ? p.bm() / 2 : p.bm(), places = c.on_cu * CUS;
    const int64_t tiles = ((features + bm - 1) / bm) * ((rows + p.bn() - 1) / p.bn());
    for (p.splits = 1; p.splits <= most_splits && (p.splits == 1 || stages / p.splits >= LEAST_STAGES); ++p.splits) {
      if (!fits(p)) continue;
      const int64_t all = tiles * p.splits, full = all / places, rest = all % places, deep = (stages + p.splits - 1) / p.splits;
      double t = (double)full * (deep * c.stage[c.on_cu - 1] * uneven + c.fixed);
      if (rest) t += deep * c.stage[(rest - 1) / CUS] * uneven + c.fixed;
      const double at_once = (double)std::min(all, places), on_cu = std::ceil(at_once / CUS);
      const double cu = full ? 0.0 : on_cu * bytes / all / (std::min(on_cu * c.flight, 1.32 * c.rate * 1e3 / CUS) * 1e3);
      t = std::max(t, std::max(cu, bytes / std::min(c.rate * 1e6, at_once * c.flight * 1e3)) + c.fixed);
      if (p.splits > 1) t += cut + 2.6 + 0.12 * p.splits + (double)features * rows * p.splits * 8 / 6.0e6;
      if (t < least) {
        least = t;
        best = p;
      }
    }
  }
  return best;
}

constexpr int64_t MB = (int64_t)1 << 20;

inline int64_t round16(int64_t x) { return (x + 15) / 16 * 16; }
inline int64_t round4(int64_t x) { return (x + 3) / 4 * 4; }
inline int64_t part_bytes(Plan p, int64_t rows, int64_t features) { return p.splits > 1 ? p.splits * rows * features * 4 : 0; }

// ---- gated feed-forward block: how the products are made, and where the workspace has what they leave for each other; `needs` bytes of it,
// `bytes` with what fewer rows need.
constexpr int FFN_SPLITS = 16;  // of a contraction over the inner width, at most
// Parts take up to 512 MB: random blocks of up to 20000 rows and 8192 channels then have the account's best choice but for 1 %
// of them, which take up to 1.10 times its time (256 MB: 3 %, 1.25).
constexpr int64_t FFN_PART_BYTES = 512 * MB;
template <typename T>
int64_t ffn_part_allowance(int64_t n, int64_t width, int64_t k) { return std::min(most_parts<T>(k, FFN_SPLITS) * n * width * 4, FFN_PART_BYTES); }

template <typename T>
struct FfnForwardPlan {
  Plan in, down;
  int64_t parts, needs, bytes;
  FfnForwardPlan(const hpd_ffn_config& c, int64_t n) {
    const int64_t allowance = ffn_part_allowance<T>(n, c.width, c.inner);
    in = plan_product<T, BY_ROWS, BY_ROWS>(c.inner, n, c.width, true, 1, 0.0, [](Plan) { return true; });
    down = plan_product<T, BY_ROWS, BY_ROWS>(c.width, n, c.inner, false, FFN_SPLITS, 0.0,
                                             [&](Plan p) { return part_bytes(p, n, c.width) <= allowance; });
    parts = round16(n * c.inner * (int64_t)sizeof(T));
    needs = parts + part_bytes(down, n, c.width);
    bytes = parts + allowance;
  }
};
template <typename T>
struct FfnBackwardPlan {
  Plan inner, dx, in_weights, down_weights;
  int64_t h, parts, needs, bytes;
  FfnBackwardPlan(const hpd_ffn_config& c, int64_t n) {
    const int64_t allowance = ffn_part_allowance<T>(n, c.width, 2 * (int64_t)c.inner);
    auto any = [](Plan) { return true; };
    inner = plan_product<T, BY_COLUMNS, BY_ROWS>(c.inner, n, c.width, false, 1, 0.0, any);
    dx = plan_product<T, BY_COLUMNS, BY_ROWS>(c.width, n, 2 * (int64_t)c.inner, false, FFN_SPLITS, 0.0,
                                              [&](Plan p) { return part_bytes(p, n, c.width) <= allowance; });
    in_weights = plan_product<T, BY_COLUMNS, BY_COLUMNS>(c.width, 2 * (int64_t)c.inner, n, false, 1, 0.0, any);
    down_weights = plan_product<T, BY_COLUMNS, BY_COLUMNS>(c.inner, c.width, n, false, 1, 0.0, any);
    h = round16(n * 2 * c.inner * (int64_t)sizeof(T));
    parts = h + round16(n * c.inner * (int64_t)sizeof(T));
    needs = parts + part_bytes(dx, n, c.width);
    bytes = parts + allowance;
  }
};

// ---- vocabulary head
constexpr int HEAD_SPLITS = 32;                 // of a contraction, at most
constexpr int64_t LOGIT_PART_BYTES = 128 * MB;  // parts of the logits, or sums of their rows (of 8000 random heads of up to 20000 rows and 160000
                                                // tokens none wanted more)
constexpr int64_t HIDDEN_PART_BYTES = 256 * MB; // parts of dhidden
// The logits' gradients of a piece of the vocabulary: what the memory side caches hold (more from 524288 bf16 or 262144 fp32 rows on: a
// piece has 256 tokens at least).  Their rows are an operand of the products behind, with a stride as any: a stage's 64 rows of bf16, those
// behind the last among them, begin within 32 bits of the first.
constexpr int64_t PIECE_BYTES = 256 * MB, PIECE_ROW_BYTES = 8 * MB;

// The logits' product.  Both calls sum a logit's products in the same order, so that the gradients' logits are those that lse was made from, to
// the bit: 1 - p of a confident token is the difference of the two (logits of 300, a contraction of 480 to 2048: with a plan of each
// call's own 1 - p = 1e-4 was off by its own size and more).  The order is that of the parts, and in a part of a tile's sums.  So the whole
// vocabulary is planned once, with what parts cost the forward call; a piece of it may take another shape with as many sums.
template <typename T>
struct HeadLogitsPlan {
  static constexpr int64_t UNIT = 256;
  int64_t pieces, piece;  // of the vocabulary in the backward call; a multiple of a tile's tokens
  int64_t of_parts, of_sums;
  Plan whole, of_piece;
  static int sums(Plan p) { return sizeof(T) == 4 && p.shape == SMALL && p.splits == 1 ? 1 : SHAPE_SUMS[p.shape]; }  // (fp32: IN_ORDER)
  static int64_t sum_bytes(int64_t n, int64_t vocab, int64_t bm) { return round16(n * ((vocab + bm - 1) / bm * 16 + 4)); }
  HeadLogitsPlan(int64_t n, int32_t width, int32_t vocab) {
    const int64_t row_bytes = std::min(PIECE_ROW_BYTES, PIECE_BYTES / std::max<int64_t>(n, 1));
    const int64_t most = std::max(UNIT, row_bytes / (int64_t)sizeof(T) / UNIT * UNIT);
    pieces = (vocab + most - 1) / most;
    piece = ((vocab + pieces - 1) / pieces + UNIT - 1) / UNIT * UNIT;
    of_parts = std::min(most_parts<T>(width, HEAD_SPLITS) * n * round4(vocab) * 4, LOGIT_PART_BYTES);
    // (the largest tiles leave the least sums: they always fit)
    of_sums = std::max(sum_bytes(n, vocab, sizeof(T) == 4 ? 64 : 256), std::min(sum_bytes(n, vocab, 64), LOGIT_PART_BYTES));
    whole = plan_product<T, BY_ROWS, BY_ROWS>(vocab, n, width, false, pieces == 1 ? HEAD_SPLITS : 1, 1.2 * (vocab / 1024 + 1),  // (a row's turns in its one workgroup)
                                              [&](Plan p) { return needs(p, n, vocab) <= (p.splits > 1 ? of_parts : of_sums); });
    of_piece = whole;
    if (pieces > 1)
      of_piece = plan_product<T, BY_ROWS, BY_ROWS>(piece, n, width, false, 1, 0.0, [&](Plan p) { return sums(p) == sums(whole); });
  }
  static int64_t needs(Plan p, int64_t n, int64_t vocab) { return p.splits > 1 ? part_bytes(p, n, round4(vocab)) : sum_bytes(n, vocab, p.bm()); }
};
template <typename T>
struct HeadForwardPlan {
  Plan product;
  int64_t tiles, of_target, needs, bytes;
  HeadForwardPlan(int64_t n, int32_t width, int32_t vocab) {
    const HeadLogitsPlan<T> l(n, width, vocab);
    product = l.whole;
    tiles = (vocab + product.bm() - 1) / product.bm();
    of_target = n * tiles * 16;
    needs = HeadLogitsPlan<T>::needs(product, n, vocab);
    bytes = std::max(l.of_sums, l.of_parts);
  }
};
template <typename T>
struct HeadBackwardPlan {
  int64_t piece;
  Plan logits, d_hidden, d_weight;
  int64_t parts, needs, bytes;
  HeadBackwardPlan(int64_t n, int32_t width, int32_t vocab) {
    constexpr int64_t UNIT = HeadLogitsPlan<T>::UNIT;
    const HeadLogitsPlan<T> l(n, width, vocab);
    logits = l.of_piece;
    piece = l.piece;
    const int64_t of_hidden = std::max(n * width * 4, std::min(most_parts<T>(vocab, HEAD_SPLITS) * n * width * 4, HIDDEN_PART_BYTES));
    d_hidden = plan_product<T, BY_COLUMNS, BY_ROWS>(width, n, std::min<int64_t>(piece, vocab), false, HEAD_SPLITS, 0.0,
                                                    [&](Plan p) { return p.splits * n * width * 4 <= of_hidden; });
    d_weight = plan_product<T, BY_COLUMNS, BY_COLUMNS>(width, std::min<int64_t>(piece, vocab), n, false, 1, 0.0, [](Plan) { return true; });
    parts = round16(n * piece * (int64_t)sizeof(T));
    // (the logits' parts have been read when those of dhidden are written)
    needs = parts + std::max(d_hidden.splits * n * width * 4, part_bytes(logits, n, round4(vocab)));
    const int64_t whole = (vocab + UNIT - 1) / UNIT * UNIT;
    bytes = round16(std::min(n * std::min(whole * (int64_t)sizeof(T), PIECE_ROW_BYTES), std::max(n * UNIT * (int64_t)sizeof(T), PIECE_BYTES))) +
            std::max(of_hidden, l.of_parts);
  }
};

}  // namespace
