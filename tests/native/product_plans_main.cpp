// The plans of the feed-forward block's and the vocabulary head's products over many sizes: a workspace that is reported for a number of rows
// holds what any smaller number needs, both of the head's calls sum logits in the same order, and a row of a
// piece's gradients is no longer than a stride may be.  Exit code 0 = no finding.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "hpd_product_plan.h"

#define CHECK(cond, ...)                                                              \
  do {                                                                                \
    if (!(cond)) {                                                                    \
      std::fprintf(stderr, "CHECK failed at line %d: %s: ", __LINE__, #cond);         \
      std::fprintf(stderr, __VA_ARGS__);                                              \
      std::fprintf(stderr, "\n");                                                     \
      std::exit(1);                                                                   \
    }                                                                                 \
  } while (0)

// Row counts up to where nothing changes any more: every one of few rows, then steps on both sides of tiles' borders.
template <typename F>
static void rows(F f) {
  for (int64_t n = 1; n <= 700; ++n) f(n);
  for (int64_t n = 704; n <= 24000; n += n < 4096 ? 32 : 256)
    for (int64_t d : {-1, 0, 1}) f(n + d);
  for (int64_t n = 1 << 15; n <= (1 << 23); n *= 2) f(n);
}

template <typename T>
static void ffn(int32_t width, int32_t inner) {
  const hpd_ffn_config c = {width, inner, 0, 0};
  int64_t forward = 0, backward = 0;
  rows([&](int64_t n) {
    const FfnForwardPlan<T> f(c, n);
    const FfnBackwardPlan<T> b(c, n);
    CHECK(f.needs <= f.bytes && b.needs <= b.bytes, "block, %lld rows, %d to %d", (long long)n, width, inner);
    CHECK(f.bytes >= forward && b.bytes >= backward, "block, fewer bytes for %lld rows, %d to %d", (long long)n, width, inner);
    forward = f.bytes;
    backward = b.bytes;
  });
}

template <typename T>
static void head(int32_t width, int32_t vocab) {
  int64_t forward = 0, backward = 0;
  rows([&](int64_t n) {
    if ((n + 127) / 128 * ((int64_t)vocab / 64 + 1) > (1 << 22)) return;
    const HeadForwardPlan<T> f(n, width, vocab);
    const HeadBackwardPlan<T> b(n, width, vocab);
    CHECK(f.needs <= f.bytes && b.needs <= b.bytes, "head, %lld rows, %d of %d", (long long)n, width, vocab);
    CHECK(f.bytes >= forward && b.bytes >= backward, "head, fewer bytes for %lld rows, %d of %d", (long long)n, width, vocab);
    // the same sums in both calls
    using L = HeadLogitsPlan<T>;
    CHECK(f.product.splits == b.logits.splits && L::sums(f.product) == L::sums(b.logits), "logits, %lld rows, %d of %d", (long long)n, width, vocab);
    CHECK(b.piece % 256 == 0 && b.piece * (int64_t)sizeof(T) <= 1 << 23, "a piece's rows, %lld rows, %d of %d", (long long)n, width, vocab);
    CHECK(b.logits.splits == 1 || b.piece >= vocab, "parts of pieces, %lld rows, %d of %d", (long long)n, width, vocab);
    forward = f.bytes;
    backward = b.bytes;
  });
}

int main() {
  std::mt19937 rng(26209);
  const int widths[] = {8, 72, 256, 480, 1152, 2048, 4096, 5120, 8192};
  for (int i = 0; i < 24; ++i) {
    const int width = widths[rng() % 9], inner = 8 * (1 + (int)(rng() % (width / 2 + 1)));
    i % 3 ? ffn<uint16_t>(width, inner) : ffn<float>(width, inner);
    const int vocab = rng() % 3 ? 1 + (int)(rng() % 4000) : 1 + (int)(rng() % 160000);
    i % 3 ? head<uint16_t>(width, vocab) : head<float>(width, vocab);
  }
  ffn<uint16_t>(4096, 12288);
  head<uint16_t>(4096, 2057);
  head<float>(1152, 50021);
  for (const int vocab : {(1 << 21) + 1, (1 << 22) + 777, 1 << 25, 1 << 28}) {
    head<uint16_t>(8, vocab);
    head<float>(8, vocab);
  }
  // (what the GPU tests of contractions in parts go by)
  const int32_t cut[][3] = {{1, 8192, 1},     {5, 8192, 67},   {69, 8192, 1119}, {130, 5120, 385}, {33, 4104, 4}, {2, 16384, 2050},
                            {70, 8192, 515}, {5, 8192, 300}, {640, 4096, 2057}};
  for (const auto& c : cut) {
    CHECK(HeadForwardPlan<float>(c[0], c[1], c[2]).product.splits > 1, "fp32, %d rows, %d of %d", c[0], c[1], c[2]);
    CHECK(HeadForwardPlan<uint16_t>(c[0], c[1], c[2]).product.splits > 1, "bf16, %d rows, %d of %d", c[0], c[1], c[2]);
  }
  std::printf("no finding\n");
  return 0;
}
