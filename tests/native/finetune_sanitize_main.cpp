// Host-side exerciser for a sanitizer build (-fsanitize=address,undefined on the host pass) of
// hpd_finetune_host.cpp: random valid and broken batches through hpd_build_finetune_layout with HPD_FLAG_HOST_ONLY (no
// GPU call), every table read back into a buffer of exactly its size, the work lists checked, the argument checks of the
// calls.  The kernel launchers are stubbed out: nothing here may reach them.  Exit code 0 = no finding.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>

#include "hpd_finetune.h"
#include "hpd_internal.h"

static int g_stub_calls = 0;
#define STUB(...) { ++g_stub_calls; return hipErrorInvalidValue; }
int hpd_hip_fail(hipError_t) { ++g_stub_calls; return HPD_E_HIP; }
hipError_t hpd_launch_ft_rope_table(const hpd_finetune_layout*, hipStream_t) STUB()
hipError_t hpd_launch_ft_rotate(const hpd_finetune_layout*, bool, const void*, const void*, void*, void*,
                                const hpd_finetune_strides&, hipStream_t) STUB()
hipError_t hpd_launch_ft_attention(const hpd_finetune_layout*, const void*, const void*, const void*, void*, float*, void*,
                                   const hpd_finetune_strides&, hipStream_t) STUB()
hipError_t hpd_launch_ft_attention_backward(const hpd_finetune_layout*, const void*, const void*, const void*, const void*,
                                            const float*, const void*, void*, void*, void*, void*, const hpd_finetune_strides&,
                                            hipStream_t) STUB()
int64_t hpd_logprobs_bytes(int32_t, int64_t n, int32_t, int32_t) { return n; }
hipError_t hpd_launch_logprobs(int32_t, const hpd_logprobs_args&, hipStream_t) STUB()
hipError_t hpd_launch_logprobs_backward(int32_t, const hpd_logprobs_backward_args&, hipStream_t) STUB()

#define CHECK(cond)                                                          \
  do {                                                                       \
    if (!(cond)) {                                                           \
      std::fprintf(stderr, "CHECK failed at line %d: %s\n", __LINE__, #cond); \
      std::exit(1);                                                          \
    }                                                                        \
  } while (0)

static std::vector<int32_t> table(const hpd_finetune_layout* L, int32_t what, size_t n) {
  std::vector<int32_t> v(n);
  int32_t dummy;
  CHECK(hpd_finetune_layout_query(L, what, n ? (void*)v.data() : (void*)&dummy, n * 4) == HPD_OK);
  if (n > 0) CHECK(hpd_finetune_layout_query(L, what, v.data(), n * 4 - 1) == HPD_E_INVALID);
  return v;
}

// every 128 tokens of every sequence are one tile of queries, longest first
static void check_tiles(const hpd_finetune_layout* L, const std::vector<int32_t>& off) {
  size_t expect = 0;
  for (int32_t s = 0; s < L->n_seq; ++s) expect += (off[s + 1] - off[s] + 127) / 128;
  CHECK(L->tiles.size() == expect);
  std::map<std::pair<int32_t, int32_t>, int> seen;
  for (size_t i = 0; i < expect; ++i) {
    const hpd_ft_tile& a = L->tiles[i];
    CHECK(a.row0 < a.len && a.row0 % 128 == 0 && a.seq0 + a.len <= L->n_tokens);
    CHECK((size_t)(a.blk0 + (a.len + 31) / 32) * 2 <= L->blk_rank.size());
    seen[{a.seq0, a.row0}] += 1;
    if (i) CHECK(std::min(L->tiles[i - 1].row0 + 128, L->tiles[i - 1].len) >= std::min(a.row0 + 128, a.len));
  }
  for (const auto& x : seen) CHECK(x.second == 1);
}

// every word of a block's mask: bit i iff token i's rank is no higher
static void check_seen(const hpd_finetune_layout* L) {
  if (L->cfg.dtype != HPD_BF16) {
    CHECK(L->seen.empty() && L->seen_off.empty());
    return;
  }
  size_t words = 0, block = 0;
  for (int32_t s = 0; s < L->n_seq; ++s)
    for (int32_t b = L->seq_off[s]; b < L->seq_off[s + 1]; b += 32, ++block) {
      const int32_t lo = L->blk_rank[2 * block], hi = L->blk_rank[2 * block + 1];
      for (int32_t r = lo - 1; r <= hi; ++r, ++words) {
        uint32_t want = 0;
        for (int32_t i = b; i < std::min(b + 32, L->seq_off[s + 1]); ++i)
          if (L->rank[i] <= r) want |= 1u << (i - b);
        CHECK((size_t)(L->seen_off[block] + r) == words && L->seen[words] == want);
      }
    }
  CHECK(words == L->seen.size() && block == L->seen_off.size());
}

// the items of a tile are its rounds, each once, the longest items first; a tile of several has as many slots in a row
template <typename Rounds>
static void check_cut(const hpd_finetune_layout* L, int32_t rows_of, const std::vector<hpd_ft_item>& items,
                      const std::vector<hpd_ft_item>& join_list, int32_t n_slots, Rounds rounds) {
  size_t expect = 0;
  for (int32_t s = 0; s < L->n_seq; ++s) expect += (L->seq_off[s + 1] - L->seq_off[s] + rows_of - 1) / rows_of;
  std::map<std::pair<int32_t, int32_t>, std::map<int32_t, hpd_ft_item>> tiles;
  for (size_t i = 0; i < items.size(); ++i) {
    const hpd_ft_item& x = items[i];
    CHECK(x.begin < x.end && x.slot < n_slots && x.row0 < x.len && x.row0 % rows_of == 0 && x.seq0 + x.len <= L->n_tokens);
    if (i) CHECK(items[i - 1].end - items[i - 1].begin >= x.end - x.begin);
    int32_t plain = 0;
    while (plain < (x.len + 31) / 32 && L->blk_rank[2 * (x.blk0 + plain) + 1] == 0) ++plain;
    CHECK(x.plain == plain);
    const bool fresh = tiles[{x.seq0, x.row0}].emplace(x.begin, x).second;
    CHECK(fresh);
  }
  CHECK(tiles.size() == expect);
  std::map<std::pair<int32_t, int32_t>, hpd_ft_item> joins;
  int32_t slots = 0;
  for (const hpd_ft_item& x : join_list) {
    CHECK(joins.emplace(std::make_pair(x.seq0, x.row0), x).second);
    slots += x.end;
  }
  CHECK(slots == n_slots);
  for (const auto& t : tiles) {
    const hpd_ft_item& first = t.second.begin()->second;
    int64_t at = 0;
    const auto join = joins.find(t.first);
    CHECK((t.second.size() > 1) == (join != joins.end()));
    int32_t n = 0;
    for (const auto& x : t.second) {
      CHECK(x.second.begin == at);
      at = x.second.end;
      CHECK(x.second.slot == (join == joins.end() ? -1 : join->second.slot + n));
      ++n;
    }
    CHECK(at == rounds(first));
    if (join != joins.end()) CHECK(join->second.end == n);
  }
}
static void check_items(const hpd_finetune_layout* L) {
  const int64_t Hq = L->cfg.n_q_heads, Hkv = L->cfg.n_kv_heads, G = Hq / Hkv;
  const int32_t rows_of = hpd_ft_key_rows(L);
  check_cut(L, rows_of, L->items, L->joins, L->slots,
            [&](const hpd_ft_item& x) { return G * ((x.len + 31) / 32 - x.row0 / 32); });
  int64_t forward = 0;
  if (L->cfg.dtype == HPD_BF16) {
    check_cut(L, 128, L->query_items, L->query_joins, L->query_slots,
              [](const hpd_ft_item& x) { return (int64_t)(std::min(x.row0 + 128, x.len) + 63) / 64; });
    forward = (int64_t)L->query_slots * Hq * 128 * (hpd_ft_padded_dim(L) + 2) * 4;
  } else {
    CHECK(L->query_items.empty() && L->query_joins.empty() && L->query_slots == 0);
  }
  CHECK(hpd_ft_padded_dim(L) >= L->cfg.head_dim && hpd_ft_padded_dim(L) % 32 == 0);
  CHECK(hpd_ft_forward_bytes(L) == forward);
  const int64_t rows = (int64_t)L->n_tokens * Hq;
  CHECK(hpd_ft_backward_bytes(L) >= rows * 8 + (int64_t)L->slots * Hkv * 2 * rows_of * hpd_ft_padded_dim(L) * 4 + forward);
}

int main() {
  std::mt19937 rng(7);
  auto pick = [&](int32_t lo, int32_t hi) { return std::uniform_int_distribution<int32_t>(lo, hi)(rng); };
  bool cut = false, whole = false;
  for (int round = 0; round < 400; ++round) {
    hpd_finetune_config cfg{};
    cfg.n_kv_heads = pick(1, 8);
    cfg.n_q_heads = cfg.n_kv_heads * pick(1, 8);
    cfg.head_dim = round % 3 ? 64 * pick(1, 2) : 8 * pick(1, 16);
    cfg.dtype = pick(0, 3) ? HPD_BF16 : HPD_F32;
    cfg.rope_base = 10000.0;
    cfg.k_max = pick(1, 40);
    cfg.flags = HPD_FLAG_HOST_ONLY;
    const int32_t n_seq = pick(0, 6);
    std::vector<int32_t> prompt, attr_ptr{0}, attr_len, value_len;
    for (int32_t s = 0; s < n_seq; ++s) {
      prompt.push_back(pick(0, round % 7 == 0 ? 6000 : 300));
      const int32_t n = pick(0, 12);
      for (int32_t i = 0; i < n; ++i) {
        attr_len.push_back(pick(1, 4));
        value_len.push_back(pick(0, cfg.k_max));
      }
      attr_ptr.push_back((int32_t)attr_len.size());
    }
    // (copies of exactly the arrays' sizes: a read behind one is a finding)
    hpd_finetune_layout* L = nullptr;
    CHECK(hpd_build_finetune_layout(&cfg, n_seq, prompt.data(), attr_ptr.data(), attr_len.data(), value_len.data(), nullptr, &L) == HPD_OK);
    int64_t c[HPD_N_FT_COUNTS];
    CHECK(hpd_finetune_layout_query(L, HPD_FTQ_COUNTS, c, sizeof(c)) == HPD_OK);
    CHECK(hpd_finetune_layout_query(L, HPD_FTQ_COUNTS, c, sizeof(c) - 1) == HPD_E_INVALID);
    CHECK(hpd_finetune_layout_query(L, 17, c, sizeof(c)) == HPD_E_INVALID);
    const auto off = table(L, HPD_FTQ_SEQ_OFF, (size_t)n_seq + 1), pos = table(L, HPD_FTQ_POS, (size_t)c[HPD_FTC_N_TOKENS]),
               rank = table(L, HPD_FTQ_RANK, (size_t)c[HPD_FTC_N_TOKENS]);
    CHECK(off[n_seq] == c[HPD_FTC_N_TOKENS]);
    for (int32_t p : pos) CHECK(p >= 0 && p <= c[HPD_FTC_MAX_POS]);
    for (int32_t r : rank) CHECK(r >= 0 && r <= cfg.k_max);
    CHECK(L->rope_rows <= L->n_tokens && (L->rope_by_token ? L->rope_rows == L->n_tokens : L->rope_rows == c[HPD_FTC_MAX_POS] + 1));
    check_tiles(L, off);
    check_seen(L);
    check_items(L);
    cut = cut || !L->joins.empty();
    whole = whole || (L->joins.empty() && !L->items.empty());
    float x[4];
    CHECK(hpd_finetune_attention(L, x, x, x, x, x, x, nullptr, nullptr) == HPD_E_INVALID);  // not on the device
    hpd_finetune_layout_free(L);
    // one field broken
    hpd_finetune_config bad = cfg;
    switch (pick(0, 5)) {
      case 0: bad.n_q_heads = 0; break;
      case 1: bad.n_kv_heads = bad.n_q_heads + 1; break;
      case 2: bad.head_dim = 7; break;
      case 3: bad.k_max = 0; break;
      case 4: bad.dtype = 9; break;
      default: bad.rope_base = 0.5;
    }
    L = nullptr;
    CHECK(hpd_build_finetune_layout(&bad, n_seq, prompt.data(), attr_ptr.data(), attr_len.data(), value_len.data(), nullptr, &L) < 0);
    CHECK(L == nullptr);
    if (!value_len.empty()) {
      value_len[pick(0, (int32_t)value_len.size() - 1)] = pick(0, 1) ? -1 : cfg.k_max + 1;
      CHECK(hpd_build_finetune_layout(&cfg, n_seq, prompt.data(), attr_ptr.data(), attr_len.data(), value_len.data(), nullptr, &L) == HPD_E_INVALID);
    }
  }
  CHECK(cut && whole);
  hpd_finetune_layout_free(nullptr);
  CHECK(g_stub_calls == 0);
  std::puts("no finding");
  return 0;
}
