// Host side of the fine-tuning operators: validation, the tables of a batch of training sequences
// (Section 4.4, Appendix A.1) and the C ABI.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <stdexcept>

#include "hpd_finetune.h"
#include "hpd_internal.h"

namespace {

#define HPD_HIP(expr)                              \
  do {                                             \
    hipError_t e_ = (expr);                        \
    if (e_ != hipSuccess) return hpd_hip_fail(e_); \
  } while (0)

constexpr int64_t LIMIT = (int64_t)1 << 30;      // positions, a token's elements, rows and columns of logits
constexpr int64_t MAX_TOKENS = (int64_t)1 << 25;
constexpr int64_t MAX_ROWS = (int64_t)1 << 27;    // tokens times query heads
constexpr int64_t MAX_THREADS = ((int64_t)1 << 32) - 1;  // of a launch

int elem_bytes(int32_t dtype) { return dtype == HPD_F32 ? 4 : 2; }

int validate(const hpd_finetune_config* c) {
  if (!c) return HPD_E_INVALID;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads % c->n_kv_heads != 0) return HPD_E_INVALID;
  if (c->head_dim < 2 || (c->head_dim & 1) || c->k_max < 1) return HPD_E_INVALID;
  if (!(c->rope_base > 1.0) || !std::isfinite(c->rope_base)) return HPD_E_INVALID;
  if (c->flags & ~HPD_FLAG_HOST_ONLY) return HPD_E_INVALID;
  if (c->dtype != HPD_F32 && c->dtype != HPD_BF16) return HPD_E_UNSUPPORTED;
  if (c->head_dim % 8 != 0 || c->head_dim > HPD_FINETUNE_MAX_DIM) return HPD_E_UNSUPPORTED;
  if ((int64_t)c->n_q_heads * c->head_dim > LIMIT) return HPD_E_OVERFLOW;  // (a head's place in its token: 32 bits of bytes)
  return HPD_OK;
}

// Cuts tiles into items of about `most` rounds, longest first.
template <typename Rounds>
void cut(const std::vector<hpd_ft_tile>& tiles, const std::vector<int32_t>& plain, int64_t most, Rounds rounds,
         std::vector<hpd_ft_item>& items, std::vector<hpd_ft_item>& joins, int32_t& slots) {
  for (const hpd_ft_tile& t : tiles) {
    const int64_t r = rounds(t), parts = r * 2 > most * 3 ? (r + most - 1) / most : 1;
    if (parts > 1) joins.push_back({t.seq0, t.len, t.row0, t.blk0, 0, (int32_t)parts, slots, 0});
    for (int64_t p = 0; p < parts; ++p)
      items.push_back({t.seq0, t.len, t.row0, t.blk0, (int32_t)(r * p / parts), (int32_t)(r * (p + 1) / parts),
                       parts > 1 ? slots++ : -1, plain[(size_t)t.blk0]});
  }
  std::stable_sort(items.begin(), items.end(),
                   [](const hpd_ft_item& a, const hpd_ft_item& b) { return a.end - a.begin > b.end - b.begin; });
}

// The items of the kernels.  Two workgroups run on a CU at a time (one for fp32 with more than 64 channels).  A tile at
// the start of a long sequence has many times the rounds of others, and a batch may have fewer tiles than the GPU has room
// for: an item has at most a third of what a workgroup's place has to do (a half: 4045 -> 4140 us for the gradients of
// 2 x 6100 tokens, 64/8 heads).  It starts and ends with the time of four rounds, and its sums are written and read once more, so
// it has no fewer than four and those of a place, up to 64.  bf16 gradients of 50 random batches, geometric means over 24 rounds
// at least (64 where there are more tiles than places): 0.89; with three 0.89, six 0.91, with 0.6 or 1.5 times those of a place 0.90 and
// 0.91.  The queries, over whole tiles (of 50 random batches ten are cut): 0.98, up to 0.71 for a single sequence; with six or ten
// 0.985 and 0.99.  In fp32 the waves of a workgroup share the rounds, and a start is two of
// them: from two, up to 32 (30 random batches, over 16 at least: 0.946; from 4 or 8 on 0.966 and 0.99; not cut at all: 473 -> 89 us
// for a sequence of 774 tokens, 12/2 heads of 96).
void plan_items(hpd_finetune_layout* L, const std::vector<int32_t>& plain, int32_t n_cus) {
  const int64_t Hq = L->cfg.n_q_heads, Hkv = L->cfg.n_kv_heads, G = Hq / Hkv;
  const int32_t rows = hpd_ft_key_rows(L);
  const bool bf16 = L->cfg.dtype == HPD_BF16;
  std::vector<hpd_ft_tile> tiles;
  for (const hpd_ft_tile& t : L->tiles)
    for (int32_t r = t.row0; r < std::min(t.row0 + HPD_FT_ROWS, t.len); r += rows) tiles.push_back({t.seq0, t.len, r, t.blk0});
  const int64_t places = (bf16 || L->cfg.head_dim <= 64 ? 2 : 1) * n_cus;
  auto most = [&](int64_t total, int64_t start, int64_t cap) { return std::max(std::min(cap, start + total / places), total / places / 3); };
  auto key_rounds = [&](const hpd_ft_tile& t) { return G * ((t.len + 31) / 32 - t.row0 / 32); };
  auto query_rounds = [&](const hpd_ft_tile& t) { return (int64_t)(std::min(t.row0 + HPD_FT_ROWS, t.len) + 63) / 64; };
  int64_t total = 0;
  for (const hpd_ft_tile& t : tiles) total += key_rounds(t) * Hkv;
  cut(tiles, plain, bf16 ? most(total, 4, 64) : most(total, 2, 32), key_rounds, L->items, L->joins, L->slots);
  if (!bf16) return;
  total = 0;
  for (const hpd_ft_tile& t : L->tiles) total += query_rounds(t) * Hq;
  cut(L->tiles, plain, most(total, 4, 64), query_rounds, L->query_items, L->query_joins, L->query_slots);
}

// Positions (Algorithm 2, values at pos_id[end(a_n)] + k), ranks, rank ranges of blocks, work tiles.
int build_tables(hpd_finetune_layout* L, const int32_t* prompt_len, const int32_t* attr_ptr, const int32_t* attr_len,
                 const int32_t* value_len, int32_t n_cus) {
  const int64_t k_max = L->cfg.k_max;
  int64_t total = 0;
  for (int32_t s = 0; s < L->n_seq; ++s) {
    int64_t len = prompt_len[s];
    for (int32_t n = attr_ptr[s]; n < attr_ptr[s + 1]; ++n) len += (int64_t)attr_len[n] + value_len[n];
    if (len + (int64_t)(attr_ptr[s + 1] - attr_ptr[s]) * k_max > LIMIT) return HPD_E_OVERFLOW;
    total += len;
    if (total > MAX_TOKENS || total * L->cfg.n_q_heads > MAX_ROWS) return HPD_E_OVERFLOW;
  }
  L->n_tokens = (int32_t)total;
  L->seq_off.reserve((size_t)L->n_seq + 1);
  L->pos.resize((size_t)total);
  L->rank.assign((size_t)total, 0);
  L->seq_off.push_back(0);
  int32_t at = 0;
  std::vector<int32_t> plain;  // at a sequence's first block: how many from there on have nothing but rank 0
  for (int32_t s = 0; s < L->n_seq; ++s) {
    const int32_t seq0 = at;
    for (int32_t i = 0; i < prompt_len[s]; ++i) L->pos[at++] = i;
    int32_t next = prompt_len[s], offset = 0;  // position of the next name token: next + offset
    for (int32_t n = attr_ptr[s]; n < attr_ptr[s + 1]; ++n) {
      for (int32_t i = 0; i < attr_len[n]; ++i) L->pos[at++] = next++ + offset;
      for (int32_t k = 1; k <= value_len[n]; ++k, ++at) {
        L->pos[at] = next - 1 + offset + k;
        L->rank[at] = k;
      }
      offset += L->cfg.k_max;
    }
    const int32_t len = at - seq0;
    L->seq_off.push_back(at);
    L->max_len = std::max(L->max_len, len);
    const int32_t blk0 = (int32_t)(L->blk_rank.size() / 2);
    for (int32_t b = 0; b < len; b += HPD_FT_BLOCK) {
      const auto mm = std::minmax_element(L->rank.begin() + seq0 + b, L->rank.begin() + seq0 + std::min(b + HPD_FT_BLOCK, len));
      L->blk_rank.push_back(*mm.first);
      L->blk_rank.push_back(*mm.second);
      plain.push_back(0);
      if (*mm.second == 0 && plain[(size_t)blk0] * HPD_FT_BLOCK == b) ++plain[(size_t)blk0];
      if (L->cfg.dtype != HPD_BF16) continue;
      const size_t at = L->seen.size();
      L->seen_off.push_back((int32_t)at - (*mm.first - 1));
      L->seen.resize(at + (size_t)(*mm.second - *mm.first + 2), 0);
      for (int32_t i = b; i < std::min(b + HPD_FT_BLOCK, len); ++i)
        L->seen[at + (size_t)(L->rank[seq0 + i] - *mm.first + 1)] |= 1u << (i - b);
      for (size_t r = at + 1; r < L->seen.size(); ++r) L->seen[r] |= L->seen[r - 1];
    }
    for (int32_t r = 0; r < len; r += HPD_FT_ROWS) L->tiles.push_back({seq0, len, r, blk0});
  }
  for (int32_t p : L->pos) L->max_pos = std::max(L->max_pos, p);
  // Longest first: what starts last is short.  A tile of queries has keys up to its last row.
  std::stable_sort(L->tiles.begin(), L->tiles.end(), [](const hpd_ft_tile& a, const hpd_ft_tile& b) {
    return std::min(a.row0 + HPD_FT_ROWS, a.len) > std::min(b.row0 + HPD_FT_ROWS, b.len);
  });
  plan_items(L, plain, n_cus);
  // (MAX_TOKENS and MAX_ROWS are enough for the kernels that go by tokens, and few tiles are cut and joined)
  if (std::max(hpd_ft_query_groups(L), hpd_ft_key_groups(L)) * 256 > MAX_THREADS) return HPD_E_OVERFLOW;
  L->rope_by_token = L->max_pos >= L->n_tokens;
  L->rope_rows = L->rope_by_token ? L->n_tokens : L->max_pos + 1;
  return HPD_OK;
}

int upload(hpd_finetune_layout* L, hipStream_t s) {
  // one allocation: tables, then the (cos, sin) rows, which a kernel writes
  auto pad = [](size_t words) { return (words + 3) / 4 * 4; };
  // (the kernels read the ranks of two whole blocks at a time: up to 63 more behind the last token)
  const size_t n = (size_t)L->n_tokens, nt = L->tiles.size() * 4;
  const size_t o_rank = pad(n), o_blk = o_rank + pad(n + 2 * HPD_FT_BLOCK), o_seen_off = o_blk + pad(L->blk_rank.size()),
               o_seen = o_seen_off + pad(L->seen_off.size()), o_tiles = o_seen + pad(L->seen.size()),
               o_items = o_tiles + nt;
  const std::vector<hpd_ft_item>* const lists[] = {&L->items, &L->joins, &L->query_items, &L->query_joins};
  size_t words = o_items;
  for (const auto* l : lists) words += l->size() * 8;
  std::vector<int32_t> host(words, 0);
  std::copy(L->pos.begin(), L->pos.end(), host.begin());
  std::copy(L->rank.begin(), L->rank.end(), host.begin() + o_rank);
  std::copy(L->blk_rank.begin(), L->blk_rank.end(), host.begin() + o_blk);
  std::copy(L->seen_off.begin(), L->seen_off.end(), host.begin() + o_seen_off);
  std::copy(L->seen.begin(), L->seen.end(), host.begin() + o_seen);
  std::memcpy(host.data() + o_tiles, L->tiles.data(), nt * 4);
  size_t at = o_items;
  for (const auto* l : lists) {
    if (!l->empty()) std::memcpy(host.data() + at, l->data(), l->size() * sizeof(hpd_ft_item));
    at += l->size() * 8;
  }
  const size_t rope_bytes = (size_t)L->rope_rows * (size_t)(L->cfg.head_dim / 2) * sizeof(float2);
  HPD_HIP(hipMalloc(&L->d_mem, words * 4 + rope_bytes));
  const int32_t* base = (const int32_t*)L->d_mem;
  L->d_pos = base;
  L->d_rank = base + o_rank;
  L->d_blk_rank = (const int2*)(base + o_blk);
  L->d_seen_off = base + o_seen_off;
  L->d_seen = (const uint32_t*)(base + o_seen);
  L->d_tiles = (const hpd_ft_tile*)(base + o_tiles);
  L->d_items = (const hpd_ft_item*)(base + o_items);
  L->d_joins = L->d_items + L->items.size();
  L->d_query_items = L->d_joins + L->joins.size();
  L->d_query_joins = L->d_query_items + L->query_items.size();
  L->d_rope = (float2*)(base + words);
  HPD_HIP(hipMemcpyAsync(L->d_mem, host.data(), words * 4, hipMemcpyHostToDevice, s));
  hipError_t e = hpd_launch_ft_rope_table(L, s);
  const hipError_t done = hipStreamSynchronize(s);  // (also after a failed launch: `host` is being read)
  if (e == hipSuccess) e = done;
  if (e != hipSuccess) return hpd_hip_fail(e);
  return HPD_OK;
}

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Fills in the distances that are 0; false if one is too short or no multiple of 16 bytes.
bool complete(const hpd_finetune_layout* L, const hpd_finetune_strides* in, hpd_finetune_strides* out) {
  *out = in ? *in : hpd_finetune_strides{0, 0, 0, 0, 0, 0};
  const int64_t D = L->cfg.head_dim, eb = elem_bytes(L->cfg.dtype);
  bool ok = true;
  auto one = [&](int64_t& x, int64_t heads) {
    if (x == 0) x = heads * D;
    ok = ok && x >= heads * D && x <= (int64_t)1 << 40 && x * eb % 16 == 0;
  };
  const int64_t hq = L->cfg.n_q_heads, hkv = L->cfg.n_kv_heads;
  one(out->q, hq); one(out->q_out, hq);
  one(out->k, hkv); one(out->k_out, hkv);
  one(out->v, hkv); one(out->v_out, hkv);
  return ok;
}

int check_logits(int32_t dtype, int64_t n_rows, int32_t vocab) {
  if (dtype != HPD_F32 && dtype != HPD_BF16) return HPD_E_UNSUPPORTED;
  if (n_rows < 0 || vocab < 1) return HPD_E_INVALID;
  if (n_rows > LIMIT || vocab > LIMIT) return HPD_E_OVERFLOW;
  return HPD_OK;
}

}  // namespace

// partial results of the queries: sums, and two numbers per token
int64_t hpd_ft_forward_bytes(const hpd_finetune_layout* L) {
  return (int64_t)L->query_slots * L->cfg.n_q_heads * HPD_FT_ROWS * (hpd_ft_padded_dim(L) + 2) * 4;
}
// two numbers per (head, token), then the partial sums of dk and dv, then those of dq
int64_t hpd_ft_backward_bytes(const hpd_finetune_layout* L) {
  const int64_t rows = (int64_t)L->n_tokens * L->cfg.n_q_heads;
  return (rows * 8 + 15) / 16 * 16 + (int64_t)L->slots * L->cfg.n_kv_heads * 2 * hpd_ft_key_rows(L) * hpd_ft_padded_dim(L) * 4 +
         hpd_ft_forward_bytes(L);
}

extern "C" {

int hpd_build_finetune_layout(const hpd_finetune_config* cfg, int32_t n_seq, const int32_t* prompt_len,
                              const int32_t* attr_ptr, const int32_t* attr_len, const int32_t* value_len,
                              void* stream, hpd_finetune_layout** out) {
  if (!out) return HPD_E_INVALID;
  int rc = validate(cfg);
  if (rc != HPD_OK) return rc;
  if (n_seq < 0 || (n_seq > 0 && (!prompt_len || !attr_ptr))) return HPD_E_INVALID;
  if (n_seq > 0 && attr_ptr[0] != 0) return HPD_E_INVALID;
  for (int32_t s = 0; s < n_seq; ++s)
    if (prompt_len[s] < 0 || attr_ptr[s + 1] < attr_ptr[s]) return HPD_E_INVALID;
  const int32_t n_attr = n_seq ? attr_ptr[n_seq] : 0;
  if (n_attr > 0 && (!attr_len || !value_len)) return HPD_E_INVALID;
  for (int32_t n = 0; n < n_attr; ++n)
    if (attr_len[n] < 1 || value_len[n] < 0 || value_len[n] > cfg->k_max) return HPD_E_INVALID;
  hpd_finetune_layout* L = nullptr;
  try {
    L = new hpd_finetune_layout();
    L->cfg = *cfg;
    L->n_seq = n_seq;
    int32_t n_cus = 256, device = 0;
    if (!(cfg->flags & HPD_FLAG_HOST_ONLY)) {
      hipError_t e = hipGetDevice(&device);
      if (e == hipSuccess) e = hipDeviceGetAttribute(&n_cus, hipDeviceAttributeMultiprocessorCount, device);
      if (e != hipSuccess) rc = hpd_hip_fail(e);
    }
    if (rc == HPD_OK) rc = build_tables(L, prompt_len, attr_ptr, attr_len, value_len, n_cus);
    if (rc == HPD_OK && !(cfg->flags & HPD_FLAG_HOST_ONLY)) {
      if (L->n_tokens > 0) rc = upload(L, (hipStream_t)stream);
      L->on_device = rc == HPD_OK;
    }
  } catch (const std::bad_alloc&) {
    rc = HPD_E_NOMEM;
  } catch (const std::length_error&) {
    rc = HPD_E_NOMEM;
  }
  if (rc != HPD_OK) {
    hpd_finetune_layout_free(L);
    return rc;
  }
  *out = L;
  return HPD_OK;
}

void hpd_finetune_layout_free(hpd_finetune_layout* L) {
  if (!L) return;
  if (L->d_mem) (void)hipFree(L->d_mem);
  delete L;
}

int hpd_finetune_layout_query(const hpd_finetune_layout* L, int32_t what, void* host_out, size_t bytes) {
  if (!L || !host_out) return HPD_E_INVALID;
  auto copy = [&](const std::vector<int32_t>& v) -> int {
    if (bytes < v.size() * sizeof(int32_t)) return HPD_E_INVALID;
    if (!v.empty()) std::memcpy(host_out, v.data(), v.size() * sizeof(int32_t));
    return HPD_OK;
  };
  switch (what) {
    case HPD_FTQ_COUNTS: {
      if (bytes < HPD_N_FT_COUNTS * sizeof(int64_t)) return HPD_E_INVALID;
      int64_t c[HPD_N_FT_COUNTS];
      c[HPD_FTC_N_SEQ] = L->n_seq; c[HPD_FTC_N_TOKENS] = L->n_tokens;
      c[HPD_FTC_MAX_LEN] = L->max_len; c[HPD_FTC_MAX_POS] = L->max_pos;
      c[HPD_FTC_FORWARD_BYTES] = hpd_ft_forward_bytes(L); c[HPD_FTC_BACKWARD_BYTES] = hpd_ft_backward_bytes(L);
      std::memcpy(host_out, c, sizeof(c));
      return HPD_OK;
    }
    case HPD_FTQ_SEQ_OFF: return copy(L->seq_off);
    case HPD_FTQ_POS: return copy(L->pos);
    case HPD_FTQ_RANK: return copy(L->rank);
    default: return HPD_E_INVALID;
  }
}

int hpd_finetune_rotate(const hpd_finetune_layout* L, int32_t inverse, const void* q, const void* k, void* q_out,
                        void* k_out, const hpd_finetune_strides* strides, void* stream) {
  if (!L || !L->on_device) return HPD_E_INVALID;
  hpd_finetune_strides st;
  if (!complete(L, strides, &st)) return HPD_E_INVALID;
  if (L->n_tokens == 0) return HPD_OK;
  for (const void* p : {q, k, (const void*)q_out, (const void*)k_out})
    if (!p || !aligned(p)) return HPD_E_INVALID;
  // in place: a token's wave has read what it writes, but not what other tokens' waves read
  if ((q_out == q && st.q_out != st.q) || (k_out == k && st.k_out != st.k)) return HPD_E_INVALID;
  HPD_HIP(hpd_launch_ft_rotate(L, inverse != 0, q, k, q_out, k_out, st, (hipStream_t)stream));
  return HPD_OK;
}

int hpd_finetune_attention(const hpd_finetune_layout* L, const void* q, const void* k, const void* v, void* out,
                           float* lse, void* workspace, const hpd_finetune_strides* strides, void* stream) {
  if (!L || !L->on_device) return HPD_E_INVALID;
  hpd_finetune_strides st;
  if (!complete(L, strides, &st)) return HPD_E_INVALID;
  if (L->n_tokens == 0) return HPD_OK;
  for (const void* p : {q, k, v, (const void*)out})
    if (!p || !aligned(p)) return HPD_E_INVALID;
  if (!lse || ((uintptr_t)lse & 3)) return HPD_E_INVALID;
  if ((hpd_ft_forward_bytes(L) && !workspace) || !aligned(workspace)) return HPD_E_INVALID;
  HPD_HIP(hpd_launch_ft_attention(L, q, k, v, out, lse, workspace, st, (hipStream_t)stream));
  return HPD_OK;
}

int hpd_finetune_attention_backward(const hpd_finetune_layout* L, const void* q, const void* k, const void* v,
                                    const void* out, const float* lse, const void* d_out, void* dq, void* dk, void* dv,
                                    void* workspace, const hpd_finetune_strides* strides, void* stream) {
  if (!L || !L->on_device) return HPD_E_INVALID;
  hpd_finetune_strides st;
  if (!complete(L, strides, &st)) return HPD_E_INVALID;
  if (L->n_tokens == 0) return HPD_OK;
  for (const void* p : {q, k, v, out, d_out, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!p || !aligned(p)) return HPD_E_INVALID;
  if (!lse || ((uintptr_t)lse & 3)) return HPD_E_INVALID;
  if ((hpd_ft_backward_bytes(L) && !workspace) || !aligned(workspace)) return HPD_E_INVALID;
  HPD_HIP(hpd_launch_ft_attention_backward(L, q, k, v, out, lse, d_out, dq, dk, dv, workspace, st, (hipStream_t)stream));
  return HPD_OK;
}

int hpd_token_logprobs_workspace(int32_t dtype, int64_t n_rows, int32_t vocab, int32_t top_k, int64_t* bytes) {
  if (!bytes) return HPD_E_INVALID;
  const int rc = check_logits(dtype, n_rows, vocab);
  if (rc != HPD_OK) return rc;
  if (top_k < 0 || top_k > HPD_MAX_TOP || top_k > vocab) return HPD_E_INVALID;
  *bytes = n_rows == 0 ? 0 : hpd_logprobs_bytes(dtype, n_rows, vocab, top_k);
  return HPD_OK;
}

int hpd_token_logprobs(int32_t dtype, int64_t n_rows, int32_t vocab, int64_t row_stride, const void* logits,
                       const int32_t* targets, int32_t top_k, float* logprob, float* lse, float* entropy,
                       int32_t* top_id, float* top_logprob, void* workspace, void* stream) {
  int64_t bytes = 0;
  const int rc = hpd_token_logprobs_workspace(dtype, n_rows, vocab, top_k, &bytes);
  if (rc != HPD_OK) return rc;
  if (row_stride < vocab) return HPD_E_INVALID;
  if (row_stride > LIMIT) return HPD_E_OVERFLOW;
  if (n_rows == 0) return HPD_OK;
  if (!logits || ((uintptr_t)logits & (elem_bytes(dtype) - 1))) return HPD_E_INVALID;
  if (top_k > 0 && (!top_id || !top_logprob)) return HPD_E_INVALID;
  if ((bytes && !workspace) || !aligned(workspace)) return HPD_E_INVALID;
  HPD_HIP(hpd_launch_logprobs(dtype, {n_rows, row_stride, vocab, top_k, logits, targets, logprob, lse, entropy, top_id,
                                      top_logprob, workspace}, (hipStream_t)stream));
  return HPD_OK;
}

int hpd_token_logprobs_backward(int32_t dtype, int64_t n_rows, int32_t vocab, int64_t row_stride, const void* logits,
                                const int32_t* targets, const float* lse, const float* entropy, const float* g_logprob,
                                const float* g_entropy, void* d_logits, int64_t d_stride, void* stream) {
  const int rc = check_logits(dtype, n_rows, vocab);
  if (rc != HPD_OK) return rc;
  if (row_stride < vocab || d_stride < vocab) return HPD_E_INVALID;
  if (row_stride > LIMIT || d_stride > LIMIT) return HPD_E_OVERFLOW;
  if (n_rows == 0) return HPD_OK;
  const uintptr_t eb = (uintptr_t)elem_bytes(dtype);
  if (!logits || !d_logits || !lse || (((uintptr_t)logits | (uintptr_t)d_logits) & (eb - 1))) return HPD_E_INVALID;
  if (g_logprob && !targets) return HPD_E_INVALID;
  if (g_entropy && !entropy) return HPD_E_INVALID;
  if (d_logits == logits && d_stride != row_stride) return HPD_E_INVALID;
  HPD_HIP(hpd_launch_logprobs_backward(dtype, {n_rows, row_stride, d_stride, vocab, logits, targets, lse, entropy,
                                               g_logprob, g_entropy, d_logits}, (hipStream_t)stream));
  return HPD_OK;
}

}  // extern "C"
