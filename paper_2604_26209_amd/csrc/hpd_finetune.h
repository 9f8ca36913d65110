// Internal declarations of the fine-tuning operators: the layout of a batch of training sequences and
// the kernel launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

#include "hpd.h"

constexpr int32_t HPD_FT_ROWS = 128;  // tokens of a work tile of the attention kernels
constexpr int32_t HPD_FT_BLOCK = 32;  // tokens of a block that has its own rank range

// One work tile: HPD_FT_ROWS tokens of a sequence.
struct hpd_ft_tile {
  int32_t seq0;  // first token of the sequence
  int32_t len;   // tokens of the sequence
  int32_t row0;  // first token of the tile, counted in the sequence
  int32_t blk0;  // the sequence's first entry in blk_rank
};

// A run of the rounds of a tile: for one of keys and a kv head, 32 queries of one head each, head by head; for one of
// queries and a head, 64 keys each.
struct hpd_ft_item {
  int32_t seq0, len, row0, blk0;  // of the tile
  int32_t begin, end;             // rounds
  int32_t slot;                   // partial sums, or -1: the item is the whole tile
  int32_t plain;                  // leading blocks of the sequence with nothing but rank 0
};

struct hpd_finetune_layout {
  hpd_finetune_config cfg;
  int32_t n_seq = 0, n_tokens = 0, max_len = 0, max_pos = -1;
  std::vector<int32_t> seq_off, pos, rank;
  std::vector<int32_t> blk_rank;        // [blocks][2]: lowest and highest rank of 32 tokens of a sequence
  // bf16: which tokens of a block have ranks up to r, for r from one below its lowest (none) to its highest rank (all); seen_off
  // [block] + r: the index of the word.  A block where a value of L tokens ends has L and two words, others 33 at most.
  std::vector<uint32_t> seen;
  std::vector<int32_t> seen_off;
  std::vector<hpd_ft_tile> tiles;       // query tiles, those with most keys first
  // the tiles of keys and (bf16) of queries as items, longest first, and for those of several items the first slot and (as
  // `end`) their number
  std::vector<hpd_ft_item> items, joins, query_items, query_joins;
  int32_t slots = 0, query_slots = 0;

  bool on_device = false;
  void* d_mem = nullptr;
  const int32_t *d_pos = nullptr, *d_rank = nullptr;
  const int2* d_blk_rank = nullptr;
  const int32_t* d_seen_off = nullptr;
  const uint32_t* d_seen = nullptr;
  const hpd_ft_tile* d_tiles = nullptr;
  const hpd_ft_item *d_items = nullptr, *d_joins = nullptr, *d_query_items = nullptr, *d_query_joins = nullptr;
  // (cos, sin) rows of D/2: one per position ID, or one per token where that is fewer
  float2* d_rope = nullptr;
  int32_t rope_rows = 0;
  bool rope_by_token = false;
};

// Tokens of a tile of keys, and channels that the kernels are made for.
inline int32_t hpd_ft_key_rows(const hpd_finetune_layout* L) { return L->cfg.dtype == HPD_BF16 ? HPD_FT_ROWS : HPD_FT_BLOCK; }
inline int32_t hpd_ft_padded_dim(const hpd_finetune_layout* L) {
  const int32_t d = (L->cfg.head_dim + 31) / 32 * 32;
  return L->cfg.dtype == HPD_F32 && d < 64 ? 64 : d;
}
// Workgroups of 256 threads of the kernels that go by queries and of those that go by keys.
inline int64_t hpd_ft_query_groups(const hpd_finetune_layout* L) {
  return (int64_t)(L->cfg.dtype == HPD_BF16 ? L->query_items.size() : L->tiles.size() * (HPD_FT_ROWS / HPD_FT_BLOCK)) * L->cfg.n_q_heads;
}
inline int64_t hpd_ft_key_groups(const hpd_finetune_layout* L) { return (int64_t)L->items.size() * L->cfg.n_kv_heads; }
// Bytes of the calls' workspaces.
int64_t hpd_ft_forward_bytes(const hpd_finetune_layout* L);
int64_t hpd_ft_backward_bytes(const hpd_finetune_layout* L);

hipError_t hpd_launch_ft_rope_table(const hpd_finetune_layout* L, hipStream_t s);
// strides: complete (no zeros)
hipError_t hpd_launch_ft_rotate(const hpd_finetune_layout* L, bool inverse, const void* q, const void* k, void* q_out,
                                void* k_out, const hpd_finetune_strides& st, hipStream_t s);
hipError_t hpd_launch_ft_attention(const hpd_finetune_layout* L, const void* q, const void* k, const void* v, void* out,
                                   float* lse, void* workspace, const hpd_finetune_strides& st, hipStream_t s);
hipError_t hpd_launch_ft_attention_backward(const hpd_finetune_layout* L, const void* q, const void* k, const void* v,
                                            const void* out, const float* lse, const void* d_out, void* dq, void* dk,
                                            void* dv, void* workspace, const hpd_finetune_strides& st, hipStream_t s);

// Token log probabilities (hpd_logprobs.hip): workgroups that share a row, and the bytes they need for it.
struct hpd_logprobs_plan {
  int32_t parts;  // pieces a row is cut into
  int32_t span;   // logits of a piece (the last one may have fewer)
  int32_t waves;  // waves that share a piece: 4, or 1 (four rows per workgroup)
};
hpd_logprobs_plan hpd_plan_logprobs(int32_t dtype, int64_t n_rows, int32_t vocab);
int64_t hpd_logprobs_bytes(int32_t dtype, int64_t n_rows, int32_t vocab, int32_t top_k);

struct hpd_logprobs_args {
  int64_t n_rows, row_stride;
  int32_t vocab, top_k;
  const void* logits;
  const int32_t* targets;
  float *logprob, *lse, *entropy;
  int32_t* top_id;
  float* top_logprob;
  void* workspace;
};
hipError_t hpd_launch_logprobs(int32_t dtype, const hpd_logprobs_args& a, hipStream_t s);

struct hpd_logprobs_backward_args {
  int64_t n_rows, row_stride, d_stride;
  int32_t vocab;
  const void* logits;
  const int32_t* targets;
  const float *lse, *entropy, *g_logprob, *g_entropy;
  void* d_logits;
};
hipError_t hpd_launch_logprobs_backward(int32_t dtype, const hpd_logprobs_backward_args& a, hipStream_t s);
