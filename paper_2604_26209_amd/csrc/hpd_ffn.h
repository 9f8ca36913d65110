// Internal declarations of the gated feed-forward block and of the vocabulary head: plans and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hpd.h"

// ---- gated feed-forward block (hpd_ffn.hip).  Strides in elements, complete (no zeros).
struct hpd_ffn_forward_args {
  hpd_ffn_config cfg;
  int64_t n_rows;
  const void *x, *w_gate, *w_up, *w_down;
  void *out, *gate, *up;
  char* workspace;
  hpd_ffn_strides st;
};
struct hpd_ffn_backward_args {
  hpd_ffn_config cfg;
  int64_t n_rows;
  const void *x, *w_gate, *w_up, *w_down, *gate, *up, *d_out;
  void *d_x, *d_w_gate, *d_w_up, *d_w_down;
  char* workspace;
  hpd_ffn_strides st;
};
int64_t hpd_ffn_forward_bytes(const hpd_ffn_config& cfg, int64_t n_rows);
int64_t hpd_ffn_backward_bytes(const hpd_ffn_config& cfg, int64_t n_rows);
hipError_t hpd_launch_ffn(const hpd_ffn_forward_args& a, hipStream_t s);
hipError_t hpd_launch_ffn_backward(const hpd_ffn_backward_args& a, hipStream_t s);

// ---- vocabulary head (hpd_head.hip).  Strides in elements.
struct hpd_head_args {
  int32_t dtype;
  int64_t n_rows;
  int32_t width, vocab;
  const void *hidden, *weight;
  int64_t hidden_stride, weight_stride;
  const int32_t* targets;
  float *logprob, *lse, *entropy;
  char* workspace;
};
struct hpd_head_backward_args {
  int32_t dtype;
  int64_t n_rows;
  int32_t width, vocab;
  const void *hidden, *weight;
  int64_t hidden_stride, weight_stride;
  const int32_t* targets;
  const float *lse, *entropy, *g_logprob, *g_entropy;
  void *d_hidden, *d_weight;
  int64_t d_hidden_stride, d_weight_stride;
  char* workspace;
};
int64_t hpd_head_forward_bytes(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab);
int64_t hpd_head_backward_bytes(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab);
hipError_t hpd_launch_head(const hpd_head_args& a, hipStream_t s);
hipError_t hpd_launch_head_backward(const hpd_head_backward_args& a, hipStream_t s);
