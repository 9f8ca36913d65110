// Host side of the feed-forward block and of the vocabulary head: validation and the C ABI.
#include <initializer_list>

#include "hpd_ffn.h"
#include "hpd_internal.h"

namespace {

#define HPD_HIP(expr)                              \
  do {                                             \
    hipError_t e_ = (expr);                        \
    if (e_ != hipSuccess) return hpd_hip_fail(e_); \
  } while (0)

constexpr int64_t MAX_ROWS = (int64_t)1 << 30, MAX_SIZE = (int64_t)1 << 30;
constexpr int64_t MAX_STRIDE_BYTES = (int64_t)1 << 23;  // 256 rows of a tile from its first: 31 bits
constexpr int64_t MAX_TILES = (int64_t)1 << 22;         // of 128 rows and 64 features: a launch stays under 2^32 threads

int64_t elem_bytes(int32_t dtype) { return dtype == HPD_F32 ? 4 : 2; }
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

// `size`: the wider side of the rows' products
int check_rows(int64_t n_rows, int64_t size) {
  if (n_rows < 0) return HPD_E_INVALID;
  if (n_rows > MAX_ROWS || size > MAX_SIZE || ((n_rows + 127) / 128) * ((size + 63) / 64) > MAX_TILES) return HPD_E_OVERFLOW;
  return HPD_OK;
}

// 0 becomes the row's elements
int check_stride(int64_t& stride, int64_t elements, int32_t dtype) {
  if (stride == 0) stride = elements;
  if (stride < elements || stride > MAX_SIZE || stride * elem_bytes(dtype) % 16 != 0) return HPD_E_INVALID;
  return stride * elem_bytes(dtype) > MAX_STRIDE_BYTES ? HPD_E_OVERFLOW : HPD_OK;
}

bool distinct(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (const void* const* o = outputs.begin(); o != outputs.end(); ++o) {
    if (!*o) continue;
    for (const void* i : inputs)
      if (*o == i) return false;
    for (const void* const* other = outputs.begin(); other != o; ++other)
      if (*o == *other) return false;
  }
  return true;
}

int check_ffn(const hpd_ffn_config* c, int64_t n_rows) {
  if (!c || c->width < 1 || c->inner < 1) return HPD_E_INVALID;
  if (c->dtype != HPD_F32 && c->dtype != HPD_BF16) return HPD_E_UNSUPPORTED;
  if (c->activation < HPD_ACT_SILU || c->activation > HPD_ACT_GELU_TANH) return HPD_E_UNSUPPORTED;
  if (c->width % 8 != 0 || c->inner % 8 != 0) return HPD_E_UNSUPPORTED;
  const int64_t widest = 2 * (int64_t)(c->width > c->inner ? c->width : c->inner);
  if (widest * elem_bytes(c->dtype) > MAX_STRIDE_BYTES) return HPD_E_OVERFLOW;
  if (((widest + 127) / 128) * ((widest + 63) / 64) > MAX_TILES) return HPD_E_OVERFLOW;  // (the weights' gradients)
  return check_rows(n_rows, widest);
}

int complete(const hpd_ffn_config& c, const hpd_ffn_strides* in, hpd_ffn_strides* st) {
  *st = in ? *in : hpd_ffn_strides{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  int worst = HPD_OK;
  for (int64_t* s : {&st->x, &st->out, &st->w_gate, &st->w_up, &st->d_out, &st->d_x, &st->d_w_gate, &st->d_w_up}) {
    const int rc = check_stride(*s, c.width, c.dtype);
    if (worst == HPD_OK) worst = rc;
  }
  for (int64_t* s : {&st->gate, &st->up, &st->w_down, &st->d_w_down}) {
    const int rc = check_stride(*s, c.inner, c.dtype);
    if (worst == HPD_OK) worst = rc;
  }
  return worst;
}

int check_head(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab) {
  if (dtype != HPD_F32 && dtype != HPD_BF16) return HPD_E_UNSUPPORTED;
  if (width < 1 || vocab < 1) return HPD_E_INVALID;
  if (width % 8 != 0) return HPD_E_UNSUPPORTED;
  if (((int64_t)vocab + 127) / 128 * ((width + 63) / 64) > MAX_TILES) return HPD_E_OVERFLOW;
  return check_rows(n_rows, vocab > width ? vocab : width);
}

}  // namespace

extern "C" {

int hpd_gated_ffn_workspace(const hpd_ffn_config* cfg, int64_t n_rows, int64_t* forward_bytes, int64_t* backward_bytes) {
  const int rc = check_ffn(cfg, n_rows);
  if (rc != HPD_OK) return rc;
  if (forward_bytes) *forward_bytes = n_rows ? hpd_ffn_forward_bytes(*cfg, n_rows) : 0;
  if (backward_bytes) *backward_bytes = n_rows ? hpd_ffn_backward_bytes(*cfg, n_rows) : 0;
  return HPD_OK;
}

int hpd_gated_ffn(const hpd_ffn_config* cfg, int64_t n_rows, const void* x, const void* w_gate, const void* w_up,
                  const void* w_down, void* out, void* gate, void* up, void* workspace, const hpd_ffn_strides* strides,
                  void* stream) {
  int rc = check_ffn(cfg, n_rows);
  if (rc != HPD_OK) return rc;
  hpd_ffn_forward_args a = {*cfg, n_rows, x, w_gate, w_up, w_down, out, gate, up, (char*)workspace, {}};
  rc = complete(*cfg, strides, &a.st);
  if (rc != HPD_OK || n_rows == 0) return rc;
  for (const void* p : {x, w_gate, w_up, w_down, (const void*)out, (const void*)workspace})
    if (!p || !aligned(p)) return HPD_E_INVALID;
  if (!aligned(gate) || !aligned(up)) return HPD_E_INVALID;
  if (!distinct({out, gate, up, workspace}, {x, w_gate, w_up, w_down})) return HPD_E_INVALID;
  HPD_HIP(hpd_launch_ffn(a, (hipStream_t)stream));
  return HPD_OK;
}

int hpd_gated_ffn_backward(const hpd_ffn_config* cfg, int64_t n_rows, const void* x, const void* w_gate, const void* w_up,
                           const void* w_down, const void* gate, const void* up, const void* d_out, void* d_x, void* d_w_gate,
                           void* d_w_up, void* d_w_down, void* workspace, const hpd_ffn_strides* strides, void* stream) {
  int rc = check_ffn(cfg, n_rows);
  if (rc != HPD_OK) return rc;
  hpd_ffn_backward_args a = {*cfg, n_rows, x, w_gate, w_up, w_down, gate, up, d_out, d_x, d_w_gate, d_w_up, d_w_down,
                             (char*)workspace, {}};
  rc = complete(*cfg, strides, &a.st);
  if (rc != HPD_OK) return rc;
  for (const void* p : {(const void*)d_x, (const void*)d_w_gate, (const void*)d_w_up, (const void*)d_w_down})
    if (!aligned(p)) return HPD_E_INVALID;
  if (n_rows > 0)
    for (const void* p : {x, w_gate, w_up, w_down, gate, up, d_out, (const void*)workspace})
      if (!p || !aligned(p)) return HPD_E_INVALID;
  if (!distinct({d_x, d_w_gate, d_w_up, d_w_down, workspace}, {x, w_gate, w_up, w_down, gate, up, d_out})) return HPD_E_INVALID;
  if (!d_x && !d_w_gate && !d_w_up && !d_w_down) return HPD_OK;
  HPD_HIP(hpd_launch_ffn_backward(a, (hipStream_t)stream));
  return HPD_OK;
}

int hpd_head_logprobs_workspace(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab, int64_t* forward_bytes,
                                int64_t* backward_bytes) {
  const int rc = check_head(dtype, n_rows, width, vocab);
  if (rc != HPD_OK) return rc;
  if (forward_bytes) *forward_bytes = n_rows ? hpd_head_forward_bytes(dtype, n_rows, width, vocab) : 0;
  if (backward_bytes) *backward_bytes = n_rows ? hpd_head_backward_bytes(dtype, n_rows, width, vocab) : 0;
  return HPD_OK;
}

int hpd_head_logprobs(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab, const void* hidden, int64_t hidden_stride,
                      const void* weight, int64_t weight_stride, const int32_t* targets, float* logprob, float* lse,
                      float* entropy, void* workspace, void* stream) {
  int rc = check_head(dtype, n_rows, width, vocab);
  for (int64_t* s : {&hidden_stride, &weight_stride})
    if (rc == HPD_OK) rc = check_stride(*s, width, dtype);
  if (rc != HPD_OK || n_rows == 0) return rc;
  for (const void* p : {hidden, weight, (const void*)workspace})
    if (!p || !aligned(p)) return HPD_E_INVALID;
  for (const void* p : {(const void*)targets, (const void*)logprob, (const void*)lse, (const void*)entropy})
    if (!aligned4(p)) return HPD_E_INVALID;
  if (!distinct({logprob, lse, entropy, workspace}, {hidden, weight, targets})) return HPD_E_INVALID;
  if (!targets) logprob = nullptr;
  if (!logprob && !lse && !entropy) return HPD_OK;
  HPD_HIP(hpd_launch_head({dtype, n_rows, width, vocab, hidden, weight, hidden_stride, weight_stride, targets, logprob, lse,
                           entropy, (char*)workspace}, (hipStream_t)stream));
  return HPD_OK;
}

int hpd_head_logprobs_backward(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab, const void* hidden,
                               int64_t hidden_stride, const void* weight, int64_t weight_stride, const int32_t* targets,
                               const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                               void* d_hidden, int64_t d_hidden_stride, void* d_weight, int64_t d_weight_stride,
                               void* workspace, void* stream) {
  int rc = check_head(dtype, n_rows, width, vocab);
  for (int64_t* s : {&hidden_stride, &weight_stride, &d_hidden_stride, &d_weight_stride})
    if (rc == HPD_OK) rc = check_stride(*s, width, dtype);
  if (rc != HPD_OK) return rc;
  if (!aligned(d_hidden) || !aligned(d_weight)) return HPD_E_INVALID;
  if (n_rows > 0) {
    for (const void* p : {hidden, weight, (const void*)workspace})
      if (!p || !aligned(p)) return HPD_E_INVALID;
    if (!lse || (g_logprob && !targets) || (g_entropy && !entropy)) return HPD_E_INVALID;
    for (const void* p : {(const void*)targets, (const void*)lse, (const void*)entropy, (const void*)g_logprob, (const void*)g_entropy})
      if (!aligned4(p)) return HPD_E_INVALID;
  }
  if (!distinct({d_hidden, d_weight, workspace}, {hidden, weight, targets, lse, entropy, g_logprob, g_entropy})) return HPD_E_INVALID;
  if (!d_hidden && !d_weight) return HPD_OK;
  HPD_HIP(hpd_launch_head_backward({dtype, n_rows, width, vocab, hidden, weight, hidden_stride, weight_stride, targets, lse, entropy,
                                    g_logprob, g_entropy, d_hidden, d_weight, d_hidden_stride, d_weight_stride, (char*)workspace},
                                   (hipStream_t)stream));
  return HPD_OK;
}

}  // extern "C"
