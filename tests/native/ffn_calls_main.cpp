// Host-side exerciser for a sanitizer build (-fsanitize=address,undefined on the host pass) of hpd_ffn_host.cpp: calls with
// random valid and broken arguments; those that are valid must reach the launcher once with their strides filled in, the
// others not at all.  The launchers are replaced: nothing runs on a GPU.  Exit code 0 = no finding.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "hpd_ffn.h"
#include "hpd_internal.h"

static int g_launches = 0;
static hpd_ffn_strides g_st;
static int64_t g_stride[4];
int hpd_hip_fail(hipError_t) { return HPD_E_HIP; }
int64_t hpd_ffn_forward_bytes(const hpd_ffn_config&, int64_t n) { return n; }
int64_t hpd_ffn_backward_bytes(const hpd_ffn_config&, int64_t n) { return 2 * n; }
int64_t hpd_head_forward_bytes(int32_t, int64_t n, int32_t, int32_t) { return 3 * n; }
int64_t hpd_head_backward_bytes(int32_t, int64_t n, int32_t, int32_t) { return 4 * n; }
hipError_t hpd_launch_ffn(const hpd_ffn_forward_args& a, hipStream_t) { ++g_launches; g_st = a.st; return hipSuccess; }
hipError_t hpd_launch_ffn_backward(const hpd_ffn_backward_args& a, hipStream_t) { ++g_launches; g_st = a.st; return hipSuccess; }
hipError_t hpd_launch_head(const hpd_head_args& a, hipStream_t) {
  ++g_launches;
  g_stride[0] = a.hidden_stride; g_stride[1] = a.weight_stride;
  return hipSuccess;
}
hipError_t hpd_launch_head_backward(const hpd_head_backward_args& a, hipStream_t) {
  ++g_launches;
  g_stride[0] = a.hidden_stride; g_stride[1] = a.weight_stride; g_stride[2] = a.d_hidden_stride; g_stride[3] = a.d_weight_stride;
  return hipSuccess;
}

#define CHECK(cond)                                                          \
  do {                                                                       \
    if (!(cond)) {                                                           \
      std::fprintf(stderr, "CHECK failed at line %d: %s\n", __LINE__, #cond); \
      std::exit(1);                                                          \
    }                                                                        \
  } while (0)

static char g_mem[32][64] __attribute__((aligned(64)));
static void* p(int i) { return g_mem[i]; }
static float* f(int i) { return (float*)g_mem[i]; }

int main() {
  std::mt19937 rng(26209);
  auto pick = [&](int n) { return (int)(rng() % (unsigned)n); };
  for (int it = 0; it < 20000; ++it) {
    hpd_ffn_config c = {8 * (1 + pick(2000)), 8 * (1 + pick(5000)), pick(2), pick(3)};
    int64_t n = pick(4) ? 1 + pick(50000) : 0;
    hpd_ffn_strides st = {};
    int64_t* const s[] = {&st.x, &st.out, &st.gate, &st.up, &st.w_gate, &st.w_up, &st.w_down, &st.d_out, &st.d_x, &st.d_w_gate, &st.d_w_up,
                          &st.d_w_down};
    const bool inner[] = {0, 0, 1, 1, 0, 0, 1, 0, 0, 0, 0, 1};
    for (int i = 0; i < 12; ++i)
      if (pick(2)) *s[i] = (inner[i] ? c.inner : c.width) + 8 * pick(10);
    int want = HPD_OK;
    switch (pick(8)) {
      case 0: c.width += 4; want = HPD_E_UNSUPPORTED; break;
      case 1: c.activation = 3 + pick(100); want = HPD_E_UNSUPPORTED; break;
      case 2: *s[pick(12)] = 1 + pick(7); want = HPD_E_INVALID; break;
      case 3: n = -1 - pick(5); want = HPD_E_INVALID; break;
      case 4: *s[pick(12)] = (int64_t)1 << 28; want = HPD_E_OVERFLOW; break;
      default: break;
    }
    g_launches = 0;
    const bool null_strides = want == HPD_OK && pick(4) == 0;
    int rc = hpd_gated_ffn(&c, n, p(0), p(1), p(2), p(3), p(4), pick(2) ? p(5) : nullptr, pick(2) ? p(6) : nullptr, p(7),
                           null_strides ? nullptr : &st, nullptr);
    CHECK(rc == want && g_launches == (want == HPD_OK && n > 0));
    if (g_launches) {
      const int64_t* const got = &g_st.x;
      for (int i = 0; i < 12; ++i) CHECK(got[i] == (null_strides || *s[i] == 0 ? (inner[i] ? c.inner : c.width) : *s[i]));
    }
    g_launches = 0;
    const int parts = pick(16);
    rc = hpd_gated_ffn_backward(&c, n, p(0), p(1), p(2), p(3), p(4), p(5), p(6), parts & 1 ? p(7) : nullptr, parts & 2 ? p(8) : nullptr,
                                parts & 4 ? p(9) : nullptr, parts & 8 ? p(10) : nullptr, p(11), &st, nullptr);
    CHECK(rc == want && g_launches == (want == HPD_OK && parts != 0));  // (without rows: zeros as the weights' gradients)
    int64_t a = 0, b = 0;
    rc = hpd_gated_ffn_workspace(&c, n, &a, &b);
    CHECK(rc == (want == HPD_E_UNSUPPORTED || n < 0 ? want : HPD_OK));
    if (rc == HPD_OK) CHECK(a == n && b == 2 * n);

    const int32_t vocab = 1 + pick(200000);
    int64_t sx = pick(2) ? 0 : c.width + 8 * pick(5), sw = pick(2) ? 0 : c.width + 8 * pick(5), w1 = 0, w2 = c.width + 64;
    int head = HPD_OK;
    if (c.width % 8) head = HPD_E_UNSUPPORTED;
    else if (n < 0) head = HPD_E_INVALID;
    else if (pick(6) == 0) { sw = c.width - 8; head = HPD_E_INVALID; if (sw == 0) head = HPD_OK; }
    const bool over = head == HPD_OK && ((n + 127) / 128) * (((vocab > c.width ? vocab : c.width) + 63) / 64) > (1 << 22);
    if (over) head = HPD_E_OVERFLOW;
    g_launches = 0;
    rc = hpd_head_logprobs(c.dtype, n, c.width, vocab, p(0), sx, p(1), sw, (int32_t*)p(2), f(3), f(4), f(5), p(6), nullptr);
    CHECK(rc == head && g_launches == (head == HPD_OK && n > 0));
    if (g_launches) CHECK(g_stride[0] == (sx ? sx : c.width) && g_stride[1] == (sw ? sw : c.width));
    g_launches = 0;
    rc = hpd_head_logprobs_backward(c.dtype, n, c.width, vocab, p(0), sx, p(1), sw, (int32_t*)p(2), f(3), f(4), f(5), pick(2) ? f(6) : nullptr,
                                    p(7), w1, p(8), w2, p(9), nullptr);
    CHECK(rc == head && g_launches == (head == HPD_OK));
    if (g_launches) CHECK(g_stride[2] == c.width && g_stride[3] == w2);
  }
  std::printf("no finding\n");
  return 0;
}
