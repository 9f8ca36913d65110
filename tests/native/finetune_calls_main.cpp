// Which calls of the fine-tuning operators reach their kernels and which are refused: hpd_finetune_host.cpp with the launchers
// replaced by counters, on a layout without device memory that counts as being on the device.  Exit code 0 = as declared.
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "hpd_finetune.h"
#include "hpd_internal.h"

static int g_launches = 0;
#define LAUNCH(...) { ++g_launches; return hipSuccess; }
int hpd_hip_fail(hipError_t) { return HPD_E_HIP; }
hipError_t hpd_launch_ft_rope_table(const hpd_finetune_layout*, hipStream_t) LAUNCH()
hipError_t hpd_launch_ft_rotate(const hpd_finetune_layout*, bool, const void*, const void*, void*, void*,
                                const hpd_finetune_strides&, hipStream_t) LAUNCH()
hipError_t hpd_launch_ft_attention(const hpd_finetune_layout*, const void*, const void*, const void*, void*, float*, void*,
                                   const hpd_finetune_strides&, hipStream_t) LAUNCH()
hipError_t hpd_launch_ft_attention_backward(const hpd_finetune_layout*, const void*, const void*, const void*, const void*,
                                            const float*, const void*, void*, void*, void*, void*, const hpd_finetune_strides&,
                                            hipStream_t) LAUNCH()
int64_t hpd_logprobs_bytes(int32_t, int64_t, int32_t, int32_t) { return 0; }
hipError_t hpd_launch_logprobs(int32_t, const hpd_logprobs_args&, hipStream_t) LAUNCH()
hipError_t hpd_launch_logprobs_backward(int32_t, const hpd_logprobs_backward_args&, hipStream_t) LAUNCH()

#define CHECK(cond)                                                           \
  do {                                                                        \
    if (!(cond)) {                                                            \
      std::fprintf(stderr, "CHECK failed at line %d: %s\n", __LINE__, #cond); \
      std::exit(1);                                                           \
    }                                                                         \
  } while (0)
#define RUNS(call) do { g_launches = 0; CHECK((call) == HPD_OK); CHECK(g_launches == 1); } while (0)
#define REFUSED(call) do { g_launches = 0; CHECK((call) == HPD_E_INVALID); CHECK(g_launches == 0); } while (0)

int main() {
  hpd_finetune_config cfg{8, 2, 64, HPD_BF16, 10000.0, 4, HPD_FLAG_HOST_ONLY};
  const int32_t prompt[] = {5}, attr_ptr[] = {0, 1}, attr_len[] = {2}, value_len[] = {3};
  hpd_finetune_layout* L = nullptr;
  CHECK(hpd_build_finetune_layout(&cfg, 1, prompt, attr_ptr, attr_len, value_len, nullptr, &L) == HPD_OK);
  L->on_device = true;
  alignas(16) static char q[64], k[64], q_out[64], k_out[64];
  auto rotate = [&](void* qo, void* ko, hpd_finetune_strides st) {
    return hpd_finetune_rotate(L, 0, q, k, qo, ko, &st, nullptr);
  };
  // in place: with equal distances only, given or not
  RUNS(rotate(q_out, k_out, {}));
  RUNS(rotate(q_out, k_out, {.q = 640, .k = 128, .q_out = 512, .k_out = 640}));
  RUNS(rotate(q, k, {}));
  RUNS(rotate(q, k, {.q = 768, .k = 768, .q_out = 768, .k_out = 768}));
  RUNS(rotate(q, k, {.q = 512, .k = 128}));
  RUNS(rotate(q, k_out, {.k = 768}));
  REFUSED(rotate(q, k_out, {.q = 768}));
  REFUSED(rotate(q, k_out, {.q_out = 768}));
  REFUSED(rotate(q_out, k, {.k = 768}));
  REFUSED(rotate(q_out, k, {.k = 768, .k_out = 776}));
  REFUSED(rotate(q, k, {.q = 768, .k = 768, .q_out = 768}));
  hpd_finetune_layout_free(L);
  std::puts("as declared");
  return 0;
}
