// What the fine-tuning attention kernels share.
#pragma once

#include "hpd_attn_bf16.h"
#include "hpd_finetune.h"

// Arguments of the attention kernels.  Token distances in elements.
struct FtArgs {
  const hpd_ft_tile* tiles;
  const int32_t* rank;
  const int2* blk_rank;
  int64_t N, sq, sk, sv, sdq, sdk, sdv;
  int32_t Hq, Hkv, D;
  float scale;  // 1 / sqrt(D)
};

// Kernels for bf16 with head_dim 64 or 128 (hpd_finetune_stream.hip).
hipError_t hpd_launch_ft_stream_forward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                        void* out, float* lse, hipStream_t s);
hipError_t hpd_launch_ft_stream_backward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                         const void* out, const float* lse, const void* d_out, void* dq, void* dk, void* dv,
                                         void* workspace, hipStream_t s);

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.69314718055994530942f;

// row of register r of a 32 x 32 result in half h of the wave
__device__ __forceinline__ int tile_row(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

__device__ __forceinline__ void zero(floatx16* acc, int n) {
#pragma unroll
  for (int b = 0; b < n; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
}

}  // namespace
