// What the fine-tuning attention kernels share.
#pragma once

#include "hpd_attn_bf16.h"
#include "hpd_finetune.h"

// Arguments of the attention kernels.  Token distances in elements.
struct FtArgs {
  const hpd_ft_tile* tiles;
  const int32_t* rank;
  const int2* blk_rank;
  const int32_t* seen_off;
  const uint32_t* seen;
  int64_t N, sq, sk, sv, sdq, sdk, sdv;
  int32_t Hq, Hkv, D;
  float scale;  // 1 / sqrt(D)
};

// Kernels for fp32 (hpd_finetune_f32.hip).
hipError_t hpd_launch_ft_f32_forward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                     void* out, float* lse, hipStream_t s);
hipError_t hpd_launch_ft_f32_backward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                      const void* out, const float* lse, const void* d_out, void* dq, void* dk, void* dv,
                                      void* workspace, hipStream_t s);
// Kernels for bf16 (hpd_finetune_stream.hip).
hipError_t hpd_launch_ft_stream_forward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                        void* out, float* lse, void* workspace, hipStream_t s);
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

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void wait_lds_and_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N>
__device__ __forceinline__ void wait_vector_memory() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Waits for values loaded in front of a loop.  The compiler would wait for them inside it, at every turn, and so
// for the loads to LDS that follow them, which it does not see.
template <typename T, int N>
__device__ __forceinline__ void arrived(T (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) char*)p);
}
// the ranks of a block's 32 tokens in scalar registers (wave-uniform address)
typedef int32_t int32x16 __attribute__((ext_vector_type(16)));
struct BlockRanks {
  int32x16 lo, hi;
  __device__ __forceinline__ void load(const int32_t* p) {
    p = reinterpret_cast<const int32_t*>(uniform(reinterpret_cast<const char*>(p)));
    asm volatile("s_load_dwordx16 %0, %2, 0x0\n\ts_load_dwordx16 %1, %2, 0x40\n\ts_waitcnt lgkmcnt(0)"
                 : "=&s"(lo), "=&s"(hi) : "s"(p) : "memory");
  }
  __device__ __forceinline__ int32_t at(int row) const { return row < 16 ? lo[row] : hi[row - 16]; }
  // of register r's row in half h
  __device__ __forceinline__ int32_t of(int r, int h) const {
    const int32_t x = at(tile_row(r, 0)), y = at(tile_row(r, 1));
    return h ? y : x;
  }
};

}  // namespace
