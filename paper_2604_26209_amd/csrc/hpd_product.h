// Products of the feed-forward block and of the vocabulary head: C[n][m] = sum_k A(m, k) B(n, k), with what becomes of C
// (activation, softmax sums, gradients, a store) done on the accumulators.
//
// m runs along the outputs' contiguous index ("features"), n along their rows.  An operand lies in memory either by rows, the
// contracted index contiguous (x and W of x W^T), or by columns, the contracted index outermost (W of d W, both
// operands of a weight's gradient); neither is transposed beforehand.
//
// A workgroup makes a tile of BM features x BN rows.  Both operands come to LDS by buffer loads that write there directly,
// 16 bytes a lane, in stages of 128 bytes of the contracted index (64 bf16, 32 fp32), several stages ahead; what lies
// outside an operand is a lane's offset out of the buffer's range, which the load makes zeros of.  A wave holds MI x NI blocks of
// 32 x 32 sums in registers.  While the products of a step (two chunks of 16 bytes of the contracted index) run, the operands of
// the next come from LDS; the one barrier of a stage stands in front of its last step, whose operands are in registers by then,
// so that the stage's place in LDS is free for the loads of another.
//
// LDS: by rows, row r has its chunk c at c ^ (r / 2 % 8): one chunk of 16 successive rows lies in different banks.  By columns,
// a row of the stage is one value of the contracted index, in granules of 64 bytes (32 bf16: a block), granule g at g ^ f(k): the
// 64 bytes of four successive k that a transposing read of bf16 takes lie in different banks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "hpd_attn_bf16.h"

struct hpd_operand {
  const void* p[2];  // second: the other half of a dual tile, or the second segment of the contraction
  int64_t stride;    // bytes from one row (by rows: of m or n; by columns: of k) to the next
  int32_t size;      // m or n of the whole operand
};

struct hpd_product_args {
  hpd_operand a, b;
  int32_t k;         // contracted elements of a segment
  int32_t segments;  // 1 or 2
  int32_t splits;    // parts the stages are cut into
  int32_t tiles_m, tiles_n;
};

namespace {

enum { BY_ROWS = 0, BY_COLUMNS = 1 };
constexpr uint32_t OUTSIDE = 0x80000000u;  // an offset that no buffer holds

template <typename T>
constexpr int CHUNK = 16 / (int)sizeof(T);  // elements of a 16-byte chunk
template <typename T>
constexpr int STAGE_K = 8 * CHUNK<T>;       // of the contracted index in a stage

typedef int32_t int32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t product_u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int32x4 buffer_of(const char* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  return {__builtin_amdgcn_readfirstlane((int32_t)(uint32_t)u), __builtin_amdgcn_readfirstlane((int32_t)(uint32_t)(u >> 32)),
          (int32_t)OUTSIDE, 0x00027000};
}
// 64 x 16 bytes to LDS, lane i's at lds + 16 i
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t off, int32x4 buf) {
  uint32_t keep;  // (M0 is the compiler's)
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(keep) : "s"(lds), "v"(off), "s"(buf) : "memory");
}
__device__ __forceinline__ uint32_t product_lds(const void* p) {
  return (uint32_t)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) char*)p);
}
__device__ __forceinline__ product_u4 read16(uint32_t at) {
  return *(const __attribute__((address_space(3))) product_u4*)(uintptr_t)at;
}
__device__ __forceinline__ uint32_t read4(uint32_t at) {
  return *(const __attribute__((address_space(3))) uint32_t*)(uintptr_t)at;
}
__device__ __forceinline__ uint2 read_tr8(uint32_t at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) hpd::short4v*)(uintptr_t)at));
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// One operand's tile of R rows (or columns) in a workgroup of WAVES waves.
template <typename T, int FORM, int R, int WAVES, bool DUAL>
struct Tile {
  static constexpr int BYTES = R * 128;
  static constexpr int LOADS = R / 8 / WAVES;        // load instructions of a wave and stage
  static constexpr int RB = R * (int)sizeof(T);      // by columns: bytes of one k
  static constexpr int GRANULES = RB / 64;
  static_assert(R % (8 * WAVES) == 0, "every wave loads whole KB");
  uint32_t off[LOADS];

  static __device__ __forceinline__ int swizzle(int k) {
    if (sizeof(T) == 2) return GRANULES >= 4 ? k & 3 : GRANULES == 2 ? (k >> 1) & 1 : 0;
    return GRANULES >= 4 ? ((k >> 2) & 1) << 1 : 0;  // (a read takes k and k + 4)
  }
  // by rows: the chunk that lane brings in its load f of the tile; by columns: the k
  static __device__ __forceinline__ int chunk_of(int f, int lane) { return (lane & 7) ^ ((4 * f + (lane >> 4)) & 7); }
  static __device__ __forceinline__ int k_of(int f, int lane) { return (f * 1024 + lane * 16) / RB; }

  // size: rows (columns) from the tile's first on
  __device__ __forceinline__ void init(int64_t stride, int64_t size, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int f = wave * LOADS + i;
      if (FORM == BY_ROWS) {
        int r = f * 8 + (lane >> 3);
        if (DUAL) r = (r >> 6) * 32 + (r & 31);  // blocks of 32 by turns from both halves
        off[i] = r < size ? (uint32_t)r * (uint32_t)stride + chunk_of(f, lane) * 16 : OUTSIDE;
      } else {
        const int k = k_of(f, lane), g = ((lane * 16 + f * 1024) % RB) / 64;
        const int c = (g ^ swizzle(k)) * 64 + (lane & 3) * 16;  // byte in the row
        off[i] = c / (int)sizeof(T) < size ? (uint32_t)k * (uint32_t)stride + c : OUTSIDE;
      }
    }
  }
  // the stage's load i to LDS; left: contracted elements from the stage's first on
  __device__ __forceinline__ void load(int i, uint32_t lds, int32x4 b0, int32x4 b1, int wave, int lane, int left) const {
    const int f = wave * LOADS + i;
    uint32_t o = off[i];
    const int k = FORM == BY_ROWS ? chunk_of(f, lane) * CHUNK<T> : k_of(f, lane);
    if (k >= left) o = OUTSIDE;
    load_to_lds(__builtin_amdgcn_readfirstlane(lds + f * 1024), o, DUAL && (f >> 2 & 1) ? b1 : b0);
  }
};

// Operands of a wave's products.  A lane's 16 bytes: row (column) lane % 32 of the block, elements CHUNK * (2 step + lane / 32) ..
template <typename T, int FORM, int R>
struct Reader {
  using TL = Tile<T, FORM, R, 1, false>;
  uint32_t at;      // by rows
  uint32_t col[4];  // by columns, bf16: of block (first + i), i % 4; fp32: one
  int first;
  __device__ __forceinline__ void init(int first_block, int lane) {
    const int l = lane & 31, h = lane >> 5;
    first = first_block;
    if (FORM == BY_ROWS) {
      at = (uint32_t)(first_block * 4096 + l * 128 + ((h ^ ((l >> 1) & 7)) << 4));
    } else if (sizeof(T) == 2) {
      const int a = lane & 15, j = a >> 2;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        col[i] = (8 * h + j) * TL::RB + (((first_block + i) ^ TL::swizzle(j)) << 6) + ((lane >> 4) & 1) * 32 + (a & 3) * 8;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        col[i] = 4 * h * TL::RB + (((2 * (first_block + i) + (l >> 4)) ^ TL::swizzle(4 * h)) << 6) + (l & 15) * 4;
    }
  }
  __device__ __forceinline__ product_u4 read(uint32_t tile, int i, int step) const {
    if (FORM == BY_ROWS) return read16(tile + (at ^ (step << 5)) + i * 4096);
    const uint32_t p = tile + col[i];
    if (sizeof(T) == 2) {
      const uint2 x = read_tr8(p + step * 16 * TL::RB), y = read_tr8(p + (step * 16 + 4) * TL::RB);
      return {x.x, x.y, y.x, y.y};
    }
    product_u4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = read4(p + (step * 8 + j) * TL::RB);
    return v;
  }
};

template <typename T>
__device__ __forceinline__ floatx16 multiply(product_u4 a, product_u4 b, floatx16 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  }
}

// Shapes of tiles: BM x BN by WM x WN waves, STAGES stages in LDS, WGS workgroups on a CU.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int WGS_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, WGS = WGS_;
  static constexpr int WAVES = WM * WN, MI = BM / 32 / WM, NI = BN / 32 / WN;
  static constexpr int STAGE_BYTES = (BM + BN) * 128;
};
using Large = Shape<256, 256, 2, 2, 2, 1>;
using Middle = Shape<128, 128, 2, 2, 2, 2>;
using Few64 = Shape<64, 64, 1, 1, 3, 3>;
using Few32 = Shape<64, 32, 1, 1, 3, 4>;
enum { LARGE = 0, MIDDLE = 1, FEW64 = 2, FEW32 = 3 };

// The place of a wave's blocks: features feature + 32 i (dual: block i is half i % 2 of features feature + 32 (i / 2)), rows row + 32 j.
struct Place {
  int64_t feature, row;
  int32_t split, tile_m;
  int wave_m, wave_n, lane;
};
// feature of register r in half h of the wave, counted from its block's first
__device__ __forceinline__ int block_row(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

// Workgroups go round the XCDs: each takes a run of tiles, so that what its L2 holds is shared.  Within a run, four tiles of m
// for one of n after another.
__device__ __forceinline__ void tile_of(int32_t id, int32_t total, int32_t tiles_m, int32_t tiles_n, int32_t& m, int32_t& n) {
  const int32_t per = total / 8, rest = total % 8, x = id % 8;
  id = x * per + (x < rest ? x : rest) + id / 8;
  constexpr int32_t G = 4;
  const int32_t group = id / (G * tiles_n), first = group * G, wide = tiles_m - first < G ? tiles_m - first : G;
  const int32_t in = id - group * G * tiles_n;
  m = first + in % wide;
  n = in / wide;
}

template <typename T, int FA, int FB, bool DUAL, typename S, typename Epilogue>
__global__ void __launch_bounds__(64 * S::WAVES, (S::WGS * S::WAVES + 3) / 4) product_kernel(hpd_product_args g, Epilogue epilogue) {
  using TA = Tile<T, FA, S::BM, S::WAVES, DUAL>;
  using TB = Tile<T, FB, S::BN, S::WAVES, false>;
  constexpr int MI = S::MI, NI = S::NI, K = STAGE_K<T>, LOADS = TA::LOADS + TB::LOADS;
  constexpr int SMEM = S::STAGES * S::STAGE_BYTES;
  __shared__ __attribute__((aligned(4096))) char smem[SMEM];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave_m = wave % S::WM, wave_n = wave / S::WM;

  const int32_t tiles = g.tiles_m * g.tiles_n;
  const int32_t split = blockIdx.x / tiles;
  int32_t tm, tn;
  tile_of(blockIdx.x - split * tiles, tiles, g.tiles_m, g.tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * (DUAL ? S::BM / 2 : S::BM), n0 = (int64_t)tn * S::BN;

  TA ta;
  TB tb;
  ta.init(g.a.stride, g.a.size - m0, wave, lane);
  tb.init(g.b.stride, g.b.size - n0, wave, lane);
  const int64_t a0 = FA == BY_ROWS ? m0 * g.a.stride : m0 * (int64_t)sizeof(T);
  const int64_t b0 = FB == BY_ROWS ? n0 * g.b.stride : n0 * (int64_t)sizeof(T);
  const char* const pa[2] = {(const char*)g.a.p[0] + a0, (const char*)g.a.p[1] + a0};
  const char* const pb[2] = {(const char*)g.b.p[0] + b0, (const char*)g.b.p[1] + b0};
  const int64_t step_a = FA == BY_ROWS ? 128 : K * g.a.stride, step_b = FB == BY_ROWS ? 128 : K * g.b.stride;
  const int32_t of_segment = (g.k + K - 1) / K, total = of_segment * g.segments;
  const int32_t begin = (int32_t)((int64_t)total * split / g.splits), end = (int32_t)((int64_t)total * (split + 1) / g.splits);
  const uint32_t lds = product_lds(smem);

  // A stage's loads, by the piece: of the wave's LOADS, load i.  A stage behind the last has buffers without bytes: zeros into
  // its place in LDS, and as many loads to wait for as ever.
  struct Stage {
    int32x4 a, a1, b;
    uint32_t at;
    int left;
  };
  auto stage_of = [&](int32_t t, int slot) -> Stage {
    const bool second = !DUAL && t >= of_segment;
    const int32_t u = second ? t - of_segment : t;
    Stage st = {buffer_of((second ? pa[1] : pa[0]) + u * step_a), buffer_of(pa[1] + u * step_a),
                buffer_of((second ? pb[1] : pb[0]) + u * step_b), lds + slot * S::STAGE_BYTES, g.k - u * K};
    if (t >= end) st.a[2] = st.a1[2] = st.b[2] = 0;
    return st;
  };
  auto load = [&](const Stage& st, int i) {
    if (i < TA::LOADS)
      ta.load(i, st.at, st.a, st.a1, wave, lane, st.left);
    else
      tb.load(i - TA::LOADS, st.at + TA::BYTES, st.b, st.b, wave, lane, st.left);
  };

  Reader<T, FA, S::BM> ra;
  Reader<T, FB, S::BN> rb;
  ra.init(wave_m * MI, lane);
  rb.init(wave_n * NI, lane);
  floatx16 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  product_u4 fa[2][MI], fb[2][NI];
  // operand i of a step's MI + NI
  auto read = [&](uint32_t at, int step, int to, int i) {
    if (i < NI)
      fb[to][i] = rb.read(at + TA::BYTES, i, step);
    else
      fa[to][i - NI] = ra.read(at, i - NI, step);
  };
  // the products of a step, between(n) after the n-th of `BLOCKS`
  constexpr int BLOCKS = MI * NI, READS = MI + NI;
  auto products = [&](int of, auto between) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        acc[i][j] = multiply<T>(fa[of][i], fb[of][j], acc[i][j]);
        between(i * NI + j);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  // the oldest stage on its way is there for all waves, and every wave has read the last of the stage in front of it
  auto meet = [&]() {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < S::STAGES; ++s) {
    const Stage st = stage_of(begin + s, s);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(st, i);
  }
  wait_loads<LOADS * (S::STAGES - 1)>();
  meet();
#pragma unroll
  for (int i = 0; i < READS; ++i) read(lds, 0, 0, i);
  int slot = 0;
  for (int32_t t = begin; t < end; ++t) {
    const int next = slot + 1 == S::STAGES ? 0 : slot + 1;
    const uint32_t here = lds + slot * S::STAGE_BYTES, there = lds + next * S::STAGE_BYTES;
#pragma unroll
    for (int step = 0; step < 3; ++step)
      products(step & 1, [&](int n) {
#pragma unroll
        for (int i = n * READS / BLOCKS; i < (n + 1) * READS / BLOCKS; ++i) read(here, step + 1, (step + 1) & 1, i);
      });
    wait_loads<LOADS * (S::STAGES - 2)>();
    meet();
    const Stage st = stage_of(t + S::STAGES, slot);
    products(1, [&](int n) {
#pragma unroll
      for (int i = n * READS / BLOCKS; i < (n + 1) * READS / BLOCKS; ++i) read(there, 0, 0, i);  // (behind the last stage: of no use)
#pragma unroll
      for (int i = n * LOADS / BLOCKS; i < (n + 1) * LOADS / BLOCKS; ++i) load(st, i);
    });
    slot = next;
  }
  wait_loads<0>();
  const Place at{m0 + wave_m * MI * (DUAL ? 16 : 32), n0 + wave_n * NI * 32, split, tm, wave_m, wave_n, lane};
  epilogue.template operator()<S, MI, NI>(acc, at, smem);
}

// four values as T at p (aligned to them)
template <typename T>
__device__ __forceinline__ void store4(T* p, const float* v) {
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
  else
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
template <typename T>
__device__ __forceinline__ void fetch4(const T* p, float* v) {
  if constexpr (sizeof(T) == 2) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
  } else {
    const float4 w = *reinterpret_cast<const float4*>(p);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  }
}

// Calls f(i, j, row, feature, values) for every four sums of successive features that exist (features come in fours).
template <int MI, int NI, typename F>
__device__ __forceinline__ void each4(floatx16 (&acc)[MI][NI], const Place& at, int64_t features, int64_t rows, F f) {
  const int l = at.lane & 31, h = at.lane >> 5;
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int64_t row = at.row + 32 * j + l;
    if (row >= rows) continue;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t m = at.feature + 32 * i + 8 * q + 4 * h;
        if (m >= features) continue;
        const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        f(row, m, v);
      }
  }
}

// C as T; rows from `second` on go to out[1]
template <typename T>
struct StoreProduct {
  T* out[2];
  int64_t stride[2], second;
  int64_t features, rows;
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char*) const {
    each4<MI, NI>(acc, at, features, rows, [&](int64_t row, int64_t m, const float* v) {
      store4(row < second ? out[0] + row * stride[0] + m : out[1] + (row - second) * stride[1] + m, v);
    });
  }
};
// C as fp32 into the split's own [rows][features], or added to what is there
struct StorePart {
  float* out;
  int64_t features, rows;
  int32_t add;
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char*) const {
    float* const mine = out + (int64_t)at.split * rows * features;
    each4<MI, NI>(acc, at, features, rows, [&](int64_t row, int64_t m, const float* v) {
      float w[4] = {v[0], v[1], v[2], v[3]};
      if (add) {
        fetch4(mine + row * features + m, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] += v[e];
      }
      store4(mine + row * features + m, w);
    });
  }
};

// out[r][m] = sum of the parts
template <typename T>
__global__ void __launch_bounds__(256) join_parts_kernel(const float* parts, int32_t n_parts, int64_t features, int64_t rows, T* out,
                                                         int64_t stride) {
  const int64_t per = features / 4, all = per * rows;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += gridDim.x * 256ll) {
    const int64_t row = i / per, m = (i - row * per) * 4;
    float s[4] = {0.f, 0.f, 0.f, 0.f}, v[4];
    for (int32_t p = 0; p < n_parts; ++p) {
      fetch4(parts + ((int64_t)p * rows + row) * features + m, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
    store4(out + row * stride + m, s);
  }
}

template <typename T>
hipError_t join_parts(const float* parts, int32_t n, int64_t features, int64_t rows, T* out, int64_t stride, hipStream_t s) {
  const int64_t all = features / 4 * rows;
  join_parts_kernel<T><<<dim3((uint32_t)std::min<int64_t>((all + 255) / 256, 1 << 16)), dim3(256), 0, s>>>(parts, n, features, rows, out, stride);
  return hipGetLastError();
}

// Which tiles a product gets, and into how many parts its contraction is cut.
struct Plan {
  int shape, splits;
  int64_t bm() const { return shape == LARGE ? 256 : shape == MIDDLE ? 128 : 64; }
  int64_t bn() const { return shape == LARGE ? 256 : shape == MIDDLE ? 128 : shape == FEW64 ? 64 : 32; }
};
// The least time by a simple account, in us: a round of workgroups takes its stages and `fixed` for its start and end; a stage takes
// `busy` where every place for a workgroup is taken, less where few are, `alone` at least.
struct ShapeCost {
  double busy, alone, fixed;
};
constexpr int CUS = 256;
inline ShapeCost shape_cost(bool f32, int shape) {
  constexpr ShapeCost BF16[] = {{1.5, 1.2, 8.0}, {1.05, 0.6, 5.0}, {1.3, 0.7, 4.0}, {1.6, 0.7, 4.0}};
  constexpr ShapeCost F32[] = {{0, 0, 0}, {3.6, 2.0, 5.0}, {2.0, 2.0, 4.0}, {1.7, 1.0, 4.0}};
  return f32 ? F32[shape] : BF16[shape];
}
// shapes: bits of those that the caller has kernels for; k: contracted elements, of all segments
template <typename T>
Plan plan_product(int64_t features, int64_t rows, int64_t k, bool dual, int most_splits, int shapes = 15) {
  constexpr int PLACES[] = {CUS, 2 * CUS, 3 * CUS, 4 * CUS};
  const bool f32 = sizeof(T) == 4;
  const int64_t stages = (k + STAGE_K<T> - 1) / STAGE_K<T>;
  Plan best = {MIDDLE, 1};
  double least = 1e30;
  for (int shape = f32 ? MIDDLE : LARGE; shape <= FEW32; ++shape) {
    if (!(shapes >> shape & 1)) continue;
    Plan p = {shape, 1};
    const ShapeCost c = shape_cost(f32, shape);
    const int64_t bm = dual ? p.bm() / 2 : p.bm();
    const int64_t tiles = ((features + bm - 1) / bm) * ((rows + p.bn() - 1) / p.bn());
    for (p.splits = 1; p.splits <= most_splits && (p.splits == 1 || stages / p.splits >= 4); ++p.splits) {
      const int64_t all = tiles * p.splits, full = all / PLACES[shape], rest = all % PLACES[shape], deep = (stages + p.splits - 1) / p.splits;
      double t = (double)full * (deep * c.busy + c.fixed);
      if (rest) t += deep * std::max(c.alone, c.busy * rest / PLACES[shape]) + c.fixed;
      if (p.splits > 1) t += 4.0 + (double)features * rows * p.splits * 8 / 4.0e6;
      if (t < least) {
        least = t;
        best = p;
      }
    }
  }
  return best;
}

template <typename T, int FA, int FB, bool DUAL, typename S, typename Epilogue>
hipError_t launch_shape(hpd_product_args g, const Epilogue& e, hipStream_t s) {
  const int64_t bm = DUAL ? S::BM / 2 : S::BM;
  g.tiles_m = (int32_t)((g.a.size + bm - 1) / bm);
  g.tiles_n = (int32_t)((g.b.size + S::BN - 1) / S::BN);
  product_kernel<T, FA, FB, DUAL, S, Epilogue><<<dim3((uint32_t)g.tiles_m * g.tiles_n * g.splits), dim3(64 * S::WAVES), 0, s>>>(g, e);
  return hipGetLastError();
}
template <typename T, int FA, int FB, bool DUAL, typename Epilogue>
hipError_t launch_product(Plan p, hpd_product_args g, const Epilogue& e, hipStream_t s) {
  g.splits = p.splits;
  if constexpr (sizeof(T) == 2)
    if (p.shape == LARGE) return launch_shape<T, FA, FB, DUAL, Large>(g, e, s);
  if constexpr (FB == BY_ROWS) {
    if (p.shape == FEW64) return launch_shape<T, FA, FB, DUAL, Few64>(g, e, s);
    if (p.shape == FEW32) return launch_shape<T, FA, FB, DUAL, Few32>(g, e, s);
  }
  return launch_shape<T, FA, FB, DUAL, Middle>(g, e, s);
}

// C as T, through parts in fp32 ([splits][rows][features] at `parts`) where the contraction is cut.
template <typename T, int FA, int FB>
hipError_t store_product(Plan p, const hpd_product_args& g, float* parts, T* out, int64_t stride, hipStream_t s) {
  const int64_t features = g.a.size, rows = g.b.size;
  if (p.splits == 1) return launch_product<T, FA, FB, false>(p, g, StoreProduct<T>{{out, nullptr}, {stride, 0}, rows, features, rows}, s);
  const hipError_t e = launch_product<T, FA, FB, false>(p, g, StorePart{parts, features, rows, 0}, s);
  return e != hipSuccess ? e : join_parts(parts, p.splits, features, rows, out, stride, s);
}

}  // namespace
