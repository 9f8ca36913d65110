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
#include <type_traits>

#include "hpd_attn_bf16.h"
#include "hpd_product_plan.h"

struct hpd_operand {
  const void* p[2];  // second: the other half of a dual tile, or the second segment of the contraction
  int64_t stride;    // bytes from one row (by rows: of m or n; by columns: of k) to the next, at most 2^23
  int32_t size;      // m or n of the whole operand
};

struct hpd_product_args {
  hpd_operand a, b;
  int32_t k;         // contracted elements (of either segment)
  int32_t splits;    // parts the stages are cut into
  int32_t tiles_m, tiles_n;
};

namespace {

constexpr uint32_t RANGE = 0x80000000u, OUTSIDE = 0xc0000000u;  // bytes of a buffer, an offset that none holds

typedef int32_t int32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t product_u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int32x4 buffer_of(const char* p, uint32_t bytes) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  return {__builtin_amdgcn_readfirstlane((int32_t)(uint32_t)u), __builtin_amdgcn_readfirstlane((int32_t)(uint32_t)(u >> 32)),
          __builtin_amdgcn_readfirstlane((int32_t)bytes), 0x00027000};
}
// N loads of 64 x 16 bytes to successive KB of LDS, lane i's at + 16 i.  The instruction's offset moves both addresses, so the
// lanes' offsets are n KB less for load n, and BIAS more.  (M0 is the compiler's.)  ONCE: the bytes will not be asked for again, the caches
// need not keep them.
constexpr uint32_t BIAS = 4096;
template <int N, bool ONCE>
__device__ __forceinline__ void load_to_lds(uint32_t lds, const uint32_t* off, int32x4 buf) {
  uint32_t keep;
#define HPD_LOADS_TO_LDS(HINT)                                                                                              \
  if constexpr (N == 4)                                                                                                     \
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"                                                      \
                 "buffer_load_dwordx4 %2, %6, 0 offen" HINT " lds\n\t"                                                      \
                 "buffer_load_dwordx4 %3, %6, 0 offen offset:0x400" HINT " lds\n\t"                                          \
                 "buffer_load_dwordx4 %4, %6, 0 offen offset:0x800" HINT " lds\n\t"                                          \
                 "buffer_load_dwordx4 %5, %6, 0 offen offset:0xc00" HINT " lds\n\t"                                          \
                 "s_mov_b32 m0, %0"                                                                                         \
                 : "=&s"(keep) : "s"(lds), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(buf) : "memory");        \
  else if constexpr (N == 2)                                                                                                \
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"                                                      \
                 "buffer_load_dwordx4 %2, %4, 0 offen" HINT " lds\n\t"                                                      \
                 "buffer_load_dwordx4 %3, %4, 0 offen offset:0x400" HINT " lds\n\t"                                          \
                 "s_mov_b32 m0, %0"                                                                                         \
                 : "=&s"(keep) : "s"(lds), "v"(off[0]), "v"(off[1]), "s"(buf) : "memory");                                  \
  else                                                                                                                      \
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"                                                      \
                 "buffer_load_dwordx4 %2, %3, 0 offen" HINT " lds\n\t"                                                      \
                 "s_mov_b32 m0, %0"                                                                                         \
                 : "=&s"(keep) : "s"(lds), "v"(off[0]), "s"(buf) : "memory");
  if constexpr (ONCE) {
    HPD_LOADS_TO_LDS(" nt")
  } else {
    HPD_LOADS_TO_LDS("")
  }
#undef HPD_LOADS_TO_LDS
}
// a dword a lane to 256 bytes of LDS that nobody reads: the lines come to the L2
__device__ __forceinline__ void touch(uint32_t lds, uint32_t off, int32x4 buf) {
  uint32_t keep;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
               "buffer_load_dword %2, %3, 0 offen lds\n\t"
               "s_mov_b32 m0, %0"
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
template <typename T, int FORM, int R, int WAVES, bool DUAL, bool ONCE = false>
struct Tile {
  static constexpr int BYTES = R * 128;
  static constexpr int LOADS = R / 8 / WAVES;        // load instructions of a wave and stage, issued in groups
  static constexpr int GROUP = LOADS % 4 == 0 ? 4 : LOADS % 2 == 0 ? 2 : 1, GROUPS = LOADS / GROUP;
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

  // size: rows (columns) from the tile's first on.  (A stride is at most 2^23 bytes, a stage has at most 64 k and a tile 256 rows: 31 bits)
  __device__ __forceinline__ void init(int64_t stride, int64_t size, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int f = wave * LOADS + i;
      if (FORM == BY_ROWS) {
        int r = f * 8 + (lane >> 3);
        if (DUAL) r %= R / 2;  // (one half's rows, then the other's)
        off[i] = r < size ? (uint32_t)r * (uint32_t)stride + chunk_of(f, lane) * 16 : OUTSIDE;
      } else {
        const int k = k_of(f, lane), g = ((lane * 16 + f * 1024) % RB) / 64;
        const int c = (g ^ swizzle(k)) * 64 + (lane & 3) * 16;  // byte in the row
        off[i] = c / (int)sizeof(T) < size ? (uint32_t)k * (uint32_t)stride + c : OUTSIDE;
      }
      off[i] += BIAS - i % GROUP * 1024;
    }
  }
  // the lane's line of a stage, of those that the wave touches
  static __device__ __forceinline__ uint32_t line(int64_t stride, int64_t size, int wave, int lane) {
    constexpr int MINE = R / WAVES;
    const int n = wave * MINE + lane;
    if (lane >= MINE) return OUTSIDE;
    if (FORM == BY_ROWS) {
      const int r = DUAL ? n % (R / 2) : n;
      return r < size ? (uint32_t)r * (uint32_t)stride + BIAS : OUTSIDE;
    }
    const int k = n / (RB / 128), c = n % (RB / 128) * 128;
    return c / (int)sizeof(T) < size ? (uint32_t)k * (uint32_t)stride + c + BIAS : OUTSIDE;
  }
  // the buffer of a stage that begins at p and has `left` (at least 1) elements of k: by columns, it ends behind the last of them
  static __device__ __forceinline__ int32x4 buffer(const char* p, int64_t stride, int left) {
    return buffer_of(p - BIAS, (FORM == BY_COLUMNS && left < STAGE_K<T> ? (uint32_t)left * (uint32_t)stride : RANGE) + BIAS);
  }
  // the stage's load group i to LDS; by rows, MASKED: nothing behind `left`
  template <bool MASKED>
  __device__ __forceinline__ void load(int i, uint32_t lds, int32x4 b0, int32x4 b1, int wave, int lane, int left) const {
    const int f = wave * LOADS + i * GROUP;
    uint32_t o[GROUP];
#pragma unroll
    for (int e = 0; e < GROUP; ++e)
      o[e] = MASKED && FORM == BY_ROWS && chunk_of(f + e, lane) * CHUNK<T> >= left ? OUTSIDE : off[i * GROUP + e];
    load_to_lds<GROUP, ONCE>(__builtin_amdgcn_readfirstlane(lds + f * 1024), o, DUAL && f >= R / 16 ? b1 : b0);
  }
};

// Operands of a wave's products.  A lane's 16 bytes: row (column) lane % 32 of the block, elements CHUNK * (2 step + lane / 32) ..
// DUAL: a block is 16 rows of one half and the same 16 of the other, whose sums then lie in the same lanes.
template <typename T, int FORM, int R, bool DUAL>
struct Reader {
  using TL = Tile<T, FORM, R, 1, false>;
  uint32_t at;      // by rows
  uint32_t col[4];  // by columns, bf16: of block (first + i), i % 4; fp32: one
  int first;
  __device__ __forceinline__ void init(int first_block, int lane) {
    const int l = lane & 31, h = lane >> 5;
    first = first_block;
    if (FORM == BY_ROWS) {
      const int row = DUAL ? first_block * 16 + (l >> 4) * (R / 2) + (l & 15) : first_block * 32 + l;
      at = (uint32_t)(row * 128 + ((h ^ ((l >> 1) & 7)) << 4));
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
    if (FORM == BY_ROWS) return read16(tile + (at ^ (step << 5)) + i * (DUAL ? 2048 : 4096));
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

// Shapes of tiles: BM x BN by WM x WN waves, STAGES stages in LDS, WGS workgroups on a CU.  (Workgroups that stay and make tile after
// tile, the next one's first stages on their way while one is stored, are slower: 8192 x 8192 x 8192 in 880 us, 840 as it is; CUs do
// not all run at one rate, and a tile goes to the one that is free.)
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int WGS_, bool ONCE_ = false>
struct Shape {
  static constexpr bool ONCE = ONCE_;  // no other workgroup reads the tile's A
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, WGS = WGS_;
  static constexpr int WAVES = WM * WN, MI = BM / 32 / WM, NI = BN / 32 / WN;
  static constexpr int STAGE_BYTES = (BM + BN) * 128;
  static constexpr int SMEM = STAGES * STAGE_BYTES, TURN = SMEM / WAVES / 4096 * 4096;  // of it, a wave's when its sums are stored
  static constexpr bool MANY = MI * NI * 16 > 128;  // the sums are in accumulation registers
  // Two stages on their way are less than the latency of memory takes: each wave touches lines of A two stages further on.  In bf16, features x rows x
  // contracted, of equal values (under the least power): 24576 x 512 x 4096 99 -> 87 us, 16544 x 3520 x 5120 513 -> 437, 5120 x 2274 x 12256
  // 276 -> 225, 8192 x 8192 x 8192 716 -> 692.  (One stage further on: the same where rows are of whole lines, else less; three, B's
  // lines too, or 128 x 128 and 64-wide tiles: slower.)
  static constexpr int TOUCH = STAGES == 2 && WGS == 1;
  // Sums of a block, each over a part of a stage's steps, added up at the end.  A sum is rounded with every product: two halve the
  // error of a long contraction, four quarter it (fp32 gradients of the block for 1801 rows: off by 5e-7 in place of 1e-6; the
  // entropies of three rows of 150001 tokens: 4e-7, 1.5e-6).
  static constexpr int SUMS = MANY ? 1 : 4 / (MI * NI);
};
// DUAL: a tile's features half and half from two A; SEGMENTS: a second A and B are contracted after the first; TAIL: any number of contracted
// elements, A by columns and B by rows, with zeros behind B's last up to a multiple of 16 bytes
enum { PLAIN = 0, DUAL = 1, SEGMENTS = 2, TAIL = 3 };
// bf16 products of 4096 elements: Large 1.2 PFLOP/s for 4096 x 4096 and more; Middle 1.06 from 4096 x 2048 (Large 0.72); Small 0.61 for
// 2048 x 1024 (Middle 0.39).  Wide where its tiles go into fewer or fuller rounds: 256 of them for 24576 features x 512 rows in 101 us,
// 192 of Large in 114.  Few rows, where the weights' bytes are what it takes: Few32 5.9 TB/s for 24576 features and a row, 6.4 for
// 48000 (without the hint that the weights will not be read again 5.3 and 5.8; Small 4.9 and 5.5), Few64 4.5 for 64 rows (Small 4.2), Few128
// 15544 features x 126 rows of 4096 in 36 us (Small 45, Middle 67; 64 x 192 tiles were never the best).  fp32: Small 0.13 to 0.14 PFLOP/s
// from 2048 x 1024 on (128 x 128 with eight waves: 0.146 at most, 0.07 for 2048 x 1024), and Few.
using Large = Shape<256, 256, 2, 2, 2, 1>;
using Middle = Shape<128, 128, 2, 4, 2, 2>;
using Small = Shape<64, 64, 2, 2, 3, 3>;
using Few64 = Shape<64, 64, 2, 2, 4, 2, true>;
using Few32 = Shape<64, 32, 2, 1, 4, 3, true>;
using Wide = Shape<192, 256, 2, 2, 2, 1>;
using Few128 = Shape<64, 128, 2, 2, 3, 2, true>;
static_assert(Large::SUMS == SHAPE_SUMS[LARGE] && Middle::SUMS == SHAPE_SUMS[MIDDLE] && Small::SUMS == SHAPE_SUMS[SMALL] &&
                  Few64::SUMS == SHAPE_SUMS[FEW64] && Few32::SUMS == SHAPE_SUMS[FEW32] && Few128::SUMS == SHAPE_SUMS[FEW128] &&
                  Wide::SUMS == SHAPE_SUMS[WIDE],
              "what the plans go by");

// f(0) .. f(N - 1), the numbers as types: what is indexed with them stays in registers however long f is
template <int N, typename F, int I = 0>
__device__ __forceinline__ void each(F f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, F, I + 1>(f);
  }
}

// The place of a wave's blocks: features feature + 32 i (dual: feature + 16 i, registers 0 to 7 one half's, 8 to 15 the other's), rows row + 32 j.
struct Place {
  int64_t feature, row;
  int32_t split, tile_m;
  int wave_m, wave_n, lane;
};
// feature of register r in half h of the wave, counted from its block's first
__device__ __forceinline__ int block_row(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

// Workgroups go round the XCDs: each takes a run of tiles, so that what its L2 holds is shared (12288 x 16384 x 4096 in bf16: 1421 us
// and 2.4 GB read, 1534 and 6.6 without).  Within a run, four tiles of m for one of n after another (two or eight were no faster).
__device__ __forceinline__ void tile_of(int32_t id, int32_t total, int32_t tiles_m, int32_t tiles_n, int32_t& m, int32_t& n) {
  const int32_t per = total / 8, rest = total % 8, x = id % 8;
  id = x * per + (x < rest ? x : rest) + id / 8;
  constexpr int32_t G = 4;
  const int32_t group = id / (G * tiles_n), first = group * G, wide = tiles_m - first < G ? tiles_m - first : G;
  const int32_t in = id - group * G * tiles_n;
  m = first + in % wide;
  n = in / wide;
}

// The epilogue wants fp32 sums taken in the order of k.
template <typename Epilogue>
constexpr bool IN_ORDER = false;

template <typename T, int FA, int FB, int MODE, typename S, typename Epilogue>
__global__ void __launch_bounds__(64 * S::WAVES, (S::WGS * S::WAVES + 3) / 4) product_kernel(hpd_product_args g, Epilogue epilogue) {
  using TA = Tile<T, FA, S::BM, S::WAVES, MODE == DUAL, S::ONCE>;
  using TB = Tile<T, FB, S::BN, S::WAVES, false>;
  constexpr int MI = S::MI, NI = S::NI, K = STAGE_K<T>, LOADS = TA::LOADS + TB::LOADS, GROUPS = TA::GROUPS + TB::GROUPS;
  // The stage with less than a whole stage's elements is the first, which is loaded in front of the loop.  Of two segments it is the
  // last of each, and where the number may be odd the last, so that rows are read at multiples of 16 bytes: loads by rows are masked
  // all the time (1 % of the largest products).
  constexpr bool MASKED = MODE == SEGMENTS || MODE == TAIL;
  constexpr int SUMS = sizeof(T) == 4 && IN_ORDER<Epilogue> && !S::ONCE ? 1 : S::SUMS;
  __shared__ __attribute__((aligned(4096))) char smem[S::SMEM + S::TOUCH * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave_m = wave % S::WM, wave_n = wave / S::WM;

  // (divisions are made in vector registers, from where their results would not come back by themselves)
  auto scalar = [](int32_t x) { return __builtin_amdgcn_readfirstlane(x); };
  const int32_t tiles = g.tiles_m * g.tiles_n, split = scalar(blockIdx.x / tiles);
  int32_t tile_m, tile_n;
  tile_of(blockIdx.x - split * tiles, tiles, g.tiles_m, g.tiles_n, tile_m, tile_n);
  tile_m = scalar(tile_m);
  const int64_t m0 = (int64_t)tile_m * (MODE == DUAL ? S::BM / 2 : S::BM), n0 = (int64_t)scalar(tile_n) * S::BN;
  const int32_t of_segment = (g.k + K - 1) / K, stages = MODE == SEGMENTS ? 2 * of_segment : of_segment;
  const int32_t first_k = MASKED ? K : g.k - (of_segment - 1) * K;  // elements of the first stage
  const int32_t begin = scalar((int32_t)((int64_t)stages * split / g.splits)), end = scalar((int32_t)((int64_t)stages * (split + 1) / g.splits));

  TA ta;
  TB tb;
  ta.init(g.a.stride, g.a.size - m0, wave, lane);
  tb.init(g.b.stride, g.b.size - n0, wave, lane);
  const int64_t a0 = FA == BY_ROWS ? m0 * g.a.stride : m0 * (int64_t)sizeof(T);
  const int64_t b0 = FB == BY_ROWS ? n0 * g.b.stride : n0 * (int64_t)sizeof(T);
  const uint32_t lds = product_lds(smem);
  // A stage's loads, by the group: of the wave's GROUPS, group i.  A stage behind the last has buffers without bytes: zeros into
  // its place in LDS, and as many loads to wait for as ever.
  struct Stage {
    int32x4 a, a1, b;
    uint32_t at;
    int left;
  };
  Stage st;
  int32_t lt = begin, plain = -1;  // the stage to be loaded; up to this one, the next lies behind the one before
  auto forward = [](int32x4& buf, int64_t step) {
    const uint64_t p = ((uint64_t)(uint32_t)buf[1] << 32 | (uint32_t)buf[0]) + (uint64_t)step;
    buf[0] = (int32_t)(uint32_t)p;
    buf[1] = (int32_t)(uint32_t)(p >> 32);
  };
  const int64_t step_a = FA == BY_ROWS ? 128 : K * g.a.stride, step_b = FB == BY_ROWS ? 128 : K * g.b.stride;
  auto next_stage = [&](int slot) {
    st.at = lds + slot * S::STAGE_BYTES;
    if (lt < plain) {
      forward(st.a, step_a);
      if (MODE == DUAL) forward(st.a1, step_a);
      forward(st.b, step_b);
      ++lt;
      return;
    }
    const bool second = MODE == SEGMENTS && lt >= of_segment;
    const int32_t u = second ? lt - of_segment : lt;
    const int64_t k = MASKED || u == 0 ? (int64_t)u * K : first_k + (int64_t)(u - 1) * K;
    const int32_t left = MASKED ? g.k - u * K : u == 0 ? first_k : K;
    const int64_t ka = a0 + k * (FA == BY_ROWS ? (int64_t)sizeof(T) : g.a.stride);
    const int64_t kb = b0 + k * (FB == BY_ROWS ? (int64_t)sizeof(T) : g.b.stride);
    st.a = TA::buffer((const char*)g.a.p[second] + ka, g.a.stride, left);
    if (MODE == DUAL) st.a1 = TA::buffer((const char*)g.a.p[1] + ka, g.a.stride, left);
    st.b = TB::buffer((const char*)g.b.p[second] + kb, g.b.stride, left);
    st.left = left < K ? left : K;
    if (lt < end) {
      ++lt;
      // (the whole stages behind it, of its segment)
      const int32_t whole = MASKED ? (second ? of_segment : 0) + g.k / K : u == 0 && first_k < K ? lt : end;
      plain = whole < end ? whole : end;
    } else {
      st.a[2] = st.b[2] = 0;
      if (MODE == DUAL) st.a1[2] = 0;
    }
    // (arguments may have been loaded: with those on their way, the wait for one operand from LDS would be one for all)
    __builtin_amdgcn_s_waitcnt(0xc07f);
  };
  // of A's stage two behind the one that was loaded last, if it is a whole one behind that
  const uint32_t line = TA::line(g.a.stride, g.a.size - m0, wave, lane), nowhere = __builtin_amdgcn_readfirstlane(lds + S::SMEM);
  auto touch_ahead = [&]() {
    if constexpr (S::TOUCH) {
      int32x4 buf = st.a;
      if (MODE == DUAL)
#pragma unroll
        for (int i = 0; i < 2; ++i) buf[i] = wave >= S::WAVES / 2 ? st.a1[i] : st.a[i];
      forward(buf, 2 * step_a);
      buf[2] = lt + 1 < plain ? (int32_t)(RANGE + BIAS) : 0;
      touch(nowhere, line, buf);
    }
  };
  auto load = [&](int i, auto masked) {
    constexpr bool M = decltype(masked)::value;
    if (i < TA::GROUPS)
      ta.template load<M>(i, st.at, st.a, MODE == DUAL ? st.a1 : st.a, wave, lane, st.left);
    else
      tb.template load<M>(i - TA::GROUPS, st.at + TA::BYTES, st.b, st.b, wave, lane, st.left);
  };

  Reader<T, FA, S::BM, MODE == DUAL> ra;
  Reader<T, FB, S::BN, false> rb;
  ra.init(wave_m * MI, lane);
  rb.init(wave_n * NI, lane);
  floatx16 sums[SUMS][MI][NI];
#pragma unroll
  for (int c = 0; c < SUMS; ++c)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[c][i][j][r] = 0.f;
  product_u4 fa[2][MI], fb[2][NI];
  // operand i of a step's MI + NI
  auto read = [&](uint32_t at, int step, int to, int i) {
    if (i < NI)
      fb[to][i] = rb.read(at + TA::BYTES, i, step);
    else
      fa[to][i - NI] = ra.read(at, i - NI, step);
  };
  // the products of a step, between(n) after the n-th of BLOCKS
  constexpr int BLOCKS = MI * NI, READS = MI + NI;
  auto products = [&](int step, auto between) {
    const int of = step & 1, c = step % SUMS;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        sums[c][i][j] = multiply<T>(fa[of][i], fb[of][j], sums[c][i][j]);
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
    next_stage(s);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) load(i, std::true_type{});
    touch_ahead();
  }
  wait_loads<LOADS * (S::STAGES - 1) + S::TOUCH * S::STAGES>();
  meet();
#pragma unroll
  for (int i = 0; i < READS; ++i) read(lds, 0, 0, i);
  int slot = 0;
  for (int32_t t = begin; t < end; ++t) {
    const int next = slot + 1 == S::STAGES ? 0 : slot + 1;
    const uint32_t here = lds + slot * S::STAGE_BYTES, there = lds + next * S::STAGE_BYTES;
#pragma unroll
    for (int step = 0; step < 3; ++step)
      products(step, [&](int n) {
#pragma unroll
        for (int i = n * READS / BLOCKS; i < (n + 1) * READS / BLOCKS; ++i) read(here, step + 1, (step + 1) & 1, i);
      });
    wait_loads<LOADS * (S::STAGES - 2) + S::TOUCH * (S::STAGES - 1)>();
    meet();
    next_stage(slot);
    products(3, [&](int n) {
#pragma unroll
      for (int i = n * READS / BLOCKS; i < (n + 1) * READS / BLOCKS; ++i) read(there, 0, 0, i);  // (behind the last stage: of no use)
#pragma unroll
      for (int i = n * GROUPS / BLOCKS; i < (n + 1) * GROUPS / BLOCKS; ++i) load(i, std::integral_constant<bool, MASKED>{});
    });
    touch_ahead();
    slot = next;
  }
  wait_loads<0>();
  __syncthreads();  // (what came behind the last stage is there, for all waves: the stages' LDS is free)
  if (S::MANY) {
    // (the last products' sums are read in sum_of, where the compiler does not see it: their 16 passes are over here)
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  floatx16(&acc)[MI][NI] = sums[0];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      if (SUMS == 2) acc[i][j] += sums[1 % SUMS][i][j];
      if (SUMS == 4) acc[i][j] = (acc[i][j] + sums[1 % SUMS][i][j]) + (sums[2 % SUMS][i][j] + sums[3 % SUMS][i][j]);
    }
  const Place at{m0 + wave_m * MI * (MODE == DUAL ? 16 : 32), n0 + wave_n * NI * 32, split, tile_m, wave_m, wave_n, lane};
  epilogue.template operator()<S, MI, NI>(acc, at, smem);
}

template <typename T>
using Four = typename std::conditional<sizeof(T) == 2, uint2, float4>::type;  // four successive values
template <typename T>
__device__ __forceinline__ Four<T> pack4(const float* v) {
  if constexpr (sizeof(T) == 2)
    return make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
  else
    return make_float4(v[0], v[1], v[2], v[3]);
}
template <typename T>
__device__ __forceinline__ void unpack4(Four<T> w, float* v) {
  if constexpr (sizeof(T) == 2) {
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
  } else {
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, const float* v) { *reinterpret_cast<Four<T>*>(p) = pack4<T>(v); }
template <typename T>
__device__ __forceinline__ void fetch4(const T* p, float* v) { unpack4<T>(*reinterpret_cast<const Four<T>*>(p), v); }

// 32 rows of WIDTH features between the accumulators' layout (lane l: row l % 32, four features of every eight) and
// whole rows, 16 bytes a lane, through a wave's own LDS; 16-byte chunk c of row r lies at c ^ r.
template <typename T, int WIDTH>
struct Turn {
  static constexpr int PLACES = WIDTH <= 16 ? 16 : WIDTH <= 32 ? 32 : WIDTH <= 64 ? 64 : 128;  // features a row has room for
  static constexpr int RB = PLACES * (int)sizeof(T), CHUNKS = RB / 16, ROWS = 64 / CHUNKS, TURNS = 32 / ROWS;
  static_assert(32 * RB <= 8192, "a wave's LDS");
  char* mine;
  int lane;
  // bytes: of a wave's LDS; the rows lie `from` bytes behind its first
  __device__ __forceinline__ Turn(const Place& at, char* smem, int bytes, int from = 0) : mine(smem + (threadIdx.x >> 6) * bytes + from), lane(at.lane) {}
  static __device__ __forceinline__ void order() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
  // of the lane's row, of the eight features from c on the lane's four
  __device__ __forceinline__ T* four(int c) const {
    const int r = lane & 31, byte = (c + 4 * (lane >> 5)) * (int)sizeof(T);
    return reinterpret_cast<T*>(mine + r * RB + (((byte >> 4) ^ (r & (CHUNKS - 1))) << 4) + (byte & 15));
  }
  // (a fence: or the sums of many blocks crowd into registers)
  __device__ __forceinline__ void put4(int c, const float* v) const {
    store4(four(c), v);
    __builtin_amdgcn_sched_barrier(0);
  }
  // the lane's chunk of rows ROWS n ..
  __device__ __forceinline__ int row(int n) const { return n * ROWS + lane / CHUNKS; }
  __device__ __forceinline__ int column() const { return lane % CHUNKS * (16 / (int)sizeof(T)); }
  __device__ __forceinline__ product_u4* chunk(int n) const {
    return reinterpret_cast<product_u4*>(mine + row(n) * RB + (((lane % CHUNKS) ^ (row(n) & (CHUNKS - 1))) << 4));
  }
  // where the chunk lies behind the first of rows ROWS n .., in bytes (a stride is at most 2^23 of them)
  __device__ __forceinline__ uint32_t behind(int64_t stride) const {
    return (uint32_t)(lane / CHUNKS) * (uint32_t)(stride * (int64_t)sizeof(T)) + (uint32_t)(lane % CHUNKS) * 16;
  }
  // To memory: rows `from` .. of `rows`, `width` features of each.  out(r), the same for the whole wave: where rows ROWS n .. begin.
  template <typename F>
  __device__ __forceinline__ void store(int64_t rows, int64_t width, int64_t stride, F out, int64_t from = 0) const {
    order();
    product_u4 v[TURNS];
#pragma unroll
    for (int n = 0; n < TURNS; ++n) v[n] = *chunk(n);
    order();
    const uint32_t at = behind(stride);
#pragma unroll
    for (int n = 0; n < TURNS; ++n)
      if (row(n) >= from && row(n) < rows && column() < width && column() < WIDTH)
        *(__attribute__((address_space(1))) product_u4*)(uniform(reinterpret_cast<const char*>(out(n * ROWS))) + at) = v[n];
    __builtin_amdgcn_sched_barrier(0);  // (the next rows' values do not crowd in here)
  }
  struct Rows {
    product_u4 v[TURNS];
  };
  template <typename F>
  __device__ __forceinline__ Rows fetch(int64_t rows, int64_t width, int64_t stride, F in) const {
    Rows x;
    const uint32_t at = behind(stride);
#pragma unroll
    for (int n = 0; n < TURNS; ++n) {
      x.v[n] = product_u4{0, 0, 0, 0};
      if (row(n) < rows && column() < width && column() < WIDTH)
        x.v[n] = *(const __attribute__((address_space(1))) product_u4*)(uniform(reinterpret_cast<const char*>(in(n * ROWS))) + at);
    }
    return x;
  }
  __device__ __forceinline__ void put(const Rows& x) const {
    order();
#pragma unroll
    for (int n = 0; n < TURNS; ++n) *chunk(n) = x.v[n];
    order();
  }
};

// Register r of a block of sums.  Shapes with MANY have them in accumulation registers, from where they are taken one by one: left to the
// compiler, whole blocks come at once and do not fit.
template <typename S>
__device__ __forceinline__ float sum_of(const floatx16& block, int r) {
  if constexpr (S::MANY) {
    float v;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(block[r]));
    return v;
  } else {
    return block[r];
  }
}

// C as T; rows from `second` on go to out[1]
template <typename T>
struct StoreProduct {
  T* out[2];
  int64_t stride[2], second;
  int64_t features, rows;
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char* smem) const {
    const Turn<T, 32 * MI> turn(at, smem, S::TURN);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t first = at.row + 32 * j;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = sum_of<S>(acc[i][j], 4 * q + e);
          turn.put4(32 * i + 8 * q, v);
        }
      const int64_t left = rows - first, here = second - first;  // rows of the block, and of them to out[0]
      if (here > 0)
        turn.store(left < here ? left : here, features - at.feature, stride[0], [&](int r) { return out[0] + (first + r) * stride[0] + at.feature; });
      if (here < 32)
        turn.store(left, features - at.feature, stride[1], [&](int r) { return out[1] + (r - here) * stride[1] + at.feature; }, here);
    }
  }
};
// C as fp32 into the split's own [rows][features], or added to what is there
struct StorePart {
  float* out;
  int64_t features, rows;
  int32_t add;
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char*) const {
    const int l = at.lane & 31, h = at.lane >> 5;
    float* const mine = out + (int64_t)at.split * rows * features;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t row = at.row + 32 * j + l;
      if (row >= rows) continue;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t m = at.feature + 32 * i + 8 * q + 4 * h;
          if (m >= features) continue;  // (features come in fours)
          float w[4] = {0.f, 0.f, 0.f, 0.f};
          if (add) fetch4(mine + row * features + m, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] += sum_of<S>(acc[i][j], 4 * q + e);
          store4(mine + row * features + m, w);
          __builtin_amdgcn_sched_barrier(0);
        }
    }
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

template <typename T, int FA, int FB, int MODE, typename S, typename Epilogue>
hipError_t launch_shape(hpd_product_args g, const Epilogue& e, hipStream_t s) {
  const int64_t bm = MODE == DUAL ? S::BM / 2 : S::BM;
  g.tiles_m = (int32_t)((g.a.size + bm - 1) / bm);
  g.tiles_n = (int32_t)((g.b.size + S::BN - 1) / S::BN);
  product_kernel<T, FA, FB, MODE, S, Epilogue><<<dim3((uint32_t)g.tiles_m * g.tiles_n * g.splits), dim3(64 * S::WAVES), 0, s>>>(g, e);
  return hipGetLastError();
}
template <typename T, int FA, int FB, int MODE, typename Epilogue>
hipError_t launch_product(Plan p, hpd_product_args g, const Epilogue& e, hipStream_t s) {
  g.splits = p.splits;
  if constexpr (sizeof(T) == 2) {
    if constexpr (FA == BY_ROWS)
      if (p.shape == WIDE) return launch_shape<T, FA, FB, MODE, Wide>(g, e, s);
    if (p.shape == LARGE) return launch_shape<T, FA, FB, MODE, Large>(g, e, s);
    if (p.shape == MIDDLE) return launch_shape<T, FA, FB, MODE, Middle>(g, e, s);
  }
  if constexpr (FB == BY_ROWS) {
    if (p.shape == FEW64) return launch_shape<T, FA, FB, MODE, Few64>(g, e, s);
    if (p.shape == FEW32) return launch_shape<T, FA, FB, MODE, Few32>(g, e, s);
    if constexpr (sizeof(T) == 2)
      if (p.shape == FEW128) return launch_shape<T, FA, FB, MODE, Few128>(g, e, s);
  }
  return launch_shape<T, FA, FB, MODE, Small>(g, e, s);
}

// C as T, through parts in fp32 ([splits][rows][features] at `parts`) where the contraction is cut.
template <typename T, int FA, int FB, int MODE = PLAIN>
hipError_t store_product(Plan p, const hpd_product_args& g, float* parts, T* out, int64_t stride, hipStream_t s) {
  const int64_t features = g.a.size, rows = g.b.size;
  if (p.splits == 1) return launch_product<T, FA, FB, MODE>(p, g, StoreProduct<T>{{out, nullptr}, {stride, 0}, rows, features, rows}, s);
  const hipError_t e = launch_product<T, FA, FB, MODE>(p, g, StorePart{parts, features, rows, 0}, s);
  return e != hipSuccess ? e : join_parts(parts, p.splits, features, rows, out, stride, s);
}

}  // namespace
