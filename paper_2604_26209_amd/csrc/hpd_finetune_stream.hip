// Fine-tuning attention in bf16: forward and gradients (formulas and operand scheme:
// hpd_finetune_attn.hip).  The other side's tokens stream through a ring of tiles in LDS that
// global_load_lds fills ahead of their use.
//
// Tiles: 32 rows of up to 64 or 128 bf16 values as they lie in memory, the 16-byte chunks of a row permuted: chunk c
// of row r lies at c ^ f(r), f(r) = 4 (r % 4) + (r / 4) % 4 for rows of 16 chunks and
// 4 (r / 2 % 2) + (r / 4) % 4 for rows of 8.  So both ways of reading a tile spread over all banks:
// one chunk of 16 successive rows (left operand of a score product), and the same 64 bytes of four
// successive rows (transposing read, left operand of a second product).
//
// Scores, softmax, delta and all sums are fp32.  The weights p and the scores' gradients ds are rounded to bf16 (half a step: 2^-8 of
// each) for the second products: the matrix instruction takes them in the type of the other operand, and value and
// remainder as two operands would be 3/2 of the forward kernel's products, 4/3 of dq's and 3/2 of dk/dv's.  The relative error against 64
// bits, in the root mean square, is 0.0019 to 0.0022 forward and 0.0024 to 0.0028 for the gradients, where rounding nothing but the
// outputs leaves 0.0016 and 0.0018 to 0.0022 (batches of perf/operators.py).
#include "hpd_finetune_dev.h"

namespace {

constexpr uint32_t BIAS = 4096;  // keeps a lane's offset positive (see Loader)

// The kernels are made for NB blocks of 32 channels.  Where a head ends inside the last block, its first chunk stands for
// the chunks behind it and the other side's operand is zero there.
template <int NB>
struct Rows {
  static constexpr int RB = NB <= 2 ? 128 : 256;  // bytes of a row
  static constexpr int TILE = 32 * RB;       // bytes of a tile
  static constexpr int CHUNKS = RB / 16;     // of a row
  static constexpr int STEPS = 2 * NB;       // products of a score
  static constexpr int BLOCKS = NB;          // blocks of 32 channels
  static constexpr int GROUP = 4096 / RB;    // rows that four load instructions bring
  static __device__ __forceinline__ int swizzle(int r) {
    return RB == 256 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
  // offset of chunk h of row n in a tile; chunk 2 s + h: ^ (s << 5)
  static __device__ __forceinline__ uint32_t row_offset(int n, int h) { return n * RB + ((h ^ swizzle(n)) << 4); }
  // transposing read, channel block b, rows 16 k + 8 e ..: (offset ^ (b << 6) ^ (e << 5)) + (16 k + 8 e) * RB
  static __device__ __forceinline__ uint32_t column_offset(int lane) {
    const int a = lane & 15, h = lane >> 5, r = 4 * h + (a >> 2);
    const int chunk = 2 * ((lane >> 4) & 1) + ((a & 3) >> 1);
    return r * RB + ((chunk ^ swizzle(r)) << 4) + (a & 1) * 8;
  }
};

// Four load instructions bring GROUP rows; instruction f rows f * GROUP / 4 .. .  Its offset field moves
// the address in memory and the one in LDS alike, so the lanes' offsets are f KB less, and a bias more.
// M0 is the compiler's: both forms put back what it held.
template <int NB>
struct Loader {
  using R = Rows<NB>;
  uint32_t off[4];
  int64_t stride;  // bytes between rows
  int32_t chunks;  // of a head's row
  bool near;       // a group's offsets fit 32 bits
  __device__ __forceinline__ void init(int64_t stride_elements, int32_t D, int lane) {
    stride = stride_elements * 2;
    chunks = D / 8;
    near = stride < 1 << 25;
#pragma unroll
    for (int f = 0; f < 4; ++f) off[f] = row(f, lane) * (uint32_t)stride + chunk(f, lane) - f * 1024 + BIAS;
  }
  static __device__ __forceinline__ int32_t row(int f, int lane) { return f * (1024 / R::RB) + lane / R::CHUNKS; }
  __device__ __forceinline__ uint32_t chunk(int f, int lane) const {
    const int32_t c = (lane % R::CHUNKS) ^ R::swizzle(row(f, lane));
    return c < chunks ? c << 4 : 0;
  }
  // GROUP rows from base (wave-uniform) to lds; rows past `last` (counted from base) are row `last` again
  // (zeros: 16 bytes of them, for the chunks behind the row's end)
  __device__ __forceinline__ void load(const char* base, uint32_t lds, int32_t last, int lane, const void* zeros = nullptr) const {
    lds = __builtin_amdgcn_readfirstlane(lds);
    uint32_t keep;
    if (!zeros && near && last >= R::GROUP - 1) {
      asm volatile(
          "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %1, %6\n\t"
          "global_load_lds_dwordx4 %2, %6 offset:1024\n\t"
          "global_load_lds_dwordx4 %3, %6 offset:2048\n\t"
          "global_load_lds_dwordx4 %4, %6 offset:3072\n\t"
          "s_mov_b32 m0, %0"
          : "=&s"(keep)
          : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(lds), "s"(uniform(base) - BIAS)
          : "memory");
    } else {
      const char* p[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const bool behind = zeros && ((lane % R::CHUNKS) ^ R::swizzle(row(f, lane))) >= chunks;
        p[f] = (behind ? reinterpret_cast<const char*>(zeros) : base + min(row(f, lane), last) * stride + chunk(f, lane)) - f * 1024;
      }
      asm volatile(
          "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %1, off\n\t"
          "global_load_lds_dwordx4 %2, off offset:1024\n\t"
          "global_load_lds_dwordx4 %3, off offset:2048\n\t"
          "global_load_lds_dwordx4 %4, off offset:3072\n\t"
          "s_mov_b32 m0, %0"
          : "=&s"(keep)
          : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "s"(lds)
          : "memory");
    }
  }
};

__device__ __forceinline__ bf16x8 lds_read(uint32_t at) {
  return __builtin_bit_cast(bf16x8, *(const __attribute__((address_space(3))) uint4v*)(uintptr_t)at);
}
__device__ __forceinline__ uint2 lds_read_tr(uint32_t at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) hpd::short4v*)(uintptr_t)at));
}
__device__ __forceinline__ floatx16 mfma(bf16x8 a, bf16x8 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// 32 columns of a transposed result (lane n: column n) times f, as 32 rows of D bf16 values through `turn`
// (TILE bytes of LDS of this wave's own); row r of the tile goes to out + r * stride, r < rows
template <int NB>
__device__ __forceinline__ void store_rows(char* turn, const floatx16* acc, float f, uint16_t* out, int64_t stride, int rows,
                                           int32_t D, int lane) {
  using R = Rows<NB>;
  const int n = lane & 31, h = lane >> 5;
#pragma unroll
  for (int b = 0; b < R::BLOCKS; ++b)
#pragma unroll
    for (int a = 0; a < 4; ++a) {  // channels 32 b + 8 a + 4 h ..: half h of chunk 4 b + a
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[b][4 * a + e] * f;
      const uint2 w = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
      *reinterpret_cast<uint2*>(turn + n * R::RB + (((4 * b + a) ^ (n & (R::CHUNKS - 1))) << 4) + h * 8) = w;
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < R::TILE / 1024; ++i) {
    const int r = i * (64 / R::CHUNKS) + lane / R::CHUNKS, c = lane % R::CHUNKS;
    const uint4 w = *reinterpret_cast<const uint4*>(turn + r * R::RB + ((c ^ (r & (R::CHUNKS - 1))) << 4));
    if (r < rows && c * 8 < D) *reinterpret_cast<uint4*>(out + r * stride + c * 8) = w;
  }
}

// a lane's chunks of a row of its own, zero from channel D on
template <int STEPS>
__device__ __forceinline__ void own_row(const uint16_t* row, int32_t D, int h, bf16x8 (&f)[STEPS]) {
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int32_t c = (2 * s + h) * 8;
    uint4 w = *reinterpret_cast<const uint4*>(row + (c < D ? c : 0));
    if (c >= D) w = make_uint4(0, 0, 0, 0);
    f[s] = __builtin_bit_cast(bf16x8, w);
  }
}

// The mask of a block of 32 tokens whose ranks differ (fine-tuning layout): a word per rank, bit i: token i's rank is no
// higher.  A lane fetches its word a round ahead; of a score it costs two instructions then.
struct Seen {
  const const_i32* off;     // of the sequence's blocks
  const const_i32* ranks;   // lowest and highest of them
  const uint32_t* words;
  __device__ __forceinline__ Seen(const FtArgs& a, int32_t blk0)
      : off((const const_i32*)(uintptr_t)(a.seen_off + blk0)), ranks((const const_i32*)(uintptr_t)(a.blk_rank + blk0)), words(a.seen) {}
  // tokens of block b with ranks up to this one
  __device__ __forceinline__ uint32_t word(int32_t b, int32_t rank) const {
    return words[(uint32_t)(off[b] + min(max(rank, ranks[2 * b] - 1), ranks[2 * b + 1]))];
  }
};
// -infinity where a bit is 0; bits: of the lane's column, by rows of the tile
__device__ __forceinline__ void hide(floatx16& s, uint32_t bits, int h) {
  bits >>= 4 * h;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const uint32_t seen = (uint32_t)__builtin_amdgcn_sbfe((int32_t)bits, tile_row(r, 0), 1);
    s[r] = __uint_as_float((__float_as_uint(s[r]) & seen) | (0xff800000u & ~seen));
  }
}

// The end of the kernels that join items: a workgroup of NB waves has 32 rows, wave x channels 32 x + 8 z + 4 h .. of row n
template <int NB>
struct Turn {
  static constexpr int PITCH = 64 * NB + 16, BYTES = 32 * PITCH;
  static __device__ __forceinline__ void store(char* turn, const float4* sum, float f, uint16_t* out, int64_t stride, int rows,
                                               int32_t D) {
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, x = threadIdx.x >> 6;
#pragma unroll
    for (int z = 0; z < 4; ++z)
      *reinterpret_cast<uint2*>(turn + n * PITCH + x * 64 + z * 16 + h * 8) =
          make_uint2(cvt_pk_bf16(sum[z].x * f, sum[z].y * f), cvt_pk_bf16(sum[z].z * f, sum[z].w * f));
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * 4 * NB; i += 64 * NB) {
      const int r = i / (4 * NB), c = i % (4 * NB);
      if (r < rows && c * 8 < D)
        *reinterpret_cast<uint4*>(out + r * stride + c * 8) = *reinterpret_cast<const uint4*>(turn + r * PITCH + c * 16);
    }
  }
};

// ---------------------------------------------------------------------------------------
// Forward and dq: four waves of 32 queries of one head; rounds of 64 keys, two rounds in LDS.  An item is a run of a
// tile's rounds; what the waves of a tile with several have goes to `partial`, register by register, and a second kernel
// joins it.  128 queries share a tile of keys because its bytes pass LDS once per wave anyway; two workgroups per CU fill the
// registers and 128 of 160 KB of LDS, and one's products run beside the other's exponentials.
// ---------------------------------------------------------------------------------------
// LDS addresses of a lane's operands in the first tile of a stage
template <int NB>
struct Addresses {
  using R = Rows<NB>;
  uint32_t row[R::STEPS], col[2 * R::BLOCKS];
  __device__ __forceinline__ Addresses(uint32_t base, int lane) {
#pragma unroll
    for (int s = 0; s < R::STEPS; ++s) row[s] = base + (R::row_offset(lane & 31, lane >> 5) ^ (s << 5));
#pragma unroll
    for (int c = 0; c < 2 * R::BLOCKS; ++c) col[c] = base + (R::column_offset(lane) ^ (c >> 1 << 6) ^ ((c & 1) << 5));
  }
  // to the other stage (base is a multiple of 2 * stage)
  __device__ __forceinline__ void flip(uint32_t stage) {
#pragma unroll
    for (int s = 0; s < R::STEPS; ++s) row[s] ^= stage;
#pragma unroll
    for (int c = 0; c < 2 * R::BLOCKS; ++c) col[c] ^= stage;
  }
  __device__ __forceinline__ bf16x8 rows(int s, int at) const { return lds_read(row[s] + at); }
  __device__ __forceinline__ bf16x8 columns(int b, int k, int at) const {
    const uint2 lo = lds_read_tr(col[2 * b] + at + 16 * k * R::RB);
    const uint2 hi = lds_read_tr(col[2 * b + 1] + at + (16 * k + 8) * R::RB);
    return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
  }
};

template <int NB>
struct QueryTile {
  using R = Rows<NB>;
  static constexpr int STAGE = 4 * R::TILE;  // 64 rows of k, 64 rows of v
  static constexpr int LOADS = 128 / R::GROUP;  // load instructions of a wave for a round, and for 32 rows of its own
  static constexpr int SUMS = 32 * 32 * NB;  // fp32 sums of a wave
  static constexpr int PARTIAL = SUMS + 64;  // of a wave in `partial`: sums; forward: reference points, sums of the weights
  const FtArgs& a;
  hpd_ft_item t;
  int lane, n, h, wave;
  int32_t hq, hk, q_first, i, ic;
  int64_t token;
  bool active;
  int32_t q_min, q_max;  // ranks of the wave's queries
  const const_i32* blk_rank;
  Loader<NB> loader;
  const char* src;
  uint32_t ring_lds;

  __device__ __forceinline__ QueryTile(const FtArgs& args, const hpd_ft_item* items, const uint16_t* k, const uint16_t* v,
                                     const char* ring)
      : a(args) {
    lane = threadIdx.x & 63;
    n = lane & 31;
    h = lane >> 5;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroup b runs on XCD b % 8: the query tiles and heads that read the same keys stay together
    const int32_t G = a.Hq / a.Hkv, rest = blockIdx.x / a.Hkv;
    hk = blockIdx.x % a.Hkv;
    hq = hk * G + rest % G;
    t = items[rest / G];
    q_first = t.row0 + wave * 32;
    i = q_first + n;
    ic = min(i, t.len - 1);
    active = q_first < t.len;
    token = t.seq0 + (int64_t)ic;
    // this wave's part of a round: waves 0 and 1 keys, 2 and 3 values
    loader.init(wave < 2 ? a.sk : a.sv, a.D, lane);
    src = reinterpret_cast<const char*>(wave < 2 ? k + t.seq0 * a.sk : v + t.seq0 * a.sv) + (int64_t)hk * a.D * 2;
    ring_lds = lds_address(ring);
    blk_rank = (const const_i32*)(uintptr_t)(a.blk_rank + t.blk0);
    const int32_t own = min(q_first, t.len - 1) / 32;
    q_min = blk_rank[2 * own];
    q_max = blk_rank[2 * own + 1];
  }
  __device__ __forceinline__ void issue(int32_t round) const {
    const uint32_t dst = ring_lds + ((round - t.begin) & 1) * STAGE + (wave >> 1) * 2 * R::TILE;
#pragma unroll
    for (int j = 0; j < 32 / R::GROUP; ++j) {
      const int32_t row = R::RB == 256 ? 32 * j + 16 * (wave & 1) : 32 * (wave & 1);
      const int32_t first = min(round * 64 + row, t.len - 1);
      loader.load(src + first * loader.stride, dst + row * R::RB, t.len - 1 - first, lane);
    }
  }
  // The wave's own rows of a tensor, through its quarter of a stage that is free: whole rows at a time (the operand's layout
  // straight from memory: 32 lines for every 16 bytes of 32 rows, fetched again for the next ones).
  __device__ __forceinline__ void load_own(const uint16_t* x, int64_t stride, int stage) const {
    Loader<NB> own;
    own.init(stride, a.D, lane);
    const int32_t row0 = min(q_first, t.len - 1);
    const char* const base = reinterpret_cast<const char*>(x + (t.seq0 + (int64_t)row0) * stride + hq * a.D);
#pragma unroll
    for (int j = 0; j < 32 / R::GROUP; ++j) {
      const int32_t first = min(j * R::GROUP, t.len - 1 - row0);
      own.load(base + first * own.stride, ring_lds + stage * STAGE + wave * R::TILE + j * R::GROUP * R::RB, t.len - 1 - row0 - first,
               lane);
    }
  }
  __device__ __forceinline__ void read_own(const Addresses<NB>& at, int stage, bf16x8 (&f)[R::STEPS]) const {
#pragma unroll
    for (int s = 0; s < R::STEPS; ++s) {
      const bf16x8 x = at.rows(s, stage * STAGE + wave * R::TILE);
      f[s] = (2 * s + h) * 8 < a.D ? x : bf16x8{};
    }
  }
  __device__ __forceinline__ float* partial_of(float* partial) const {
    return partial + (((int64_t)t.slot * a.Hq + hq) * 4 + wave) * PARTIAL;
  }
  __device__ __forceinline__ void put(float* p, const floatx16* acc) const {
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int z = 0; z < 4; ++z)
        *reinterpret_cast<float4*>(p + (x * 4 + z) * 256 + lane * 4) =
            make_float4(acc[x][4 * z], acc[x][4 * z + 1], acc[x][4 * z + 2], acc[x][4 * z + 3]);
  }
  // block b of 32 keys has a key that a query of the wave sees / one that a query does not see (the first blocks of a
  // sequence, its prompt, without a look at their ranks: it takes as long as the rest of a round's scalar work)
  __device__ __forceinline__ bool reaches(int32_t b) const {
    return active && b * 32 <= q_first && (b < t.plain || blk_rank[2 * b] <= q_max);
  }
  __device__ __forceinline__ bool masked(int32_t b) const {
    return b * 32 >= q_first || (b >= t.plain && blk_rank[2 * b + 1] > q_min);
  }
  // words of the blocks of a round, for the lane's query
  __device__ __forceinline__ void fetch(const Seen& seen, int32_t round, int32_t rank, uint32_t (&bits)[2]) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int32_t b = 2 * round + j;
      bits[j] = 0;
      if (active && b * 32 <= q_first) bits[j] = masked(b) ? seen.word(b, rank) : ~0u;
    }
  }
  __device__ __forceinline__ void mask(floatx16& s, int32_t b, uint32_t bits) const {
    hide(s, b * 32 == q_first ? bits & ~0u >> (31 - n) : bits, h);
  }
};

// o_i = sum_j p_ij v_j / l_i in one pass, with a reference point that moves when the maximum leaves it by 2^8.  Bound by matrix and
// vector instructions by turns, under a clock that falls with them: 4 x 5900 tokens, 64/8 heads of 128: 2.3 ms, 950 TFLOP/s of visible
// pairs (a large library product: 1190), matrix units busy 49 %, vector units 46 %.
template <int NB>
__global__ void __launch_bounds__(256, 2) ft_stream_forward_kernel(FtArgs a, const hpd_ft_item* __restrict__ items,
                                                                  const uint16_t* __restrict__ q,
                                                                  const uint16_t* __restrict__ k,
                                                                  const uint16_t* __restrict__ v, uint16_t* __restrict__ out,
                                                                  float* __restrict__ lse, float* __restrict__ partial) {
  using R = Rows<NB>;
  using Q = QueryTile<NB>;
  __shared__ __attribute__((aligned(2 * Q::STAGE))) char ring[2 * Q::STAGE];
  const Q w(a, items, k, v, ring);
  Addresses<NB> at(w.ring_lds, w.lane);
  int32_t rank_i[1] = {a.rank[w.token]};
  bf16x8 qf[R::STEPS];
  w.load_own(q, a.sq, 1);
  w.issue(w.t.begin);
  wait_vector_memory<Q::LOADS>();  // the queries
  w.read_own(at, 1, qf);
  arrived(qf);
  arrived(rank_i);
  const Seen seen(a, w.t.blk0);
  uint32_t bits[2], next[2];
  w.fetch(seen, w.t.begin, rank_i[0], next);
  const float c = a.scale * LOG2E;

  floatx16 acc[R::BLOCKS];
  zero(acc, R::BLOCKS);
  float m = NEG_BIG, l = 0.f;  // reference point (log2 units; within 2^8 of the maximum) and this lane's share of the sum

  // One round, two blocks of 32 keys: both scores, one look at the maximum, then the second block's weights while the
  // first block's products with v run.
  auto step = [&](int32_t b) __attribute__((always_inline)) {
    floatx16 s[2] = {};
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int x = 0; x < R::STEPS; ++x) s[j] = mfma(at.rows(x, j * R::TILE), qf[x], s[j]);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (w.masked(b + j)) w.mask(s[j], b + j, bits[j]);
    float top = s[0][0];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[j][r]);
    top *= c;
    if (__any(top > m + MAX_SLACK)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = fmaxf(m, top), alpha = fast_exp2(m - next);
      m = next;
      l *= alpha;
#pragma unroll
      for (int x = 0; x < R::BLOCKS; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[x][r] *= alpha;
    }
    float p[2][16], l0 = 0.f, l1 = 0.f;
    auto weights = [&](int j, int first, int last) __attribute__((always_inline)) {
#pragma unroll
      for (int r = first; r < last; ++r) {
        p[j][r] = fast_exp2(fmaf(s[j][r], c, -m));
        if (r & 1) l1 += p[j][r];
        else l0 += p[j][r];
      }
    };
    bf16x8 f[3], pf[2][2];
    auto ld = [&](int i) __attribute__((always_inline)) -> bf16x8 {  // columns of v, block by block
      constexpr int C = 2 * R::BLOCKS;
      return at.columns(i % C / 2, i % 2, (2 + i / C) * R::TILE);
    };
    f[0] = ld(0);
    f[1] = ld(1);
    weights(0, 0, 16);
    pf[0][0] = pack8(p[0]);
    pf[0][1] = pack8(p[0] + 8);
    __builtin_amdgcn_sched_barrier(0);
    constexpr int C = 2 * R::BLOCKS;
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
      if (i + 2 < 2 * C) f[(i + 2) % 3] = ld(i + 2);
      acc[i % C / 2] = mfma(f[i % 3], pf[i / C][i % 2], acc[i % C / 2]);
      if (i < C) weights(1, 16 * i / C, 16 * (i + 1) / C);
      if (i == C / 2 - 1) pf[1][0] = pack8(p[1]);
      if (i == C - 1) pf[1][1] = pack8(p[1] + 8);
      __builtin_amdgcn_sched_barrier(0);
    }
    l += l0 + l1;
  };
  for (int32_t round = w.t.begin; round < w.t.end; ++round) {
    wait_vector_memory<0>();
    arrived(next);
    bits[0] = next[0];
    bits[1] = next[1];
    wait_lds_and_barrier();  // the round is in LDS, the other half of the ring is free
    if (round + 1 < w.t.end) {
      w.issue(round + 1);
      w.fetch(seen, round + 1, rank_i[0], next);
    }
    if (w.reaches(2 * round) || w.reaches(2 * round + 1)) step(2 * round);
    at.flip(Q::STAGE);
  }
  wait_lds_and_barrier();
  if (!w.active) return;
  l += __shfl_xor(l, 32);
  if (w.t.slot >= 0) {
    float* const p = w.partial_of(partial);
    w.put(p, acc);
    p[Q::SUMS + w.lane] = w.h ? l : m;
    return;
  }
  if (w.h == 0 && w.i < w.t.len) lse[w.hq * a.N + w.token] = (m + __builtin_amdgcn_logf(l)) * LN2;
  store_rows<NB>(ring + w.wave * R::TILE, acc, 1.f / l, out + ((w.t.seq0 + (int64_t)w.q_first) * a.Hq + w.hq) * a.D,
                 (int64_t)a.Hq * a.D, w.t.len - w.q_first, a.D, w.lane);
}

// Joins the items of a tile.  A workgroup has 32 queries of a head, a wave one block of channels; four items are on
// their way at a time.
template <int NB>
__global__ void __launch_bounds__(64 * NB) ft_stream_join_kernel(FtArgs a, const hpd_ft_item* __restrict__ joins,
                                                               const float* __restrict__ partial, uint16_t* __restrict__ out,
                                                               float* __restrict__ lse) {
  using Q = QueryTile<NB>;
  __shared__ __attribute__((aligned(16))) char turn[Turn<NB>::BYTES];
  const int lane = threadIdx.x & 63, n = lane & 31, x = threadIdx.x >> 6;
  const int32_t rows32 = blockIdx.x & 3, hq = (blockIdx.x >> 2) % a.Hq;
  const hpd_ft_item t = joins[(blockIdx.x >> 2) / a.Hq];  // slots [slot, slot + end)
  const int32_t first = t.row0 + rows32 * 32;
  if (first >= t.len) return;
  const int64_t step = (int64_t)a.Hq * 4 * Q::PARTIAL;
  const float* const p = partial + (((int64_t)t.slot * a.Hq + hq) * 4 + rows32) * Q::PARTIAL;
  float4 sum[4] = {};
  float m = NEG_BIG, l = 0.f;
  for (int32_t i = 0; i < t.end; i += 4) {
    float4 w[4][4];
    float mi[4], li[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      mi[j] = NEG_BIG;
      if (i + j >= t.end) continue;
      const float* const from = p + (i + j) * step;
      mi[j] = from[Q::SUMS + n];
      li[j] = from[Q::SUMS + 32 + n];
#pragma unroll
      for (int z = 0; z < 4; ++z) w[j][z] = *reinterpret_cast<const float4*>(from + (x * 4 + z) * 256 + lane * 4);
    }
    const float top = fmaxf(fmaxf(fmaxf(mi[0], mi[1]), fmaxf(mi[2], mi[3])), m), alpha = fast_exp2(m - top);
    m = top;
    l *= alpha;
#pragma unroll
    for (int z = 0; z < 4; ++z) sum[z] = make_float4(sum[z].x * alpha, sum[z].y * alpha, sum[z].z * alpha, sum[z].w * alpha);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i + j >= t.end) continue;
      const float f = fast_exp2(mi[j] - m);
      l = fmaf(li[j], f, l);
#pragma unroll
      for (int z = 0; z < 4; ++z)
        sum[z] = make_float4(fmaf(w[j][z].x, f, sum[z].x), fmaf(w[j][z].y, f, sum[z].y), fmaf(w[j][z].z, f, sum[z].z),
                             fmaf(w[j][z].w, f, sum[z].w));
    }
  }
  if (threadIdx.x < 32 && first + n < t.len) lse[hq * a.N + t.seq0 + first + n] = (m + __builtin_amdgcn_logf(l)) * LN2;
  Turn<NB>::store(turn, sum, 1.f / l, out + ((t.seq0 + (int64_t)first) * a.Hq + hq) * a.D, (int64_t)a.Hq * a.D, t.len - first, a.D);
}

// stat, which this kernel makes and the dk/dv kernel reads: per (head, token) -lse * sqrt(D), where its row's score
// products start, then -delta, delta_i = do_i . o_i, where its row's products with v start:
// p = exp((q . k - lse sqrt(D)) / sqrt(D)).
// dq_i = sum_j ds_ij k_j, ds = p (do v - delta) / sqrt(D); s and do v are made again here and in the dk/dv kernel: sums of dq over
// key tiles would need atomics, whose order changes the result, or ds in memory, two bytes per pair and head.  2 x 6000 tokens, 64/8
// heads of 128: 1.7 ms, matrix units busy 59 %; 32 x 617 tokens, 32/8 heads: 0.28 ms, 32 % and 3.3 TB/s (starts of short
// workgroups, queries and gradients of the output read for few rounds).
template <int NB>
__global__ void __launch_bounds__(256, 2) ft_stream_dq_kernel(FtArgs a, const hpd_ft_item* __restrict__ items,
                                                             const uint16_t* __restrict__ q,
                                                             const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                             const uint16_t* __restrict__ out, const uint16_t* __restrict__ d_out,
                                                             const float* __restrict__ lse, float* __restrict__ stat,
                                                             float* __restrict__ partial, uint16_t* __restrict__ dq) {
  using R = Rows<NB>;
  using Q = QueryTile<NB>;
  __shared__ __attribute__((aligned(2 * Q::STAGE))) char ring[2 * Q::STAGE];
  const Q w(a, items, k, v, ring);
  Addresses<NB> at(w.ring_lds, w.lane);
  bf16x8 qf[R::STEPS], of[R::STEPS];
  float nl[1], nd[1];
  const float minus_lse = -lse[w.hq * a.N + w.token];
  int32_t rank_i[1] = {a.rank[w.token]};
  {
    const int64_t row = (int64_t)a.Hq * a.D;
    bf16x8 o[R::STEPS];
    w.load_own(q, a.sq, 0);
    w.load_own(d_out, row, 1);
    wait_vector_memory<0>();
    w.read_own(at, 0, qf);
    w.read_own(at, 1, of);
    arrived(qf);
    arrived(of);
    wait_lds_and_barrier();  // (stage 0 is the round's from here on)
    w.load_own(out, row, 1);
    w.issue(w.t.begin);
    wait_vector_memory<Q::LOADS>();
    w.read_own(at, 1, o);
    float delta = 0.f;
#pragma unroll
    for (int s = 0; s < R::STEPS; ++s) {
      float y[8], z[8];
      unpack8(__builtin_bit_cast(uint4, of[s]), y);
      unpack8(__builtin_bit_cast(uint4, o[s]), z);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf(y[e], z[e], delta);
    }
    nd[0] = -(delta + __shfl_xor(delta, 32));
    nl[0] = LOG2E * minus_lse;
    if (w.t.begin == 0 && w.h == 0 && w.i < w.t.len) {
      stat[w.hq * a.N + w.token] = minus_lse / a.scale;
      stat[(a.Hq + w.hq) * a.N + w.token] = nd[0];
    }
  }
  arrived(nl);
  arrived(nd);
  arrived(rank_i);
  const Seen seen(a, w.t.blk0);
  uint32_t bits[2], next[2];
  w.fetch(seen, w.t.begin, rank_i[0], next);
  const float c = a.scale * LOG2E;
  floatx16 acc[R::BLOCKS];
  zero(acc, R::BLOCKS);
  // One round, two blocks of 32 keys.  The first block's weights and gradients are made while the second block's
  // score products run, the second block's while the first block's last products do.
  auto step = [&](int32_t b) __attribute__((always_inline)) {
    constexpr int S = R::STEPS, C = 2 * R::BLOCKS;
    floatx16 s[2] = {}, dp[2] = {};
    bf16x8 f[3], df[2][2];
    float e[2][16];
    // operands: rows of k, v of block 0, then of block 1, then columns of k
    auto ld = [&](int i) __attribute__((always_inline)) -> bf16x8 {
      if (i < 4 * S) return at.rows(i % S, (2 * (i / S % 2) + i / (2 * S)) * R::TILE);
      i -= 4 * S;
      return at.columns(i % C / 2, i % 2, i / C * R::TILE);
    };
    auto gradient = [&](int j, int first, int last) __attribute__((always_inline)) {
#pragma unroll
      for (int r = first; r < last; ++r) e[j][r] = fast_exp2(fmaf(s[j][r], c, nl[0])) * (dp[j][r] + nd[0]);
    };
    f[0] = ld(0);
    f[1] = ld(1);
#pragma unroll
    for (int i = 0; i < 4 * S; ++i) {
      f[(i + 2) % 3] = ld(i + 2);
      const int j = i / (2 * S), x = i % S;
      if (i / S % 2 == 0) s[j] = mfma(f[i % 3], qf[x], s[j]);
      else dp[j] = mfma(f[i % 3], of[x], dp[j]);
      if (i == 2 * S - 1 && w.masked(b)) w.mask(s[0], b, bits[0]);
      if (i >= 2 * S) {  // (a step behind: the last product is on its way)
        const int y = i - 2 * S;
        gradient(0, 16 * (y > 0 ? y - 1 : 0) / (2 * S - 1), 16 * y / (2 * S - 1));
        if (y == S) df[0][0] = pack8(e[0]);
        if (y == 2 * S - 1) df[0][1] = pack8(e[0] + 8);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (w.masked(b + 1)) w.mask(s[1], b + 1, bits[1]);
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
      const int at_ = 4 * S + i;
      if (i + 2 < 2 * C) f[(at_ + 2) % 3] = ld(at_ + 2);
      acc[i % C / 2] = mfma(f[at_ % 3], df[i / C][i % 2], acc[i % C / 2]);
      if (i < C) gradient(1, 16 * i / C, 16 * (i + 1) / C);
      if (i == C / 2 - 1) df[1][0] = pack8(e[1]);
      if (i == C - 1) df[1][1] = pack8(e[1] + 8);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int32_t round = w.t.begin; round < w.t.end; ++round) {
    wait_vector_memory<0>();
    arrived(next);
    bits[0] = next[0];
    bits[1] = next[1];
    wait_lds_and_barrier();
    if (round + 1 < w.t.end) {
      w.issue(round + 1);
      w.fetch(seen, round + 1, rank_i[0], next);
    }
    if (w.reaches(2 * round) || w.reaches(2 * round + 1)) step(2 * round);
    at.flip(Q::STAGE);
  }
  wait_lds_and_barrier();
  if (!w.active) return;
  if (w.t.slot >= 0) {
    w.put(w.partial_of(partial), acc);
    return;
  }
  store_rows<NB>(ring + w.wave * R::TILE, acc, a.scale, dq + (w.t.seq0 + (int64_t)w.q_first) * a.sdq + w.hq * a.D, a.sdq,
                 w.t.len - w.q_first, a.D, w.lane);
}

// dk and dv: four waves of 32 keys of one kv head, over the queries of all its heads; rounds of 32 queries, two in
// LDS.  The wave's keys are in registers, its values, for want of room there, in LDS.  An item is a run of
// a tile's rounds; the sums of a tile that is cut into several go to `partial`, register by register, and a
// second kernel adds them up.  dv_j = sum_i p_ij do_i, dk_j = sum_i ds_ij q_i, over the heads of the kv head as well, in registers.
// 2 x 6000 tokens, 64/8 heads of 128: 2.2 ms, matrix units busy 59 %; 32 x 617 tokens, 32/8 heads: 0.27 ms, 45 % and 3.5 TB/s.  All
// registers are taken; the 40 KB that a wave reads from LDS in a round are, at 128 bytes a cycle and CU, 1.25 times its products' time.
template <int NB>
struct KeyTile {
  static constexpr int SUMS = 32 * 32 * NB;          // fp32 sums of a wave
  static constexpr int PARTIAL = 2 * 4 * SUMS;       // of an item and kv head: dk and dv of four waves
};
template <int NB>
__global__ void __launch_bounds__(256, 2) ft_stream_dkv_kernel(FtArgs a, const hpd_ft_item* __restrict__ items,
                                                              const uint16_t* __restrict__ q, const uint16_t* __restrict__ k,
                                                              const uint16_t* __restrict__ v, const uint16_t* __restrict__ d_out,
                                                              const float* __restrict__ stat, float* __restrict__ partial,
                                                              uint16_t* __restrict__ dk, uint16_t* __restrict__ dv) {
  using R = Rows<NB>;
  constexpr int STAGE = 2 * R::TILE;  // rows of q and of do
  __shared__ __attribute__((aligned(2 * STAGE))) char ring[2 * STAGE];
  __shared__ __attribute__((aligned(1024))) char values[4 * R::TILE];
  __shared__ __attribute__((aligned(1024))) float stats[2][64];  // of a round's rows: -lse sqrt(D), then -delta
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t G = a.Hq / a.Hkv, hk = blockIdx.x % a.Hkv;
  const hpd_ft_item t = items[blockIdx.x / a.Hkv];
  const int32_t k_first = t.row0 + wave * 32, j = k_first + n;
  const bool active = k_first < t.len;
  const int32_t own = min(k_first, t.len - 1);  // first key of the wave, if it has one
  const int64_t token = t.seq0 + (int64_t)min(j, t.len - 1);

  // this wave's part of a round: waves 0 and 1 queries, 2 and 3 gradients of the output
  Loader<NB> loader;
  loader.init(wave < 2 ? a.sq : (int64_t)a.Hq * a.D, a.D, lane);
  const char* const src = reinterpret_cast<const char*>(wave < 2 ? q + t.seq0 * a.sq : d_out + (int64_t)t.seq0 * a.Hq * a.D);
  const uint32_t ring_lds = lds_address(ring), stats_lds = lds_address(stats);
  const int32_t b_first = t.row0 / 32, per_head = (t.len + 31) / 32 - b_first;
  int32_t next_g = t.begin / per_head, next_b = b_first + t.begin % per_head;  // the round that is requested next
  auto issue = [&](int32_t slot) {
    const int32_t hq = hk * G + next_g;
    if (R::RB == 256 || (wave & 1) == 0) {  // (a tile of 64 channels is one group)
      const int32_t row = R::RB == 256 ? 16 * (wave & 1) : 0, first = min(next_b * 32 + row, t.len - 1);
      loader.load(src + first * loader.stride + hq * a.D * 2, ring_lds + slot * STAGE + (wave >> 1) * R::TILE + row * R::RB,
                  t.len - 1 - first, lane);
    }
    if (wave == 3) {
      const float* p = stat + (h * (int64_t)a.Hq + hq) * a.N + t.seq0 + min(next_b * 32 + n, t.len - 1);
      const uint32_t dst = __builtin_amdgcn_readfirstlane(stats_lds + slot * 256);
      uint32_t keep;
      asm volatile(
          "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
          "global_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
          : "=&s"(keep)
          : "v"(p), "s"(dst)
          : "memory");
    }
    if (++next_b == b_first + per_head) {
      next_b = b_first;
      ++next_g;
    }
  };
  int32_t b = next_b;
  if (t.begin < t.end) issue(0);
  {
    Loader<NB> own_values;
    own_values.init(a.sv, a.D, lane);
    const char* const base = reinterpret_cast<const char*>(v + t.seq0 * a.sv + (int64_t)hk * a.D);
    const void* const zeros = a.D < 32 * NB ? a.rank + a.N : nullptr;
#pragma unroll
    for (int x = 0; x < 32 / R::GROUP; ++x) {
      const int32_t first = min(own + x * R::GROUP, t.len - 1);
      own_values.load(base + first * own_values.stride, lds_address(values) + wave * R::TILE + x * R::GROUP * R::RB,
                      t.len - 1 - first, lane, zeros);
    }
  }
  bf16x8 kf[R::STEPS];
  own_row(k + token * a.sk + (int64_t)hk * a.D, a.D, h, kf);
  int32_t rank_j[1] = {a.rank[token]};
  arrived(kf);
  arrived(rank_j);
  const Seen seen(a, t.blk0);
  uint32_t next[1], bits;  // of a round's queries: ranks below the lane's key's
  const const_i32* const blk_rank = (const const_i32*)(uintptr_t)(a.blk_rank + t.blk0);
  const int32_t k_min = blk_rank[2 * (own / 32)], k_max = blk_rank[2 * (own / 32) + 1];
  const float c = a.scale * LOG2E;
  const uint32_t row_at = ring_lds + R::row_offset(n, h), col_at = ring_lds + R::column_offset(lane);
  const uint32_t to_values = lds_address(values) + wave * R::TILE - ring_lds;

  floatx16 acc_k[R::BLOCKS], acc_v[R::BLOCKS];
  zero(acc_k, R::BLOCKS);
  zero(acc_v, R::BLOCKS);
  auto step = [&](int slot, bool masked) __attribute__((always_inline)) {
    constexpr int S = R::STEPS, C = 2 * R::BLOCKS;
    uint32_t row = row_at, col = col_at;
    asm volatile("" : "+v"(row), "+v"(col));  // (the addresses made from them are not kept for the next round: there is no room)
    auto start = [&](int at) __attribute__((always_inline)) {  // one number per row of the tile, as a result's registers lie
      floatx16 x;
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const float4 w = *reinterpret_cast<const float4*>(&stats[slot][at + 8 * z + 4 * h]);
        x[4 * z] = w.x; x[4 * z + 1] = w.y; x[4 * z + 2] = w.z; x[4 * z + 3] = w.w;
      }
      return x;
    };
    // left operands: rows of q, rows of do, columns of do, columns of q
    auto ld = [&](int i) __attribute__((always_inline)) -> bf16x8 {
      if (i < 2 * S) return lds_read((row ^ (i % S << 5)) + slot * STAGE + i / S * R::TILE);
      i -= 2 * S;
      const uint32_t at = (col ^ (i % C / 2 << 6)) + slot * STAGE + (i < C ? R::TILE : 0) + i % 2 * 16 * R::RB;
      const uint32_t at8 = (col ^ (i % C / 2 << 6) ^ 32) + slot * STAGE + (i < C ? R::TILE : 0) + (i % 2 * 16 + 8) * R::RB;
      const uint2 lo = lds_read_tr(at), hi = lds_read_tr(at8);
      return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
    };
    bf16x8 f[3], g[2], pf[2], df[2];
    floatx16 s = start(0), dp;
    f[0] = ld(0);
    f[1] = ld(1);
#pragma unroll
    for (int i = 0; i < S; ++i) {
      f[(i + 2) % 3] = ld(i + 2);
      s = mfma(f[i % 3], kf[i], s);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (masked) {
      uint32_t x = ~bits;
      if (b * 32 == k_first) x &= ~0u << n;
      if ((b + 1) * 32 > t.len) x &= ~(~0u << (t.len - b * 32));
      hide(s, x, h);
    }
    dp = start(32);
    g[0] = lds_read(row + to_values);
#pragma unroll
    for (int i = 0; i < S; ++i) {
      f[(S + i + 2) % 3] = ld(S + i + 2);
      if (i + 1 < S) g[(i + 1) % 2] = lds_read((row ^ ((i + 1) << 5)) + to_values);
      dp = mfma(f[(S + i) % 3], g[i % 2], dp);
#pragma unroll
      for (int r = 16 * i / S; r < 16 * (i + 1) / S; ++r) s[r] = fast_exp2(s[r] * c);
      __builtin_amdgcn_sched_barrier(0);
    }
    float e[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) e[r] = s[r];
    pf[0] = pack8(e);
    pf[1] = pack8(e + 8);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
      const int at = 2 * S + i;
      if (i + 2 < 2 * C) f[(at + 2) % 3] = ld(at + 2);
      if (i < C) {
        acc_v[i / 2] = mfma(f[at % 3], pf[i % 2], acc_v[i / 2]);
#pragma unroll
        for (int r = 16 * i / C; r < 16 * (i + 1) / C; ++r) e[r] *= dp[r];
        if (i == C / 2 - 1) df[0] = pack8(e);
        if (i == C - 1) df[1] = pack8(e + 8);
      } else {
        acc_k[(i - C) / 2] = mfma(f[at % 3], df[i % 2], acc_k[(i - C) / 2]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto masked = [&](int32_t x) {
    return x * 32 < k_first + 31 || (x + 1) * 32 > t.len || (k_max > 0 && k_max > blk_rank[2 * x]);
  };
  auto fetch = [&](int32_t x) {
    next[0] = 0;
    if (masked(x)) next[0] = seen.word(x, rank_j[0] - 1);
  };
  fetch(b);
  auto turn = [&](int32_t round, int slot) __attribute__((always_inline)) {
    wait_vector_memory<0>();
    arrived(next);
    bits = next[0];
    wait_lds_and_barrier();
    const int32_t after = b + 1 == b_first + per_head ? b_first : b + 1;
    if (round + 1 < t.end) {
      issue(slot ^ 1);
      fetch(after);
    }
    if (active && b * 32 + 31 >= k_first && (k_min == 0 || k_min <= blk_rank[2 * b + 1])) step(slot, masked(b));
    b = after;
  };
  for (int32_t round = t.begin; round < t.end; round += 2) {
    turn(round, 0);
    if (round + 1 < t.end) turn(round + 1, 1);
  }
  wait_vector_memory<0>();
  wait_lds_and_barrier();
  if (t.slot >= 0) {
    float* p = partial + ((int64_t)t.slot * a.Hkv + hk) * KeyTile<NB>::PARTIAL + wave * KeyTile<NB>::SUMS + lane * 4;
#pragma unroll
    for (int x = 0; x < R::BLOCKS; ++x)
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const int at = (x * 4 + z) * 256;
        *reinterpret_cast<float4*>(p + at) = make_float4(acc_k[x][4 * z], acc_k[x][4 * z + 1], acc_k[x][4 * z + 2], acc_k[x][4 * z + 3]);
        *reinterpret_cast<float4*>(p + at + 4 * KeyTile<NB>::SUMS) =
            make_float4(acc_v[x][4 * z], acc_v[x][4 * z + 1], acc_v[x][4 * z + 2], acc_v[x][4 * z + 3]);
      }
    return;
  }
  if (!active) return;
  const int64_t first = t.seq0 + (int64_t)k_first;
  store_rows<NB>(ring + wave * R::TILE, acc_v, 1.f, dv + first * a.sdv + hk * a.D, a.sdv, t.len - k_first, a.D, lane);
  store_rows<NB>(ring + wave * R::TILE, acc_k, a.scale, dk + first * a.sdk + hk * a.D, a.sdk, t.len - k_first, a.D, lane);
}

// Adds up the partial sums of the tiles of keys (n_key workgroups) and of queries, in the order of their items.  A
// workgroup has 32 rows of dk, dv or dq of one head, a wave one block of channels; the sums of four items are on their way at a
// time.
template <int NB>
__global__ void __launch_bounds__(64 * NB) ft_stream_join_gradients_kernel(FtArgs a, uint32_t n_key,
                                                                         const hpd_ft_item* __restrict__ key_joins,
                                                                         const hpd_ft_item* __restrict__ query_joins,
                                                                         const float* __restrict__ key_partial,
                                                                         const float* __restrict__ query_partial,
                                                                         uint16_t* __restrict__ dq, uint16_t* __restrict__ dk,
                                                                         uint16_t* __restrict__ dv) {
  using K = KeyTile<NB>;
  using Q = QueryTile<NB>;
  __shared__ __attribute__((aligned(16))) char turn[Turn<NB>::BYTES];
  const int lane = threadIdx.x & 63, x = threadIdx.x >> 6;
  const bool keys = blockIdx.x < n_key;
  const uint32_t rest = keys ? blockIdx.x >> 1 : blockIdx.x - n_key;
  const int32_t y = blockIdx.x & 1, rows32 = rest & 3, heads = keys ? a.Hkv : a.Hq, head = (rest >> 2) % heads;  // (y: dv)
  const hpd_ft_item t = (keys ? key_joins : query_joins)[(rest >> 2) / heads];  // slots [slot, slot + end)
  const int32_t first = t.row0 + rows32 * 32;
  if (first >= t.len) return;
  const int64_t step = keys ? (int64_t)heads * K::PARTIAL : (int64_t)heads * 4 * Q::PARTIAL;
  const float* const p = (keys ? key_partial + ((int64_t)t.slot * heads + head) * K::PARTIAL + (4 * y + rows32) * K::SUMS
                               : query_partial + (((int64_t)t.slot * heads + head) * 4 + rows32) * Q::PARTIAL) +
                         x * 1024 + lane * 4;
  float4 sum[4] = {};
  for (int32_t i = 0; i < t.end; i += 4) {
    float4 w[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int z = 0; z < 4; ++z)
        if (i + j < t.end) w[j][z] = *reinterpret_cast<const float4*>(p + (i + j) * step + z * 256);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int z = 0; z < 4; ++z)
        if (i + j < t.end) {
          sum[z].x += w[j][z].x; sum[z].y += w[j][z].y; sum[z].z += w[j][z].z; sum[z].w += w[j][z].w;
        }
  }
  uint16_t* const to = keys ? (y ? dv : dk) : dq;
  const int64_t stride = keys ? (y ? a.sdv : a.sdk) : a.sdq;
  Turn<NB>::store(turn, sum, keys && y ? 1.f : a.scale, to + (t.seq0 + (int64_t)first) * stride + head * a.D, stride, t.len - first,
                  a.D);
}

template <int NB>
hipError_t forward(const hpd_finetune_layout* L, const FtArgs& a, const uint16_t* q, const uint16_t* k, const uint16_t* v,
                   uint16_t* out, float* lse, float* partial, hipStream_t s) {
  ft_stream_forward_kernel<NB><<<dim3((unsigned)hpd_ft_query_groups(L)), 256, 0, s>>>(a, L->d_query_items, q, k, v, out, lse, partial);
  if (!L->query_joins.empty())
    ft_stream_join_kernel<NB><<<dim3((unsigned)L->query_joins.size() * a.Hq * 4), 64 * NB, 0, s>>>(a, L->d_query_joins, partial, out,
                                                                                             lse);
  return hipGetLastError();
}

template <int NB>
hipError_t backward(const hpd_finetune_layout* L, FtArgs a, const uint16_t* q, const uint16_t* k, const uint16_t* v,
                    const uint16_t* out, const float* lse, const uint16_t* d_out, uint16_t* dq, uint16_t* dk, uint16_t* dv,
                    float* stat, hipStream_t s) {
  float* const key_partial = stat + 2 * a.N * a.Hq + (-2 * a.N * a.Hq & 3);  // (on 16 bytes)
  float* const query_partial = key_partial + (int64_t)L->slots * a.Hkv * KeyTile<NB>::PARTIAL;
  ft_stream_dq_kernel<NB><<<dim3((unsigned)hpd_ft_query_groups(L)), 256, 0, s>>>(a, L->d_query_items, q, k, v, out, d_out, lse, stat,
                                                                             query_partial, dq);
  ft_stream_dkv_kernel<NB><<<dim3((unsigned)hpd_ft_key_groups(L)), 256, 0, s>>>(a, L->d_items, q, k, v, d_out, stat, key_partial, dk, dv);
  const uint32_t n_key = (uint32_t)L->joins.size() * a.Hkv * 8, n_query = (uint32_t)L->query_joins.size() * a.Hq * 4;
  if (n_key + n_query)
    ft_stream_join_gradients_kernel<NB><<<dim3(n_key + n_query), 64 * NB, 0, s>>>(a, n_key, L->d_joins, L->d_query_joins, key_partial,
                                                                                query_partial, dq, dk, dv);
  return hipGetLastError();
}

}  // namespace

hipError_t hpd_launch_ft_stream_forward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                        void* out, float* lse, void* workspace, hipStream_t s) {
  const auto run = a.D <= 32 ? forward<1> : a.D <= 64 ? forward<2> : a.D <= 96 ? forward<3> : forward<4>;
  return run(L, a, (const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (uint16_t*)out, lse, (float*)workspace, s);
}

hipError_t hpd_launch_ft_stream_backward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                         const void* out, const float* lse, const void* d_out, void* dq, void* dk, void* dv,
                                         void* workspace, hipStream_t s) {
  const auto run = a.D <= 32 ? backward<1> : a.D <= 64 ? backward<2> : a.D <= 96 ? backward<3> : backward<4>;
  return run(L, a, (const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (const uint16_t*)out, lse,
             (const uint16_t*)d_out, (uint16_t*)dq, (uint16_t*)dk, (uint16_t*)dv, (float*)workspace, s);
}
