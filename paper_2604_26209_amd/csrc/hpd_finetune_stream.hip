// Fine-tuning attention in bf16 with head_dim 64 or 128: forward and gradients (formulas and operand
// scheme: hpd_finetune_attn.hip).  The other side's tokens stream through a ring of tiles in LDS that
// global_load_lds fills ahead of their use.
//
// Tiles: 32 rows of D bf16 values as they lie in memory, the 16-byte chunks of a row permuted: chunk c
// of row r lies at c ^ f(r), f(r) = 4 (r % 4) + (r / 4) % 4 for rows of 16 chunks and
// 4 (r / 2 % 2) + (r / 4) % 4 for rows of 8.  So both ways of reading a tile spread over all banks:
// one chunk of 16 successive rows (left operand of a score product), and the same 64 bytes of four
// successive rows (transposing read, left operand of a second product).
#include "hpd_finetune_dev.h"

namespace {

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
constexpr uint32_t BIAS = 4096;  // keeps a lane's offset positive (see Loader)

__device__ __forceinline__ void wait_lds_and_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N>
__device__ __forceinline__ void wait_vector_memory() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int D>
struct Rows {
  static constexpr int RB = D * 2;           // bytes of a row
  static constexpr int TILE = 32 * RB;       // bytes of a tile
  static constexpr int CHUNKS = RB / 16;     // of a row
  static constexpr int STEPS = D / 16;       // products of a score
  static constexpr int BLOCKS = D / 32;      // blocks of 32 channels
  static constexpr int GROUP = 4096 / RB;    // rows that four load instructions bring
  static __device__ __forceinline__ int swizzle(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
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
template <int D>
struct Loader {
  using R = Rows<D>;
  uint32_t off[4];
  int64_t stride;  // bytes between rows
  bool near;       // a group's offsets fit 32 bits
  __device__ __forceinline__ void init(int64_t stride_elements, int lane) {
    stride = stride_elements * 2;
    near = stride < 1 << 25;
#pragma unroll
    for (int f = 0; f < 4; ++f) off[f] = row(f, lane) * (uint32_t)stride + chunk(f, lane) - f * 1024 + BIAS;
  }
  static __device__ __forceinline__ int32_t row(int f, int lane) { return f * (1024 / R::RB) + lane / R::CHUNKS; }
  static __device__ __forceinline__ uint32_t chunk(int f, int lane) {
    return ((lane % R::CHUNKS) ^ R::swizzle(row(f, lane))) << 4;
  }
  // GROUP rows from base (wave-uniform) to lds; rows past `last` (counted from base) are row `last` again
  __device__ __forceinline__ void load(const char* base, uint32_t lds, int32_t last, int lane) const {
    lds = __builtin_amdgcn_readfirstlane(lds);
    uint32_t keep;
    if (near && last >= R::GROUP - 1) {
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
      for (int f = 0; f < 4; ++f) p[f] = base + min(row(f, lane), last) * stride + chunk(f, lane) - f * 1024;
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
__device__ __forceinline__ bf16x8 lds_rows(const char* p) {
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(p));
}
// the same by LDS address
__device__ __forceinline__ bf16x8 lds_read(uint32_t at) {
  return __builtin_bit_cast(bf16x8, *(const __attribute__((address_space(3))) uint4v*)(uintptr_t)at);
}
__device__ __forceinline__ uint2 lds_read_tr(uint32_t at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) hpd::short4v*)(uintptr_t)at));
}
template <int D>
__device__ __forceinline__ bf16x8 lds_columns(const char* tile, uint32_t col, int b, int k) {
  using R = Rows<D>;
  const uint2 lo = hpd::lds_read_tr16(tile + (col ^ (b << 6)) + 16 * k * R::RB);
  const uint2 hi = hpd::lds_read_tr16(tile + (col ^ (b << 6) ^ 32) + (16 * k + 8) * R::RB);
  return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
}
__device__ __forceinline__ floatx16 mfma(bf16x8 a, bf16x8 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// The same, adding up in the accumulation registers, which only these instructions touch between
// the two hold(): the gradient kernels have a wave per SIMD and up to 256 accumulators, and left to
// itself the compiler moves them to and fro.
__device__ __forceinline__ void add_product(bf16x8 a, bf16x8 b, floatx16& c) {
  asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
// In front of the loop and behind it, so that inside they are never anywhere else.
template <int N>
__device__ __forceinline__ void hold(floatx16* c) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+a"(c[i]));
}
// Behind the loop: waits out the last product (8 passes of 4 cycles).
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

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

// 32 columns of a transposed result (lane n: column n) times f, as 32 rows of D values through `turn`
// (TILE bytes of LDS of this wave's own); row r of the tile goes to out + r * stride, r < rows
template <int D>
__device__ __forceinline__ void store_rows(char* turn, const floatx16* acc, float f, uint16_t* out, int64_t stride, int rows,
                                           int lane) {
  using R = Rows<D>;
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
    if (r < rows) *reinterpret_cast<uint4*>(out + r * stride + c * 8) = w;
  }
}

// ---------------------------------------------------------------------------------------
// Forward and dq: four waves of 32 queries of one head; rounds of 64 keys, two rounds in LDS.
// ---------------------------------------------------------------------------------------
template <int D>
struct QueryTile {
  using R = Rows<D>;
  static constexpr int STAGE = 4 * R::TILE;  // 64 rows of k, 64 rows of v
  const FtArgs& a;
  hpd_ft_tile t;
  int lane, n, h, wave;
  int32_t hq, hk, q_first, i, ic, rounds;
  int64_t token;
  bool active;
  int32_t q_min, q_max;  // ranks of the wave's queries
  const int32_t* ranks;
  const const_i32* blk_rank;
  Loader<D> loader;
  const char* src;
  uint32_t ring_lds;

  __device__ __forceinline__ QueryTile(const FtArgs& args, const uint16_t* k, const uint16_t* v, const char* ring) : a(args) {
    lane = threadIdx.x & 63;
    n = lane & 31;
    h = lane >> 5;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroup b runs on XCD b % 8: the query tiles and heads that read the same keys stay together
    const int32_t G = a.Hq / a.Hkv, rest = blockIdx.x / a.Hkv;
    hk = blockIdx.x % a.Hkv;
    hq = hk * G + rest % G;
    t = a.tiles[rest / G];
    q_first = t.row0 + wave * 32;
    i = q_first + n;
    ic = min(i, t.len - 1);
    active = q_first < t.len;
    token = t.seq0 + (int64_t)ic;
    rounds = (min(t.row0 + 128, t.len) + 63) / 64;
    // this wave's part of a round: waves 0 and 1 keys, 2 and 3 values
    loader.init(wave < 2 ? a.sk : a.sv, lane);
    src = reinterpret_cast<const char*>(wave < 2 ? k + t.seq0 * a.sk : v + t.seq0 * a.sv) + (int64_t)hk * D * 2;
    ring_lds = lds_address(ring);
    ranks = a.rank + t.seq0;
    blk_rank = (const const_i32*)(uintptr_t)(a.blk_rank + t.blk0);
    const int32_t own = min(q_first, t.len - 1) / 32;
    q_min = blk_rank[2 * own];
    q_max = blk_rank[2 * own + 1];
  }
  __device__ __forceinline__ void issue(int32_t round) const {
    const uint32_t dst = ring_lds + (round & 1) * STAGE + (wave >> 1) * 2 * R::TILE;
#pragma unroll
    for (int j = 0; j < 32 / R::GROUP; ++j) {
      const int32_t row = D == 128 ? 32 * j + 16 * (wave & 1) : 32 * (wave & 1);
      const int32_t first = min(round * 64 + row, t.len - 1);
      loader.load(src + first * loader.stride, dst + row * R::RB, t.len - 1 - first, lane);
    }
  }
  static __device__ __forceinline__ void own_row(const uint16_t* row, bf16x8* f) {
#pragma unroll
    for (int s = 0; s < R::STEPS; ++s) f[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(row + s * 16));
  }
  // block b of 32 keys has a key that a query of the wave sees / one that a query does not see
  __device__ __forceinline__ bool reaches(int32_t b) const { return active && b * 32 <= q_first && blk_rank[2 * b] <= q_max; }
  __device__ __forceinline__ bool masked(int32_t b) const { return b * 32 >= q_first || blk_rank[2 * b + 1] > q_min; }
  __device__ __forceinline__ void mask(floatx16& s, int32_t b, int32_t rank_i) const {
    BlockRanks rk;
    rk.load(ranks + b * 32);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = b * 32 + tile_row(r, h) <= ic && rk.of(r, h) <= rank_i ? s[r] : -INFINITY;
  }
};

// LDS addresses of a lane's operands in the first tile of a stage
template <int D>
struct Addresses {
  using R = Rows<D>;
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

template <int D>
__global__ void __launch_bounds__(256, 2) ft_stream_forward_kernel(FtArgs a, const uint16_t* __restrict__ q,
                                                                  const uint16_t* __restrict__ k,
                                                                  const uint16_t* __restrict__ v, uint16_t* __restrict__ out,
                                                                  float* __restrict__ lse) {
  using R = Rows<D>;
  using Q = QueryTile<D>;
  __shared__ __attribute__((aligned(2 * Q::STAGE))) char ring[2 * Q::STAGE];
  const Q w(a, k, v, ring);
  w.issue(0);
  bf16x8 qf[R::STEPS];
  Q::own_row(q + w.token * a.sq + w.hq * D + w.h * 8, qf);
  int32_t rank_i[1] = {a.rank[w.token]};
  arrived(qf);
  arrived(rank_i);
  const float c = a.scale * LOG2E;
  Addresses<D> at(w.ring_lds, w.lane);

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
      if (w.masked(b + j)) w.mask(s[j], b + j, rank_i[0]);
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
  for (int32_t round = 0; round < w.rounds; ++round) {
    wait_vector_memory<0>();
    wait_lds_and_barrier();  // the round is in LDS, the other half of the ring is free
    if (round + 1 < w.rounds) w.issue(round + 1);
    if (w.reaches(2 * round) || w.reaches(2 * round + 1)) step(2 * round);
    at.flip(Q::STAGE);
  }
  wait_lds_and_barrier();
  if (!w.active) return;
  l += __shfl_xor(l, 32);
  if (w.h == 0 && w.i < w.t.len) lse[w.hq * a.N + w.token] = (m + __builtin_amdgcn_logf(l)) * LN2;
  store_rows<D>(ring + w.wave * R::TILE, acc, 1.f / l, out + ((w.t.seq0 + (int64_t)w.q_first) * a.Hq + w.hq) * D,
                (int64_t)a.Hq * D, w.t.len - w.q_first, w.lane);
}

// stat, which this kernel makes and the dk/dv kernel reads: per (head, token) -lse * sqrt(D), where its row's score
// products start, then -delta, delta_i = do_i . o_i, where its row's products with v start:
// p = exp((q . k - lse sqrt(D)) / sqrt(D)).
template <int D>
__global__ void __launch_bounds__(256, 2) ft_stream_dq_kernel(FtArgs a, const uint16_t* __restrict__ q,
                                                             const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                             const uint16_t* __restrict__ out, const uint16_t* __restrict__ d_out,
                                                             const float* __restrict__ lse, float* __restrict__ stat,
                                                             uint16_t* __restrict__ dq) {
  using R = Rows<D>;
  using Q = QueryTile<D>;
  __shared__ __attribute__((aligned(2 * Q::STAGE))) char ring[2 * Q::STAGE];
  const Q w(a, k, v, ring);
  w.issue(0);
  bf16x8 qf[R::STEPS], of[R::STEPS];
  float nl[1], nd[1];
  {
    bf16x8 o[R::STEPS];
    const int64_t row = (w.token * a.Hq + w.hq) * D + w.h * 8;
    Q::own_row(q + w.token * a.sq + w.hq * D + w.h * 8, qf);
    Q::own_row(d_out + row, of);
    Q::own_row(out + row, o);
    const float minus_lse = -lse[w.hq * a.N + w.token];
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
    if (w.h == 0 && w.i < w.t.len) {
      stat[w.hq * a.N + w.token] = minus_lse / a.scale;
      stat[(a.Hq + w.hq) * a.N + w.token] = nd[0];
    }
  }
  int32_t rank_i[1] = {a.rank[w.token]};
  arrived(qf);
  arrived(of);
  arrived(nl);
  arrived(nd);
  arrived(rank_i);
  const float c = a.scale * LOG2E;
  Addresses<D> at(w.ring_lds, w.lane);
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
      if (i == 2 * S - 1 && w.masked(b)) w.mask(s[0], b, rank_i[0]);
      if (i >= 2 * S) {  // (a step behind: the last product is on its way)
        const int y = i - 2 * S;
        gradient(0, 16 * (y > 0 ? y - 1 : 0) / (2 * S - 1), 16 * y / (2 * S - 1));
        if (y == S) df[0][0] = pack8(e[0]);
        if (y == 2 * S - 1) df[0][1] = pack8(e[0] + 8);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (w.masked(b + 1)) w.mask(s[1], b + 1, rank_i[0]);
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
  for (int32_t round = 0; round < w.rounds; ++round) {
    wait_vector_memory<0>();
    wait_lds_and_barrier();
    if (round + 1 < w.rounds) w.issue(round + 1);
    if (w.reaches(2 * round) || w.reaches(2 * round + 1)) step(2 * round);
    at.flip(Q::STAGE);
  }
  wait_lds_and_barrier();
  if (!w.active) return;
  store_rows<D>(ring + w.wave * R::TILE, acc, a.scale, dq + (w.t.seq0 + (int64_t)w.q_first) * a.sdq + w.hq * D, a.sdq,
                w.t.len - w.q_first, w.lane);
}

// dk and dv: two waves of 64 keys of one kv head, over the queries of all its heads; rounds of 32 queries.
template <int D>
__global__ void __launch_bounds__(128, 1) ft_stream_dkv_kernel(FtArgs a, const uint16_t* __restrict__ q,
                                                              const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                              const uint16_t* __restrict__ d_out,
                                                              const float* __restrict__ stat, uint16_t* __restrict__ dk,
                                                              uint16_t* __restrict__ dv) {
  using R = Rows<D>;
  constexpr int STAGE = 2 * R::TILE + 512, SLOTS = 4, LOADS = R::TILE / 1024 + 1;  // rows of q and do; each wave's own -lse, -delta
  __shared__ __attribute__((aligned(1024))) char ring[SLOTS * STAGE];
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t G = a.Hq / a.Hkv, hk = blockIdx.x % a.Hkv;
  const hpd_ft_tile t = a.tiles[blockIdx.x / a.Hkv];
  const int32_t k_first = t.row0 + wave * 64;
  const bool active = k_first < t.len;

  Loader<D> loader;
  loader.init(wave == 0 ? a.sq : (int64_t)a.Hq * D, lane);
  const char* const src = reinterpret_cast<const char*>(wave == 0 ? q + t.seq0 * a.sq : d_out + (int64_t)t.seq0 * a.Hq * D);
  const uint32_t ring_lds = lds_address(ring);
  const int32_t b_first = t.row0 / 32, per_head = (t.len + 31) / 32 - b_first, rounds = G * per_head;
  int32_t next_g = 0, next_b = b_first;  // the round that is requested next
  auto issue = [&](int32_t round) {
    const uint32_t slot = ring_lds + (round & (SLOTS - 1)) * STAGE;
    const int32_t hq = hk * G + next_g;
#pragma unroll
    for (int j = 0; j < 32 / R::GROUP; ++j) {
      const int32_t first = min(next_b * 32 + j * R::GROUP, t.len - 1);
      loader.load(src + first * loader.stride + hq * D * 2, slot + wave * R::TILE + j * R::GROUP * R::RB,
                  t.len - 1 - first, lane);
    }
    const float* p = stat + (h * (int64_t)a.Hq + hq) * a.N + t.seq0 + min(next_b * 32 + n, t.len - 1);
    const uint32_t dst = __builtin_amdgcn_readfirstlane(slot + 2 * R::TILE + wave * 256);
    uint32_t keep;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
        "global_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
        : "=&s"(keep)
        : "v"(p), "s"(dst)
        : "memory");
    if (++next_b == b_first + per_head) {
      next_b = b_first;
      ++next_g;
    }
  };
  issue(0);
  if (rounds > 1) issue(1);
  if (rounds > 2) issue(2);
  bf16x8 kf[2][R::STEPS], vf[2][R::STEPS];
  int32_t j[2], rank_j[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    j[x] = k_first + 32 * x + n;
    const int64_t token = t.seq0 + (int64_t)min(j[x], t.len - 1);
    const uint16_t* krow = k + token * a.sk + hk * D + h * 8;
    const uint16_t* vrow = v + token * a.sv + hk * D + h * 8;
#pragma unroll
    for (int s = 0; s < R::STEPS; ++s) {
      kf[x][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(krow + s * 16));
      vf[x][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(vrow + s * 16));
    }
    rank_j[x] = a.rank[token];
  }
  arrived(kf[0]);
  arrived(kf[1]);
  arrived(vf[0]);
  arrived(vf[1]);
  arrived(rank_j);
  const int32_t* const ranks = a.rank + t.seq0;
  const const_i32* const blk_rank = (const const_i32*)(uintptr_t)(a.blk_rank + t.blk0);
  const int32_t b0 = min(k_first, t.len - 1) / 32, b1 = min(k_first + 32, t.len - 1) / 32;
  const int32_t k_min = min(blk_rank[2 * b0], blk_rank[2 * b1]), k_max = max(blk_rank[2 * b0 + 1], blk_rank[2 * b1 + 1]);
  const float c = a.scale * LOG2E;
  const uint32_t row_at = R::row_offset(n, h), col_at = R::column_offset(lane);

  floatx16 acc_k[2][R::BLOCKS], acc_v[2][R::BLOCKS];
  zero(acc_k[0], R::BLOCKS);
  zero(acc_k[1], R::BLOCKS);
  zero(acc_v[0], R::BLOCKS);
  zero(acc_v[1], R::BLOCKS);
  hold<R::BLOCKS>(acc_k[0]);
  hold<R::BLOCKS>(acc_k[1]);
  hold<R::BLOCKS>(acc_v[0]);
  hold<R::BLOCKS>(acc_v[1]);
  // The scores of the two columns one after the other (both at once do not fit the registers), each
  // while the other's exponentials run.
  auto block = [&](const char* tq, const char* to, const char* st, int32_t b, bool masked) __attribute__((always_inline)) {
    uint32_t rows = row_at, cols = col_at;
    asm volatile("" : "+v"(rows), "+v"(cols));  // (the addresses made from them are not kept for the next round: they are 16 registers)
    constexpr int S = R::STEPS, C = 2 * R::BLOCKS;  // operands: rows of q, do, q, do (S each), columns of do and q (C each)
    auto ld = [&](int i) __attribute__((always_inline)) -> bf16x8 {
      if (i < 4 * S) return lds_rows(((i / S) & 1 ? to : tq) + (rows ^ ((i % S) << 5)));
      i -= 4 * S;
      return lds_columns<D>(i < C ? to : tq, cols, i % C / 2, i % 2);
    };
    auto stats = [&](const char* p) __attribute__((always_inline)) {  // one number per row of the tile, as a result's registers lie
      floatx16 v;
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const float4 w = *reinterpret_cast<const float4*>(p + (8 * z + 4 * h) * 4);
        v[4 * z] = w.x; v[4 * z + 1] = w.y; v[4 * z + 2] = w.z; v[4 * z + 3] = w.w;
      }
      return v;
    };
    // where a score starts: hidden ones at -infinity, where they stay (weight 0)
    auto start = [&](int x) __attribute__((always_inline)) {
      floatx16 v = stats(st);
      if (masked) {
        BlockRanks rk;
        rk.load(ranks + b * 32);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int32_t i = b * 32 + tile_row(r, h);
          v[r] = i < t.len && i >= j[x] && rank_j[x] <= rk.of(r, h) ? v[r] : -INFINITY;
        }
      }
      return v;
    };
    bf16x8 f[3], pf[2][2], df[2][2];
    floatx16 s, dp;
    auto weight = [&](int r) __attribute__((always_inline)) { s[r] = fast_exp2(s[r] * c); };
    auto pack_half = [&](int x, int z) __attribute__((always_inline)) {
      float p[8], e[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        p[r] = s[8 * z + r];
        e[r] = p[r] * dp[8 * z + r];
      }
      pf[x][z] = pack8(p);
      df[x][z] = pack8(e);
    };
    f[0] = ld(0);
    f[1] = ld(1);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      floatx16 next = start(x);
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const int at = 2 * x * S + i;
        f[(at + 2) % 3] = ld(at + 2);
        next = mfma(f[at % 3], kf[x][i], next);
        if (x == 1 && i == S / 2 - 1) pack_half(0, 0);
        if (x == 1 && i == S - 1) pack_half(0, 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      s = next;
      dp = stats(st + 128);
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const int at = (2 * x + 1) * S + i;
        f[(at + 2) % 3] = ld(at + 2);
        dp = mfma(f[at % 3], vf[x][i], dp);
#pragma unroll
        for (int r = 16 * (i - 1) / (S - 1); i > 0 && r < 16 * i / (S - 1); ++r) weight(r);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    pack_half(1, 0);
    pack_half(1, 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
      const int at = 4 * S + i;
      if (i + 2 < 2 * C) f[(at + 2) % 3] = ld(at + 2);
      if (i < C) {
        add_product(f[at % 3], pf[0][i % 2], acc_v[0][i / 2]);
        add_product(f[at % 3], pf[1][i % 2], acc_v[1][i / 2]);
      } else {
        add_product(f[at % 3], df[0][i % 2], acc_k[0][(i - C) / 2]);
        add_product(f[at % 3], df[1][i % 2], acc_k[1][(i - C) / 2]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int32_t b = b_first;
  for (int32_t round = 0; round < rounds; ++round) {
    const int32_t ahead = rounds - 1 - round;
    if (ahead >= 2) wait_vector_memory<2 * LOADS>();
    else if (ahead == 1) wait_vector_memory<LOADS>();
    else wait_vector_memory<0>();
    wait_lds_and_barrier();
    if (round + 3 < rounds) issue(round + 3);
    const int32_t q_min = blk_rank[2 * b], q_max = blk_rank[2 * b + 1];
    const char* const slot = ring + (round & (SLOTS - 1)) * STAGE;
    const char* const st = slot + 2 * R::TILE + wave * 256;
    if (active && b * 32 + 31 >= k_first && k_min <= q_max)
      block(slot, slot + R::TILE, st, b, b * 32 < k_first + 63 || k_max > q_min || (b + 1) * 32 > t.len);
    if (++b == b_first + per_head) b = b_first;
  }
  settle();
  hold<R::BLOCKS>(acc_k[0]);
  hold<R::BLOCKS>(acc_k[1]);
  hold<R::BLOCKS>(acc_v[0]);
  hold<R::BLOCKS>(acc_v[1]);
  wait_lds_and_barrier();
  if (!active) return;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int64_t token = t.seq0 + (int64_t)k_first + 32 * x;
    const int rows = t.len - k_first - 32 * x;
    store_rows<D>(ring + wave * R::TILE, acc_v[x], 1.f, dv + token * a.sdv + hk * D, a.sdv, rows, lane);
    store_rows<D>(ring + wave * R::TILE, acc_k[x], a.scale, dk + token * a.sdk + hk * D, a.sdk, rows, lane);
  }
}

template <int D>
hipError_t forward(const hpd_finetune_layout* L, const FtArgs& a, const void* q, const void* k, const void* v, void* out,
                   float* lse, hipStream_t s) {
  ft_stream_forward_kernel<D><<<dim3((unsigned)L->tiles.size() * a.Hq), 256, 0, s>>>(
      a, (const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (uint16_t*)out, lse);
  return hipGetLastError();
}

template <int D>
hipError_t backward(const hpd_finetune_layout* L, FtArgs a, const uint16_t* q, const uint16_t* k, const uint16_t* v,
                    const uint16_t* out, const float* lse, const uint16_t* d_out, uint16_t* dq, uint16_t* dk, uint16_t* dv,
                    float* stat, hipStream_t s) {
  const unsigned tiles = (unsigned)L->tiles.size();
  ft_stream_dq_kernel<D><<<dim3(tiles * a.Hq), 256, 0, s>>>(a, q, k, v, out, d_out, lse, stat, dq);
  a.tiles = L->d_key_tiles;
  ft_stream_dkv_kernel<D><<<dim3(tiles * a.Hkv), 128, 0, s>>>(a, q, k, v, d_out, stat, dk, dv);
  return hipGetLastError();
}

}  // namespace

bool hpd_ft_stream_supported(const hpd_finetune_layout* L) {
  return L->cfg.dtype == HPD_BF16 && (L->cfg.head_dim == 64 || L->cfg.head_dim == 128);
}

hipError_t hpd_launch_ft_stream_forward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                        void* out, float* lse, hipStream_t s) {
  return a.D == 64 ? forward<64>(L, a, q, k, v, out, lse, s) : forward<128>(L, a, q, k, v, out, lse, s);
}

hipError_t hpd_launch_ft_stream_backward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                         const void* out, const float* lse, const void* d_out, void* dq, void* dk, void* dv,
                                         void* workspace, hipStream_t s) {
  const auto run = a.D == 64 ? backward<64> : backward<128>;
  return run(L, a, (const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (const uint16_t*)out, lse,
             (const uint16_t*)d_out, (uint16_t*)dq, (uint16_t*)dk, (uint16_t*)dv, (float*)workspace, s);
}
