// Fine-tuning attention in fp32: forward and gradients (formulas and operand scheme: hpd_finetune_attn.hip).
//
// The matrix instruction (32 x 32 x 2, 64 cycles) is what bounds these kernels: the chain of products of one wave
// is long before the GPU is full.  So the four waves of a workgroup share 32 tokens and take every fourth block of
// the other side, each through tiles of its own in LDS, without barriers; their sums meet at the end.  The forward kernel has one tile
// per wave, keys and values by turns, so that two workgroups run on a CU (three for 64 channels) and one's loads
// are behind the other's products: 1.3 to 1.5 times as fast as with a tile of each kind and one workgroup.  So has dq from 96 channels
// on, for 128 with the gradients of the output in LDS as well (up to 1.3 times the gradients' speed).  dq of 64 channels and dk/dv, whose
// sums leave no room for a second workgroup of 96 or 128 channels, have two: a tile is loaded again (global_load_lds) as soon as its
// last product has read it, and the order of the products leaves one of them between that and the tile's next use.
// 16 x 307 tokens, 4 heads of 64: forward 24 us, gradients 76 us, matrix units busy 23 to 30 %: three rounds
// of a wave and the latencies of a start; 5 x 2500 tokens, 32/8 heads of 128: forward 2.2 ms, 104 of 153 TFLOP/s.
//
// Tiles: 32 rows of 64 or 128 values, of which the first DP count (64, 96 or 128).  Chunk c (16 bytes) of row r lies at c ^ f(r),
// f(r) = 8 (r / 4 % 2) + 4 (r / 8 % 2) + r % 4: sixteen rows' chunk c in different banks (left operand of four score products),
// and 32 channels of the rows r and r + 4 too (left operand of a second product).
#include "hpd_finetune_dev.h"

namespace {

__device__ __forceinline__ floatx16 mfma(float a, float b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

template <int DP>
struct Tile {
  static constexpr int RB = DP <= 64 ? 256 : 512, BYTES = 32 * RB, CHUNKS = RB / 16, STEPS = DP / 8, NB = DP / 32;
  static constexpr int LOADS = BYTES / 1024;  // load instructions
  static __device__ __forceinline__ int swizzle(int r) { return ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3); }

  // Rows first .. first + 31 of a sequence's head; src: its row 0, last: its last row, which stands for those behind it.  The
  // lanes' offsets in whole tiles are kept: 0.92 of the time with the address of every row made anew, in the mean of 36 random batches,
  // down to 0.84.
  struct Source {
    static constexpr int SETS = RB / 256;  // the chunks of odd groups of 8 rows differ
    static constexpr uint32_t BIAS = 4096;
    const char* src;
    int64_t stride;  // bytes
    uint32_t off[SETS][4];
    int32_t D, last;
    bool near;  // a group's offsets fit 32 bits
    static __device__ __forceinline__ int32_t row(int g, int f, int lane) { return (4 * g + f) * (1024 / RB) + lane / CHUNKS; }
    static __device__ __forceinline__ int32_t chunk(int g, int f, int lane) { return (lane % CHUNKS) ^ swizzle(row(g, f, lane)); }
    __device__ __forceinline__ void init(const float* x, int64_t elements, int32_t len, int32_t D_, int lane) {
      src = reinterpret_cast<const char*>(x);
      stride = elements * 4;
      D = D_;
      last = len - 1;
      near = elements < 1 << 24;
#pragma unroll
      for (int g = 0; g < SETS; ++g)
#pragma unroll
        for (int f = 0; f < 4; ++f) {  // (behind the row's end: its first chunk, the other side's operand is zero there)
          const int32_t c = chunk(g, f, lane);
          off[g][f] = row(0, f, lane) * (uint32_t)stride + (c * 4 < D ? c << 4 : 0) - f * 1024 + BIAS;
        }
    }
    // shift: bytes from src to the head; zeros: 16 bytes of them for the chunks behind the row's end
    __device__ __forceinline__ void load(uint32_t lds, int32_t first, int lane, int64_t shift = 0, const void* zeros = nullptr) const {
      const char* const head = src + shift;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the tile's last reads)
      const bool whole = !zeros && near && first + 31 <= last;
#pragma unroll
      for (int g = 0; g < LOADS / 4; ++g) {
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds + g * 4096);
        uint32_t keep;  // M0 is the compiler's
        if (whole) {
          const uint32_t* o = off[g % SETS];
          asm volatile(
              "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\t"
              "global_load_lds_dwordx4 %1, %6\n\t"
              "global_load_lds_dwordx4 %2, %6 offset:1024\n\t"
              "global_load_lds_dwordx4 %3, %6 offset:2048\n\t"
              "global_load_lds_dwordx4 %4, %6 offset:3072\n\t"
              "s_mov_b32 m0, %0"
              : "=&s"(keep)
              : "v"(o[0]), "v"(o[1]), "v"(o[2]), "v"(o[3]), "s"(dst),
                "s"(uniform(head + (first + g * (4096 / RB)) * stride) - BIAS)
              : "memory");
          continue;
        }
        const char* p[4];
        int32_t here = lane;
        asm volatile("" : "+v"(here));  // (nothing of this is kept from tile to tile)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const int32_t c = chunk(g, f, here);
          p[f] = c * 4 < D || !zeros ? head + min(first + row(g, f, here), last) * stride + (c * 4 < D ? c << 4 : 0)
                                     : reinterpret_cast<const char*>(zeros);
          p[f] -= f * 1024;  // (the instruction's offset moves both addresses)
        }
        asm volatile(
            "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\t"
            "global_load_lds_dwordx4 %1, off\n\t"
            "global_load_lds_dwordx4 %2, off offset:1024\n\t"
            "global_load_lds_dwordx4 %3, off offset:2048\n\t"
            "global_load_lds_dwordx4 %4, off offset:3072\n\t"
            "s_mov_b32 m0, %0"
            : "=&s"(keep)
            : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "s"(dst)
            : "memory");
      }
    }
  };
  struct Own { float4 f[STEPS]; };  // chunk 2 s + h of the lane's row
  static __device__ __forceinline__ void load(Own& x, const float* row, int h, int32_t D) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = (2 * s + h) * 4;
      x.f[s] = *reinterpret_cast<const float4*>(row + (c < D ? c : 0));
      if (c >= D) x.f[s] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  // tile rows x own rows; at: row_offset
  static __device__ __forceinline__ uint32_t row_offset(int n, int h) { return n * RB + ((h ^ swizzle(n)) << 4); }
  static __device__ __forceinline__ floatx16 scores(uint32_t tile, uint32_t at, const Own& b, floatx16 s) {
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      const float4 a = __builtin_bit_cast(float4, *(const __attribute__((address_space(3))) uint4v*)(uintptr_t)(tile + (at ^ (x << 5))));
      s = mfma(a.x, b.f[x].x, s);
      s = mfma(a.y, b.f[x].y, s);
      s = mfma(a.z, b.f[x].z, s);
      s = mfma(a.w, b.f[x].w, s);
    }
    return s;
  }
  // the same, own rows in a tile too
  static __device__ __forceinline__ floatx16 scores(uint32_t tile, uint32_t at, uint32_t own, floatx16 s) {
#pragma unroll
    for (int x = 0; x < STEPS; ++x) {
      const float4 a = __builtin_bit_cast(float4, *(const __attribute__((address_space(3))) uint4v*)(uintptr_t)(tile + (at ^ (x << 5))));
      const float4 b = __builtin_bit_cast(float4, *(const __attribute__((address_space(3))) uint4v*)(uintptr_t)(own + (at ^ (x << 5))));
      s = mfma(a.x, b.x, s);
      s = mfma(a.y, b.y, s);
      s = mfma(a.z, b.z, s);
      s = mfma(a.w, b.w, s);
    }
    return s;
  }
  // (columns of the tile)^T x p
  static __device__ __forceinline__ void add(uint32_t tile, int n, int h, const float* p, floatx16* acc) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = tile_row(r, h);  // swizzle: 8 h + (4 (row / 8 % 2) + row % 4), the latter of r alone
      const uint32_t at = tile + row * RB + (((n >> 2) ^ (h << 3) ^ (((r >> 2) & 1) << 2 | (r & 3))) << 4) + (n & 3) * 4;
#pragma unroll
      for (int b = 0; b < NB; ++b)
        acc[b] = mfma(*(const __attribute__((address_space(3))) float*)(uintptr_t)(at ^ (b << 7)), p[r], acc[b]);
    }
  }
};

template <int N>
__device__ __forceinline__ void own_arrived(float4 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i].x), "+v"(f[i].y), "+v"(f[i].z), "+v"(f[i].w));
}

// 32 tokens of a sequence: block s of a work tile
struct Block {
  hpd_ft_tile t;
  int lane, n, h, wave;
  int32_t first, i, ic;  // first token, the lane's, and the last one instead of what lies behind it
  __device__ __forceinline__ Block(const hpd_ft_tile& tile, int32_t s) : t(tile) {
    lane = threadIdx.x & 63;
    n = lane & 31;
    h = lane >> 5;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    first = t.row0 + s * 32;
    i = first + n;
    ic = min(i, t.len - 1);
  }
};

// One or two tiles of every wave and OWN of the workgroup; at the end the waves' sums, row by row
template <int DP, int TILES, int OWN = 0>
union Shared {
  struct {
    float sums[4][32][DP + 4];
    float m[4][32], l[4][32];
  } end;
  char tiles[4 * TILES + OWN][Tile<DP>::BYTES];
};
template <int DP, int TILES, int OWN>
__device__ __forceinline__ void put(Shared<DP, TILES, OWN>& sh, const Block& w, const floatx16* acc, float f) {
#pragma unroll
  for (int b = 0; b < DP / 32; ++b)
#pragma unroll
    for (int a = 0; a < 4; ++a)
      *reinterpret_cast<float4*>(&sh.end.sums[w.wave][w.n][32 * b + 8 * a + 4 * w.h]) =
          make_float4(acc[b][4 * a] * f, acc[b][4 * a + 1] * f, acc[b][4 * a + 2] * f, acc[b][4 * a + 3] * f);
}
// the sum of the waves' rows r to out + r * stride
template <int DP, int TILES, int OWN>
__device__ __forceinline__ void join(const Shared<DP, TILES, OWN>& sh, const Block& w, float* out, int64_t stride, int32_t D) {
  for (int x = threadIdx.x; x < 32 * DP / 4; x += 256) {
    const int r = x / (DP / 4), c = x % (DP / 4) * 4;
    if (w.first + r >= w.t.len || c >= D) continue;
    float4 s = *reinterpret_cast<const float4*>(&sh.end.sums[0][r][c]);
#pragma unroll
    for (int y = 1; y < 4; ++y) {
      const float4 z = *reinterpret_cast<const float4*>(&sh.end.sums[y][r][c]);
      s.x += z.x; s.y += z.y; s.z += z.z; s.w += z.w;
    }
    *reinterpret_cast<float4*>(out + r * stride + c) = s;
  }
}

// What the forward and the dq kernel share: 32 queries of a head and the blocks of keys that they see
template <int DP, int TILES>
struct Queries : Block {
  using TL = Tile<DP>;
  const FtArgs& a;
  int32_t hq, hk, own, q_min, q_max;
  const int32_t* ranks;
  const const_i32* blk_rank;
  typename TL::Source keys, values;
  uint32_t key_tile, value_tile;  // (one tile: keys and values by turns)
  int64_t token;
  __device__ __forceinline__ Queries(const FtArgs& args, const float* k, const float* v, const char* tiles)
      : Block(args.tiles[blockIdx.x / args.Hq / 4], blockIdx.x / args.Hq % 4), a(args) {
    const int32_t G = a.Hq / a.Hkv, x = blockIdx.x % a.Hq;
    hk = x % a.Hkv;
    hq = hk * G + x / a.Hkv;
    token = t.seq0 + (int64_t)ic;
    keys.init(k + t.seq0 * a.sk + (int64_t)hk * a.D, a.sk, t.len, a.D, lane);
    values.init(v + t.seq0 * a.sv + (int64_t)hk * a.D, a.sv, t.len, a.D, lane);
    ranks = a.rank + t.seq0;
    blk_rank = (const const_i32*)(uintptr_t)(a.blk_rank + t.blk0);
    own = min(first, t.len - 1) / 32;
    q_min = blk_rank[2 * own];
    q_max = blk_rank[2 * own + 1];
    key_tile = lds_address(tiles) + wave * TILES * TL::BYTES;
    value_tile = key_tile + (TILES - 1) * TL::BYTES;
  }
  // the wave's first block from b on that a query sees; past `own`: none
  __device__ __forceinline__ int32_t next(int32_t b) const {
    while (b <= own && blk_rank[2 * b] > q_max) b += 4;
    return b;
  }
  __device__ __forceinline__ void load_keys(int32_t b) const { keys.load(key_tile, b * 32, lane); }
  __device__ __forceinline__ void load_values(int32_t b) const { values.load(value_tile, b * 32, lane); }
  __device__ __forceinline__ void mask(floatx16& s, int32_t b, int32_t rank_i) const {
    if (b < own && blk_rank[2 * b + 1] <= q_min) return;
    BlockRanks rk;
    rk.load(ranks + b * 32);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = b * 32 + tile_row(r, h) <= ic && rk.of(r, h) <= rank_i ? s[r] : -INFINITY;
  }
};

template <int DP>
__global__ void __launch_bounds__(256, DP > 64 ? 2 : 3) ft_f32_forward_kernel(FtArgs a, const float* __restrict__ q,
                                                                            const float* __restrict__ k,
                                                                            const float* __restrict__ v, float* __restrict__ out,
                                                                            float* __restrict__ lse) {
  using TL = Tile<DP>;
  constexpr int TILES = 1;
  __shared__ __attribute__((aligned(1024))) Shared<DP, TILES> sh;
  const Queries<DP, TILES> w(a, k, v, &sh.tiles[0][0]);
  if (w.first >= w.t.len) return;
  int32_t b = w.next(w.wave);
  if (b <= w.own) w.load_keys(b);
  typename TL::Own qf;
  TL::load(qf, q + w.token * a.sq + (int64_t)w.hq * a.D, w.h, a.D);
  int32_t rank_i[1] = {w.ranks[w.ic]};
  own_arrived(qf.f);
  arrived(rank_i);
  const float c = a.scale * LOG2E;
  const uint32_t at = TL::row_offset(w.n, w.h);
  floatx16 acc[TL::NB];
  zero(acc, TL::NB);
  float m = NEG_BIG, l = 0.f;  // maximum (log2 units), this lane's share of the sum
  while (b <= w.own) {
    const int32_t after = w.next(b + 4);
    wait_vector_memory<0>();
    floatx16 s = TL::scores(w.key_tile, at, qf, floatx16{});
    w.load_values(b);
    w.mask(s, b, rank_i[0]);
    float p[16], top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    top = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)) * c);
    const float alpha = fast_exp2(m - top);
    m = top;
    l *= alpha;
#pragma unroll
    for (int x = 0; x < TL::NB; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][r] *= alpha;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = fast_exp2(fmaf(s[r], c, -m));
      l += p[r];
    }
    wait_vector_memory<0>();
    TL::add(w.value_tile, w.n, w.h, p, acc);
    if (after <= w.own) w.load_keys(after);
    b = after;
  }
  __syncthreads();
  l += __shfl_xor(l, 32);
  if (w.h == 0) {
    sh.end.m[w.wave][w.n] = m;
    sh.end.l[w.wave][w.n] = l;
  }
  __syncthreads();
  const float top = fmaxf(fmaxf(sh.end.m[0][w.n], sh.end.m[1][w.n]), fmaxf(sh.end.m[2][w.n], sh.end.m[3][w.n]));
  float total = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) total = fmaf(sh.end.l[x][w.n], fast_exp2(sh.end.m[x][w.n] - top), total);
  put(sh, w, acc, fast_exp2(m - top) / total);
  if (w.wave == 0 && w.h == 0 && w.i < w.t.len) lse[w.hq * a.N + w.token] = (top + __builtin_amdgcn_logf(total)) * LN2;
  __syncthreads();
  join(sh, w, out + ((w.t.seq0 + (int64_t)w.first) * a.Hq + w.hq) * a.D, (int64_t)a.Hq * a.D, a.D);
}

// delta_i = do_i . o_i: 16 lanes a row
__global__ void __launch_bounds__(256) ft_f32_delta_kernel(int64_t N, int32_t Hq, int32_t D, const float* __restrict__ out,
                                                         const float* __restrict__ d_out, float* __restrict__ delta) {
  const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
  if (row >= N * Hq) return;
  float s = 0.f;
  for (int32_t c = (threadIdx.x % 16) * 4; c < D; c += 64) {
    const float4 x = *reinterpret_cast<const float4*>(out + row * D + c), y = *reinterpret_cast<const float4*>(d_out + row * D + c);
    s = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s))));
  }
#pragma unroll
  for (int d = 8; d; d >>= 1) s += __shfl_xor(s, d);
  if (threadIdx.x % 16 == 0) delta[(row % Hq) * N + row / Hq] = s;
}

// Products in the order do . v, q . k, ds . k: with two tiles the next values are on their way during the last two, the next
// keys during the first.
template <int DP>
__global__ void __launch_bounds__(256, 2) ft_f32_dq_kernel(FtArgs a, const float* __restrict__ q,
                                                                       const float* __restrict__ k, const float* __restrict__ v,
                                                                       const float* __restrict__ d_out,
                                                                       const float* __restrict__ lse,
                                                                       const float* __restrict__ delta, float* __restrict__ dq) {
  using TL = Tile<DP>;
  constexpr int TILES = DP >= 96 ? 1 : 2, OWN = DP > 96 ? 1 : 0;  // (what two workgroups per CU have room for)
  __shared__ __attribute__((aligned(1024))) Shared<DP, TILES, OWN> sh;
  const Queries<DP, TILES> w(a, k, v, &sh.tiles[0][0]);
  if (w.first >= w.t.len) return;
  int32_t b = w.next(w.wave);
  if (b <= w.own) {
    w.load_values(b);
    if (TILES == 2) w.load_keys(b);
  }
  typename TL::Own qf, of;
  const uint32_t own = lds_address(&sh.tiles[4 * TILES + OWN - 1][0]);
  TL::load(qf, q + w.token * a.sq + (int64_t)w.hq * a.D, w.h, a.D);
  if (OWN) {
    if (w.wave == 0) {
      typename TL::Source rows;
      rows.init(d_out + (w.t.seq0 * (int64_t)a.Hq + w.hq) * a.D, (int64_t)a.Hq * a.D, w.t.len, a.D, w.lane);
      rows.load(own, w.first, w.lane, 0, a.D < DP ? a.rank + a.N : nullptr);
      wait_vector_memory<0>();
    }
    __syncthreads();
  } else {
    TL::load(of, d_out + (w.token * a.Hq + w.hq) * a.D, w.h, a.D);
  }
  float row[2] = {lse[w.hq * a.N + w.token], delta[w.hq * a.N + w.token]};
  int32_t rank_i[1] = {w.ranks[w.ic]};
  own_arrived(qf.f);
  if (!OWN) own_arrived(of.f);
  arrived(row);
  arrived(rank_i);
  const float c = a.scale * LOG2E, lse2 = row[0] * LOG2E;
  const uint32_t at = TL::row_offset(w.n, w.h);
  floatx16 acc[TL::NB];
  zero(acc, TL::NB);
  while (b <= w.own) {
    const int32_t after = w.next(b + 4);
    if (TILES == 2) wait_vector_memory<TL::LOADS>();  // the values; the keys were requested behind them
    else wait_vector_memory<0>();
    const floatx16 dp = OWN ? TL::scores(w.value_tile, at, own, floatx16{}) : TL::scores(w.value_tile, at, of, floatx16{});
    if (TILES == 1) w.load_keys(b);
    if (TILES == 2 && after <= w.own) {
      w.load_values(after);
      wait_vector_memory<TL::LOADS>();
    } else {
      wait_vector_memory<0>();
    }
    floatx16 s = TL::scores(w.key_tile, at, qf, floatx16{});
    w.mask(s, b, rank_i[0]);
    float ds[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) ds[r] = fast_exp2(fmaf(s[r], c, -lse2)) * (dp[r] - row[1]);
    TL::add(w.key_tile, w.n, w.h, ds, acc);
    if (after <= w.own) {
      if (TILES == 1) w.load_values(after);
      else w.load_keys(after);
    }
    b = after;
  }
  __syncthreads();
  put(sh, w, acc, a.scale);
  __syncthreads();
  join(sh, w, dq + (w.t.seq0 + (int64_t)w.first) * a.sdq + (int64_t)w.hq * a.D, a.sdq, a.D);
}

// Products in the order q . k, do . v, ds . q, p . do: the next queries are on their way during the last, the next
// gradients of the output during the first.  An item is a run of the (head, block of queries) of 32 keys, head by head; the
// sums of keys with several items go to `partial`, and a second kernel adds them up.
template <int DP>
__global__ void __launch_bounds__(256, DP > 64 ? 1 : 2) ft_f32_dkv_kernel(FtArgs a, const hpd_ft_item* __restrict__ items,
                                                                        const float* __restrict__ q,
                                                                        const float* __restrict__ k, const float* __restrict__ v,
                                                                        const float* __restrict__ d_out,
                                                                        const float* __restrict__ lse,
                                                                        const float* __restrict__ delta, float* __restrict__ partial,
                                                                        float* __restrict__ dk,
                                                                        float* __restrict__ dv) {
  using TL = Tile<DP>;
  __shared__ __attribute__((aligned(1024))) Shared<DP, 2> sh;
  __shared__ __attribute__((aligned(256))) float stats[4][64];  // of every wave: lse, then delta of its 32 queries
  // the block's values, for 128 channels: the registers are full
  constexpr bool LDS_VALUES = DP > 64;
  __shared__ __attribute__((aligned(1024))) char values[LDS_VALUES ? TL::BYTES : 16];
  const int32_t G = a.Hq / a.Hkv, hk = blockIdx.x % a.Hkv;
  const hpd_ft_item item = items[blockIdx.x / a.Hkv];
  const Block w({item.seq0, item.len, item.row0, item.blk0}, 0);
  const int32_t* const ranks = a.rank + w.t.seq0;
  const const_i32* const blk_rank = (const const_i32*)(uintptr_t)(a.blk_rank + w.t.blk0);
  const int64_t token = w.t.seq0 + (int64_t)w.ic, so = (int64_t)a.Hq * a.D;
  const int32_t own = w.first / 32, blocks = (w.t.len + 31) / 32, k_min = blk_rank[2 * own], k_max = blk_rank[2 * own + 1];
  const uint32_t q_tile = lds_address(&sh.tiles[0][0]) + w.wave * 2 * TL::BYTES, o_tile = q_tile + TL::BYTES;
  // the wave takes every fourth round
  const int32_t per_head = blocks - own;
  struct Where { int32_t round, g, b; };
  auto settle = [&](int32_t round) -> Where {  // the first from this one on, in steps of four, with a query that sees a key
    Where x{round, round / per_head, own + round % per_head};
    while (x.round < item.end && k_min > blk_rank[2 * x.b + 1]) {
      x.round += 4;
      for (x.b += 4; x.b >= blocks; ++x.g) x.b -= per_head;
    }
    return x;
  };
  typename TL::Source queries, gradients;
  queries.init(q + w.t.seq0 * a.sq, a.sq, w.t.len, a.D, w.lane);
  gradients.init(d_out + w.t.seq0 * so, so, w.t.len, a.D, w.lane);
  auto load_queries = [&](Where x) { queries.load(q_tile, x.b * 32, w.lane, (int64_t)(hk * G + x.g) * a.D * 4); };
  auto load_gradients = [&](Where x) {
    const int32_t hq = hk * G + x.g;
    gradients.load(o_tile, x.b * 32, w.lane, (int64_t)hq * a.D * 4);
    const float* p = (w.h ? delta : lse) + hq * a.N + w.t.seq0 + min(x.b * 32 + w.n, w.t.len - 1);
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_address(&stats[w.wave][0]));
    uint32_t keep;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
        "global_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
        : "=&s"(keep)
        : "v"(p), "s"(dst)
        : "memory");
  };
  if (LDS_VALUES) {
    if (w.wave == 0) {
      typename TL::Source own;
      own.init(v + w.t.seq0 * a.sv + (int64_t)hk * a.D, a.sv, w.t.len, a.D, w.lane);
      own.load(lds_address(values), w.first, w.lane, 0, a.D < DP ? a.rank + a.N : nullptr);
      wait_vector_memory<0>();
    }
    __syncthreads();
  }
  Where x = settle(item.begin + w.wave);
  if (x.round < item.end) {
    load_queries(x);
    load_gradients(x);
  }
  typename TL::Own kf, vf;
  TL::load(kf, k + token * a.sk + (int64_t)hk * a.D, w.h, a.D);
  if (!LDS_VALUES) TL::load(vf, v + token * a.sv + (int64_t)hk * a.D, w.h, a.D);
  int32_t rank_j[1] = {ranks[w.ic]};
  own_arrived(kf.f);
  if (!LDS_VALUES) own_arrived(vf.f);
  arrived(rank_j);
  const float c = a.scale * LOG2E;
  const uint32_t at = TL::row_offset(w.n, w.h);
  floatx16 acc_k[TL::NB], acc_v[TL::NB];
  zero(acc_k, TL::NB);
  zero(acc_v, TL::NB);
  while (x.round < item.end) {
    const Where after = settle(x.round + 4);
    wait_vector_memory<TL::LOADS + 1>();  // the queries; the gradients and the rows' numbers were requested behind them
    floatx16 s = TL::scores(q_tile, at, kf, floatx16{});
    wait_vector_memory<0>();
    const floatx16 dp = LDS_VALUES ? TL::scores(o_tile, at, lds_address(values), floatx16{})
                                   : TL::scores(o_tile, at, vf, floatx16{});
    if (x.b == own || k_max > blk_rank[2 * x.b] || (x.b + 1) * 32 > w.t.len) {
      BlockRanks rk;
      rk.load(ranks + x.b * 32);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int32_t i = x.b * 32 + tile_row(r, w.h);
        s[r] = i < w.t.len && i >= w.i && rank_j[0] <= rk.of(r, w.h) ? s[r] : -INFINITY;
      }
    }
    float p[16], ds[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = fast_exp2(fmaf(s[r], c, -LOG2E * stats[w.wave][tile_row(r, w.h)]));
      ds[r] = p[r] * (dp[r] - stats[w.wave][32 + tile_row(r, w.h)]);
    }
    TL::add(q_tile, w.n, w.h, ds, acc_k);
    if (after.round < item.end) load_queries(after);
    TL::add(o_tile, w.n, w.h, p, acc_v);
    if (after.round < item.end) load_gradients(after);
    x = after;
  }
  __syncthreads();
  put(sh, w, acc_v, 1.f);
  __syncthreads();
  if (item.slot >= 0) {
    float* const p = partial + ((int64_t)item.slot * a.Hkv + hk) * (2 * 32 * DP);
    join(sh, w, p + 32 * DP, DP, DP);
    __syncthreads();
    put(sh, w, acc_k, 1.f);
    __syncthreads();
    join(sh, w, p, DP, DP);
    return;
  }
  join(sh, w, dv + (w.t.seq0 + (int64_t)w.first) * a.sdv + (int64_t)hk * a.D, a.sdv, a.D);
  __syncthreads();
  put(sh, w, acc_k, a.scale);
  __syncthreads();
  join(sh, w, dk + (w.t.seq0 + (int64_t)w.first) * a.sdk + (int64_t)hk * a.D, a.sdk, a.D);
}

// Adds up the partial sums of 32 keys, in the order of their items, those of four items on their way at a time.  A
// workgroup has eight keys of dk (even) or dv.
template <int DP>
__global__ void __launch_bounds__(8 * DP / 4) ft_f32_dkv_join_kernel(FtArgs a, const hpd_ft_item* __restrict__ joins,
                                                                    const float* __restrict__ partial,
                                                                    float* __restrict__ dk, float* __restrict__ dv) {
  const int32_t y = blockIdx.x & 1, r = (blockIdx.x >> 1 & 3) * 8 + threadIdx.x / (DP / 4), c = threadIdx.x % (DP / 4) * 4;
  const int32_t hk = (blockIdx.x >> 3) % a.Hkv;
  const hpd_ft_item t = joins[(blockIdx.x >> 3) / a.Hkv];  // slots [slot, slot + end)
  if (t.row0 + r >= t.len || c >= a.D) return;
  const int64_t step = (int64_t)a.Hkv * (2 * 32 * DP);
  const float* p = partial + ((int64_t)t.slot * a.Hkv + hk) * (2 * 32 * DP) + (y * 32 + r) * DP + c;
  float4 sum = {};
  for (int32_t i = 0; i < t.end; i += 4) {
    float4 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < t.end) w[j] = *reinterpret_cast<const float4*>(p + (i + j) * step);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < t.end) {
        sum.x += w[j].x; sum.y += w[j].y; sum.z += w[j].z; sum.w += w[j].w;
      }
  }
  const float f = y ? 1.f : a.scale;
  const int64_t token = t.seq0 + (int64_t)t.row0 + r;
  *reinterpret_cast<float4*>((y ? dv + token * a.sdv : dk + token * a.sdk) + (int64_t)hk * a.D + c) =
      make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f);
}

template <int DP>
hipError_t forward(const hpd_finetune_layout* L, const FtArgs& a, const float* q, const float* k, const float* v, float* out,
                   float* lse, hipStream_t s) {
  ft_f32_forward_kernel<DP><<<dim3((unsigned)hpd_ft_query_groups(L)), 256, 0, s>>>(a, q, k, v, out, lse);
  return hipGetLastError();
}

template <int DP>
hipError_t backward(const hpd_finetune_layout* L, FtArgs a, const float* q, const float* k, const float* v, const float* out,
                    const float* lse, const float* d_out, float* dq, float* dk, float* dv, float* delta, hipStream_t s) {
  ft_f32_delta_kernel<<<dim3((unsigned)((a.N * a.Hq + 15) / 16)), 256, 0, s>>>(a.N, a.Hq, a.D, out, d_out, delta);
  ft_f32_dq_kernel<DP><<<dim3((unsigned)hpd_ft_query_groups(L)), 256, 0, s>>>(a, q, k, v, d_out, lse, delta, dq);
  float* partial = delta + 2 * a.N * a.Hq + (-2 * a.N * a.Hq & 3);  // (on 16 bytes)
  ft_f32_dkv_kernel<DP><<<dim3((unsigned)hpd_ft_key_groups(L)), 256, 0, s>>>(a, L->d_items, q, k, v, d_out, lse, delta, partial, dk, dv);
  if (!L->joins.empty())
    ft_f32_dkv_join_kernel<DP><<<dim3((unsigned)L->joins.size() * a.Hkv * 8), 2 * DP, 0, s>>>(a, L->d_joins, partial, dk, dv);
  return hipGetLastError();
}

}  // namespace

hipError_t hpd_launch_ft_f32_forward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                     void* out, float* lse, hipStream_t s) {
  const auto run = a.D <= 64 ? forward<64> : a.D <= 96 ? forward<96> : forward<128>;
  return run(L, a, (const float*)q, (const float*)k, (const float*)v, (float*)out, lse, s);
}

hipError_t hpd_launch_ft_f32_backward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v,
                                      const void* out, const float* lse, const void* d_out, void* dq, void* dk, void* dv,
                                      void* workspace, hipStream_t s) {
  const auto run = a.D <= 64 ? backward<64> : a.D <= 96 ? backward<96> : backward<128>;
  return run(L, a, (const float*)q, (const float*)k, (const float*)v, (const float*)out, lse, (const float*)d_out, (float*)dq,
             (float*)dk, (float*)dv, (float*)workspace, s);
}
