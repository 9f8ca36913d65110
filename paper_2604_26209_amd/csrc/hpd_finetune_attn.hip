// Attention of a fine-tuning step under the HPD mask (Section 4.4), its gradient, and the rotation of
// queries and keys at the position IDs of the training sequences.
//
// Mask: token i of a sequence sees token j iff j <= i and rank_j <= rank_i (rank k for the k-th token
// of a value, 0 for prompt and attribute names).
//
// Forward, per query head:  p_ij = exp(s_ij - lse_i),  s_ij = q_i . k_j / sqrt(D),  o_i = sum_j p_ij v_j
// Backward:  delta_i = do_i . o_i,  dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - delta_i) / sqrt(D),
//            dq_i = sum_j ds_ij k_j,  dk_j = sum_i ds_ij q_i  (dk, dv: over the query heads of the kv head too)
//
// All products run on the 32x32 matrix instructions with the same scheme.  A wave owns 32 tokens as
// the columns of its tiles (queries in the forward and dq kernels, keys in the dk/dv kernel) and
// holds their rows in registers as the right operand.  The other side's tokens come as tiles of 32
// rows in LDS: read by rows they are the left operand of the score products, read by columns the
// left operand of the second products, whose right operand is the result of the first as it lies in
// the registers: register r of a lane in half h of the wave holds row 8 (r / 4) + 4 h + r % 4 of the
// lane's column, and the column reads take the rows in that order.
#include "hpd_finetune_dev.h"

namespace {

constexpr int ROWS = HPD_FT_ROWS;
constexpr int BLK = HPD_FT_BLOCK;
constexpr int WAVES = ROWS / 32;

typedef hpd::bf16_t T;

// Operand layouts.  A fragment is 16 bytes a lane: the chunk 2 * step + h of the row of the lane (h = lane / 32).
struct Elem {
  static constexpr int CHUNK = 8;  // elements of 16 bytes
  static __device__ __forceinline__ floatx16 product(uint4 a, uint4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  struct Right {  // a 32 x 32 result as the right operand of the next product
    bf16x8 f[2];
  };
  static __device__ __forceinline__ Right right(const float* p) { return {{pack8(p), pack8(p + 8)}}; }
  // acc += (columns of the tile)^T . p; at: the lane's address of block 0 (see column_address), pitch in bytes
  template <int PITCH>
  static __device__ __forceinline__ floatx16 columns(const char* at, const Right& p, floatx16 c) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint2 lo = hpd::lds_read_tr16(at + k * 16 * PITCH), hi = hpd::lds_read_tr16(at + (k * 16 + 8) * PITCH);
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y)), p.f[k], c,
                                                  0, 0, 0);
    }
    return c;
  }
  // The transposing read gives lane i of 16 the channel i of four rows; the lanes 4 j .. 4 j + 3 address row j.
  template <int PITCH>
  static __device__ __forceinline__ int column_address(int lane) {
    return (4 * (lane >> 5) + ((lane & 15) >> 2)) * PITCH + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
  }
  static __device__ __forceinline__ void store4(hpd::bf16_t* p, const float* v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
  }
};
// Kernels for bf16 with any D up to DP (zeros behind it): tiles through registers, one tile at a time.
template <int DP>
struct Tile {
  using E = Elem;
  static constexpr int PITCH = DP * (int)sizeof(T) + 16;  // odd in chunks: the rows of a read start in different banks
  static constexpr int CHUNKS = DP / E::CHUNK;
  static constexpr int STEPS = CHUNKS / 2;
  static constexpr int BYTES = BLK * PITCH;
  // rows [first, first + 32) of a sequence; zeros from its end and from D on.  src: the sequence's
  // first token, this head
  static __device__ __forceinline__ void load(char* lds, const T* src, int64_t stride, int32_t first, int32_t len, int32_t D) {
    for (int i = threadIdx.x; i < BLK * CHUNKS; i += WAVES * 64) {
      const int r = i / CHUNKS, c = i % CHUNKS;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (first + r < len && c * E::CHUNK < D) v = *reinterpret_cast<const uint4*>(src + (first + r) * stride + c * E::CHUNK);
      *reinterpret_cast<uint4*>(lds + r * PITCH + c * 16) = v;
    }
  }
  // the wave's own rows as right operands; row: the lane's token, clamped to the sequence
  static __device__ __forceinline__ void own(uint4* f, const T* row, int h, int32_t D) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = 2 * s + h;
      f[s] = c * E::CHUNK < D ? *reinterpret_cast<const uint4*>(row + c * E::CHUNK) : make_uint4(0, 0, 0, 0);
    }
  }
  // tile rows x own rows
  static __device__ __forceinline__ floatx16 scores(const char* lds, const uint4* f, int lane) {
    const char* at = lds + (lane & 31) * PITCH + (lane >> 5) * 16;
    floatx16 c;
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i] = 0.f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) c = E::product(*reinterpret_cast<const uint4*>(at + s * 32), f[s], c);
    return c;
  }
  static __device__ __forceinline__ void add_columns(const char* lds, const E::Right& p, floatx16* acc, int lane) {
    const char* at = lds + E::column_address<PITCH>(lane);
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) acc[b] = E::columns<PITCH>(at + b * 32 * (int)sizeof(T), p, acc[b]);
  }
  // acc * f to one row of the output
  static __device__ __forceinline__ void store(T* row, const floatx16* acc, float f, int h, int32_t D) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int c = 32 * b + 8 * a + 4 * h;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[b][4 * a + e] * f;
        if (c < D) E::store4(row + c, v);
      }
  }
};

template <int DP>
__global__ void __launch_bounds__(WAVES * 64) ft_forward_kernel(FtArgs a, const T* __restrict__ q, const T* __restrict__ k,
                                                               const T* __restrict__ v, T* __restrict__ out,
                                                               float* __restrict__ lse) {
  using TL = Tile<DP>;
  __shared__ __attribute__((aligned(16))) char lds_k[TL::BYTES], lds_v[TL::BYTES];
  __shared__ int32_t lds_rank[BLK];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, h = lane >> 5;
  const int32_t hq = blockIdx.x % a.Hq, hk = hq / (a.Hq / a.Hkv);
  const hpd_ft_tile t = a.tiles[blockIdx.x / a.Hq];
  const int32_t q_first = t.row0 + wave * 32;
  const bool active = q_first < t.len;
  const int32_t i = q_first + n, ic = min(i, t.len - 1);  // own row; behind the end: the last one
  const int64_t token = t.seq0 + (int64_t)ic;
  uint4 qf[TL::STEPS];
  TL::own(qf, q + token * a.sq + hq * (int64_t)a.D, h, a.D);
  const int32_t rank_i = a.rank[token];
  const int2 rank_q = active ? a.blk_rank[t.blk0 + q_first / BLK] : make_int2(0, 0);
  const float c = a.scale * LOG2E;

  floatx16 acc[DP / 32];
  zero(acc, DP / 32);
  float m = -INFINITY, l = 0.f;  // running maximum (log2 units) and sum
  const int32_t blocks = (min(t.row0 + ROWS, t.len) + BLK - 1) / BLK;
  for (int32_t b = 0; b < blocks; ++b) {
    __syncthreads();
    TL::load(lds_k, k + t.seq0 * a.sk + hk * (int64_t)a.D, a.sk, b * BLK, t.len, a.D);
    TL::load(lds_v, v + t.seq0 * a.sv + hk * (int64_t)a.D, a.sv, b * BLK, t.len, a.D);
    if (threadIdx.x < BLK) lds_rank[threadIdx.x] = a.rank[t.seq0 + min(b * BLK + (int32_t)threadIdx.x, t.len - 1)];
    __syncthreads();
    if (!active || b * BLK > q_first + 31) continue;
    const int2 rank_k = a.blk_rank[t.blk0 + b];
    if (rank_k.x > rank_q.y) continue;  // no query sees any of these keys
    const floatx16 s = TL::scores(lds_k, qf, lane);
    float p[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = s[r] * c;
    if (b * BLK + BLK - 1 > q_first || rank_k.y > rank_q.x) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = tile_row(r, h);
        p[r] = b * BLK + row <= ic && lds_rank[row] <= rank_i ? p[r] : -INFINITY;
      }
    }
    float top = m;
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, p[r]);
    top = fmaxf(top, __shfl_xor(top, 32));
    const float ref = top == -INFINITY ? 0.f : top;  // (no key seen so far: every weight below is 0)
    const float alpha = fast_exp2(m - ref);
    m = top;
    l *= alpha;
#pragma unroll
    for (int x = 0; x < DP / 32; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][r] *= alpha;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = fast_exp2(p[r] - ref);
      l += p[r];
    }
    TL::add_columns(lds_v, TL::E::right(p), acc, lane);
  }
  if (!active || i >= t.len) return;
  l += __shfl_xor(l, 32);
  TL::store(out + (token * a.Hq + hq) * a.D, acc, 1.f / l, h, a.D);
  if (h == 0) lse[hq * a.N + token] = (m + __builtin_amdgcn_logf(l)) * LN2;
}

// delta_i = do_i . o_i: 16 lanes a row
__global__ void __launch_bounds__(256) ft_delta_kernel(int64_t N, int32_t Hq, int32_t D, const T* __restrict__ out,
                                                       const T* __restrict__ d_out, float* __restrict__ delta) {
  const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;  // 16 lanes a row
  if (row >= N * Hq) return;
  float s = 0.f;
  for (int32_t c = (threadIdx.x % 16) * 8; c < D; c += 128) {
    float x[8], y[8];
    hpd::load8(out + row * D + c, x);
    hpd::load8(d_out + row * D + c, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
  }
#pragma unroll
  for (int d = 8; d; d >>= 1) s += __shfl_xor(s, d);
  if (threadIdx.x % 16 == 0) delta[(row % Hq) * N + row / Hq] = s;
}

template <int DP>
__global__ void __launch_bounds__(WAVES * 64, 1) ft_dq_kernel(FtArgs a, const T* __restrict__ q, const T* __restrict__ k,
                                                          const T* __restrict__ v, const T* __restrict__ d_out,
                                                          const float* __restrict__ lse, const float* __restrict__ delta,
                                                          T* __restrict__ dq) {
  using TL = Tile<DP>;
  __shared__ __attribute__((aligned(16))) char lds_k[TL::BYTES], lds_v[TL::BYTES];
  __shared__ int32_t lds_rank[BLK];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, h = lane >> 5;
  const int32_t hq = blockIdx.x % a.Hq, hk = hq / (a.Hq / a.Hkv);
  const hpd_ft_tile t = a.tiles[blockIdx.x / a.Hq];
  const int32_t q_first = t.row0 + wave * 32;
  const bool active = q_first < t.len;
  const int32_t i = q_first + n, ic = min(i, t.len - 1);
  const int64_t token = t.seq0 + (int64_t)ic;
  uint4 qf[TL::STEPS], of[TL::STEPS];
  TL::own(qf, q + token * a.sq + hq * (int64_t)a.D, h, a.D);
  TL::own(of, d_out + (token * a.Hq + hq) * a.D, h, a.D);
  const int32_t rank_i = a.rank[token];
  const int2 rank_q = active ? a.blk_rank[t.blk0 + q_first / BLK] : make_int2(0, 0);
  const float c = a.scale * LOG2E, lse2 = lse[hq * a.N + token] * LOG2E, dl = delta[hq * a.N + token];

  floatx16 acc[DP / 32];
  zero(acc, DP / 32);
  const int32_t blocks = (min(t.row0 + ROWS, t.len) + BLK - 1) / BLK;
  for (int32_t b = 0; b < blocks; ++b) {
    __syncthreads();
    TL::load(lds_k, k + t.seq0 * a.sk + hk * (int64_t)a.D, a.sk, b * BLK, t.len, a.D);
    TL::load(lds_v, v + t.seq0 * a.sv + hk * (int64_t)a.D, a.sv, b * BLK, t.len, a.D);
    if (threadIdx.x < BLK) lds_rank[threadIdx.x] = a.rank[t.seq0 + min(b * BLK + (int32_t)threadIdx.x, t.len - 1)];
    __syncthreads();
    if (!active || b * BLK > q_first + 31) continue;
    const int2 rank_k = a.blk_rank[t.blk0 + b];
    if (rank_k.x > rank_q.y) continue;
    const floatx16 s = TL::scores(lds_k, qf, lane), dp = TL::scores(lds_v, of, lane);
    const bool masked = b * BLK + BLK - 1 > q_first || rank_k.y > rank_q.x;
    float ds[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      ds[r] = fast_exp2(fmaf(s[r], c, -lse2)) * (dp[r] - dl);
      if (masked) {
        const int row = tile_row(r, h);
        ds[r] = b * BLK + row <= ic && lds_rank[row] <= rank_i ? ds[r] : 0.f;
      }
    }
    TL::add_columns(lds_k, TL::E::right(ds), acc, lane);
  }
  if (!active || i >= t.len) return;
  TL::store(dq + token * a.sdq + hq * (int64_t)a.D, acc, a.scale, h, a.D);
}

template <int DP>
__global__ void __launch_bounds__(WAVES * 64, 1) ft_dkv_kernel(FtArgs a, const T* __restrict__ q, const T* __restrict__ k,
                                                           const T* __restrict__ v, const T* __restrict__ d_out,
                                                           const float* __restrict__ lse, const float* __restrict__ delta,
                                                           T* __restrict__ dk, T* __restrict__ dv) {
  using TL = Tile<DP>;
  __shared__ __attribute__((aligned(16))) char lds_q[TL::BYTES], lds_o[TL::BYTES];
  __shared__ int32_t lds_rank[BLK];
  __shared__ float lds_lse[BLK], lds_delta[BLK];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 31, h = lane >> 5;
  const int32_t hk = blockIdx.x % a.Hkv, G = a.Hq / a.Hkv;
  const hpd_ft_tile t = a.tiles[blockIdx.x / a.Hkv];
  const int32_t k_first = t.row0 + wave * 32;
  const bool active = k_first < t.len;
  const int32_t j = k_first + n, jc = min(j, t.len - 1);
  const int64_t token = t.seq0 + (int64_t)jc;
  uint4 kf[TL::STEPS], vf[TL::STEPS];
  TL::own(kf, k + token * a.sk + hk * (int64_t)a.D, h, a.D);
  TL::own(vf, v + token * a.sv + hk * (int64_t)a.D, h, a.D);
  const int32_t rank_j = a.rank[token];
  const int2 rank_k = active ? a.blk_rank[t.blk0 + k_first / BLK] : make_int2(0, 0);
  const float c = a.scale * LOG2E;

  floatx16 acc_k[DP / 32], acc_v[DP / 32];
  zero(acc_k, DP / 32);
  zero(acc_v, DP / 32);
  const int32_t blocks = (t.len + BLK - 1) / BLK;
  for (int32_t g = 0; g < G; ++g) {
    const int32_t hq = hk * G + g;
    for (int32_t b = t.row0 / BLK; b < blocks; ++b) {
      __syncthreads();
      TL::load(lds_q, q + t.seq0 * a.sq + hq * (int64_t)a.D, a.sq, b * BLK, t.len, a.D);
      TL::load(lds_o, d_out + ((int64_t)t.seq0 * a.Hq + hq) * a.D, (int64_t)a.Hq * a.D, b * BLK, t.len, a.D);
      if (threadIdx.x < BLK) {
        const int64_t tok = t.seq0 + (int64_t)min(b * BLK + (int32_t)threadIdx.x, t.len - 1);
        lds_rank[threadIdx.x] = a.rank[tok];
        lds_lse[threadIdx.x] = lse[hq * a.N + tok] * LOG2E;
        lds_delta[threadIdx.x] = delta[hq * a.N + tok];
      }
      __syncthreads();
      if (!active || b * BLK + BLK - 1 < k_first) continue;
      const int2 rank_q = a.blk_rank[t.blk0 + b];
      if (rank_k.x > rank_q.y) continue;
      const floatx16 s = TL::scores(lds_q, kf, lane), dp = TL::scores(lds_o, vf, lane);
      const bool masked = b * BLK < k_first + 31 || rank_k.y > rank_q.x || (b + 1) * BLK > t.len;
      float p[16], ds[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = tile_row(r, h);
        p[r] = fast_exp2(fmaf(s[r], c, -lds_lse[row]));
        ds[r] = p[r] * (dp[r] - lds_delta[row]);
        if (masked) {
          const bool seen = b * BLK + row < t.len && b * BLK + row >= j && rank_j <= lds_rank[row];
          p[r] = seen ? p[r] : 0.f;
          ds[r] = seen ? ds[r] : 0.f;
        }
      }
      TL::add_columns(lds_o, TL::E::right(p), acc_v, lane);
      TL::add_columns(lds_q, TL::E::right(ds), acc_k, lane);
    }
  }
  if (!active || j >= t.len) return;
  TL::store(dv + token * a.sdv + hk * (int64_t)a.D, acc_v, 1.f, h, a.D);
  TL::store(dk + token * a.sdk + hk * (int64_t)a.D, acc_k, a.scale, h, a.D);
}

// (cos, sin) of position * base^(-2m/D), in 64 bits
__global__ void __launch_bounds__(256) ft_rope_table_kernel(const int32_t* __restrict__ pos, int32_t rows, int32_t half,
                                                            double base, float2* __restrict__ table) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)rows * half) return;
  const int32_t r = (int32_t)(i / half), m = (int32_t)(i % half);
  double s, c;
  sincos((double)(pos ? pos[r] : r) * pow(base, -(double)m / half), &s, &c);
  table[i] = make_float2((float)c, (float)s);
}

// V consecutive elements to fp32 and back
template <int V, typename E>
__device__ __forceinline__ void load_vec(const E* p, float* f) {
  if constexpr (sizeof(E) == 4) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
  } else if constexpr (V == 8) {
    unpack8(*reinterpret_cast<const uint4*>(p), f);
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    f[0] = __uint_as_float(x.x << 16); f[1] = __uint_as_float(x.x & 0xffff0000u);
    f[2] = __uint_as_float(x.y << 16); f[3] = __uint_as_float(x.y & 0xffff0000u);
  }
}
template <int V, typename E>
__device__ __forceinline__ void store_vec(E* p, const float* f) {
  if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  else if constexpr (V == 8) *reinterpret_cast<uint4*>(p) = __builtin_bit_cast(uint4, pack8(f));
  else Elem::store4(p, f);
}

// A wave per token: D / (2 V) lanes a head, as many heads side by side as fit; the token's (cos, sin)
// stay in registers over its heads.  Bytes-bound.
template <typename E, int V>
__global__ void __launch_bounds__(256) ft_rotate_kernel(int32_t N, int32_t Hq, int32_t Hkv, int32_t D, int64_t sq, int64_t sk,
                                                        int64_t sqo, int64_t sko, float sign, const float2* __restrict__ rope,
                                                        const int32_t* __restrict__ row, const E* q, const E* k, E* q_out,
                                                        E* k_out) {
  const int32_t token = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (token >= N) return;
  const int32_t half = D / 2, lanes = half / V, side = 64 / lanes;
  const int32_t m = lane % lanes * V;
  if (lane / lanes >= side) return;
  const float2* cs = rope + (int64_t)(row ? row[token] : token) * half + m;
  float c[V], s[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    c[e] = cs[e].x;
    s[e] = cs[e].y * sign;
  }
  for (int32_t h = lane / lanes; h < Hq + Hkv; h += side) {
    const E* in = h < Hq ? q + token * sq + (int64_t)h * D : k + token * sk + (int64_t)(h - Hq) * D;
    E* to = h < Hq ? q_out + token * sqo + (int64_t)h * D : k_out + token * sko + (int64_t)(h - Hq) * D;
    float x[V], y[V], rx[V], ry[V];
    load_vec<V>(in + m, x);
    load_vec<V>(in + half + m, y);
#pragma unroll
    for (int e = 0; e < V; ++e) hpd::rope_pair(x[e], y[e], c[e], s[e], rx[e], ry[e]);
    store_vec<V>(to + m, rx);
    store_vec<V>(to + half + m, ry);
  }
}

FtArgs make_args(const hpd_finetune_layout* L, const hpd_finetune_strides& st) {
  FtArgs a{};
  a.tiles = L->d_tiles;
  a.rank = L->d_rank;
  a.blk_rank = L->d_blk_rank;
  a.N = L->n_tokens;
  a.sq = st.q; a.sk = st.k; a.sv = st.v;
  a.sdq = st.q_out; a.sdk = st.k_out; a.sdv = st.v_out;
  a.Hq = L->cfg.n_q_heads; a.Hkv = L->cfg.n_kv_heads; a.D = L->cfg.head_dim;
  a.scale = (float)(1.0 / sqrt((double)a.D));
  return a;
}

template <int DP>
hipError_t forward(const hpd_finetune_layout* L, const FtArgs& a, const void* q, const void* k, const void* v, void* out,
                   float* lse, hipStream_t s) {
  ft_forward_kernel<DP><<<dim3((unsigned)L->tiles.size() * a.Hq), WAVES * 64, 0, s>>>(
      a, (const T*)q, (const T*)k, (const T*)v, (T*)out, lse);
  return hipGetLastError();
}

template <int DP>
hipError_t backward(const hpd_finetune_layout* L, FtArgs a, const void* q, const void* k, const void* v, const void* out,
                    const float* lse, const void* d_out, void* dq, void* dk, void* dv, float* delta, hipStream_t s) {
  ft_delta_kernel<<<dim3((unsigned)((a.N * a.Hq + 15) / 16)), 256, 0, s>>>(a.N, a.Hq, a.D, (const T*)out, (const T*)d_out,
                                                                            delta);
  ft_dq_kernel<DP><<<dim3((unsigned)L->tiles.size() * a.Hq), WAVES * 64, 0, s>>>(
      a, (const T*)q, (const T*)k, (const T*)v, (const T*)d_out, lse, delta, (T*)dq);
  a.tiles = L->d_key_tiles;
  ft_dkv_kernel<DP><<<dim3((unsigned)L->tiles.size() * a.Hkv), WAVES * 64, 0, s>>>(
      a, (const T*)q, (const T*)k, (const T*)v, (const T*)d_out, lse, delta, (T*)dk, (T*)dv);
  return hipGetLastError();
}

template <typename E, int V>
hipError_t rotate(const hpd_finetune_layout* L, float sign, const void* q, const void* k, void* q_out, void* k_out,
                  const hpd_finetune_strides& st, hipStream_t s) {
  ft_rotate_kernel<E, V><<<dim3((unsigned)(L->n_tokens + 3) / 4), 256, 0, s>>>(
      L->n_tokens, L->cfg.n_q_heads, L->cfg.n_kv_heads, L->cfg.head_dim, st.q, st.k, st.q_out, st.k_out, sign, L->d_rope,
      L->rope_by_token ? nullptr : L->d_pos, (const E*)q, (const E*)k, (E*)q_out, (E*)k_out);
  return hipGetLastError();
}

}  // namespace

hipError_t hpd_launch_ft_rope_table(const hpd_finetune_layout* L, hipStream_t s) {
  const int32_t half = L->cfg.head_dim / 2;
  const int64_t n = (int64_t)L->rope_rows * half;
  ft_rope_table_kernel<<<dim3((unsigned)((n + 255) / 256)), 256, 0, s>>>(L->rope_by_token ? L->d_pos : nullptr, L->rope_rows,
                                                                       half, L->cfg.rope_base, L->d_rope);
  return hipGetLastError();
}

hipError_t hpd_launch_ft_rotate(const hpd_finetune_layout* L, bool inverse, const void* q, const void* k, void* q_out,
                                void* k_out, const hpd_finetune_strides& st, hipStream_t s) {
  const float sign = inverse ? -1.f : 1.f;
  if (L->cfg.dtype == HPD_F32) return rotate<float, 4>(L, sign, q, k, q_out, k_out, st, s);
  if (L->cfg.head_dim % 16 == 0) return rotate<hpd::bf16_t, 8>(L, sign, q, k, q_out, k_out, st, s);
  return rotate<hpd::bf16_t, 4>(L, sign, q, k, q_out, k_out, st, s);
}

hipError_t hpd_launch_ft_attention(const hpd_finetune_layout* L, const void* q, const void* k, const void* v, void* out,
                                   float* lse, void*, const hpd_finetune_strides& st, hipStream_t s) {
  const FtArgs a = make_args(L, st);
  if (hpd_ft_stream_supported(L)) return hpd_launch_ft_stream_forward(L, a, q, k, v, out, lse, s);
  if (L->cfg.dtype == HPD_F32) return hpd_launch_ft_f32_forward(L, a, q, k, v, out, lse, s);
  return a.D <= 64 ? forward<64>(L, a, q, k, v, out, lse, s)
                   : forward<128>(L, a, q, k, v, out, lse, s);
}

hipError_t hpd_launch_ft_attention_backward(const hpd_finetune_layout* L, const void* q, const void* k, const void* v,
                                            const void* out, const float* lse, const void* d_out, void* dq, void* dk,
                                            void* dv, void* workspace, const hpd_finetune_strides& st, hipStream_t s) {
  const FtArgs a = make_args(L, st);
  if (hpd_ft_stream_supported(L))
    return hpd_launch_ft_stream_backward(L, a, q, k, v, out, lse, d_out, dq, dk, dv, workspace, s);
  if (L->cfg.dtype == HPD_F32) return hpd_launch_ft_f32_backward(L, a, q, k, v, out, lse, d_out, dq, dk, dv, workspace, s);
  float* delta = (float*)workspace;
  return a.D <= 64 ? backward<64>(L, a, q, k, v, out, lse, d_out, dq, dk, dv, delta, s)
                   : backward<128>(L, a, q, k, v, out, lse, d_out, dq, dk, dv, delta, s);
}
