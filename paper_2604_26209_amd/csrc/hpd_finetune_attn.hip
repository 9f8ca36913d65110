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
  else *reinterpret_cast<uint2*>(p) = make_uint2(cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]));
}

// A wave per token: D / (2 V) lanes a head, as many heads side by side as fit; the token's (cos, sin)
// stay in registers over its heads.  Bound by its bytes: 19740 tokens, 32/8 heads of 128, bf16: 79 us, 5.1 TB/s (a large copy: 5.0).
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
  a.seen_off = L->d_seen_off;
  a.seen = L->d_seen;
  a.N = L->n_tokens;
  a.sq = st.q; a.sk = st.k; a.sv = st.v;
  a.sdq = st.q_out; a.sdk = st.k_out; a.sdv = st.v_out;
  a.Hq = L->cfg.n_q_heads; a.Hkv = L->cfg.n_kv_heads; a.D = L->cfg.head_dim;
  a.scale = (float)(1.0 / sqrt((double)a.D));
  return a;
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
                                   float* lse, void* workspace, const hpd_finetune_strides& st, hipStream_t s) {
  const FtArgs a = make_args(L, st);
  if (L->cfg.dtype == HPD_F32) return hpd_launch_ft_f32_forward(L, a, q, k, v, out, lse, s);
  return hpd_launch_ft_stream_forward(L, a, q, k, v, out, lse, workspace, s);
}

hipError_t hpd_launch_ft_attention_backward(const hpd_finetune_layout* L, const void* q, const void* k, const void* v,
                                            const void* out, const float* lse, const void* d_out, void* dq, void* dk,
                                            void* dv, void* workspace, const hpd_finetune_strides& st, hipStream_t s) {
  const FtArgs a = make_args(L, st);
  if (L->cfg.dtype == HPD_F32) return hpd_launch_ft_f32_backward(L, a, q, k, v, out, lse, d_out, dq, dk, dv, workspace, s);
  return hpd_launch_ft_stream_backward(L, a, q, k, v, out, lse, d_out, dq, dk, dv, workspace, s);
}
