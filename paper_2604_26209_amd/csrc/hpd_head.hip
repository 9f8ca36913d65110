// Log probabilities of given tokens from hidden states and the vocabulary's weights, and their gradients; the logits
// x = hidden W^T stay in registers.
//
// Forward: a tile's rows give (m, s, t) = (max x, sum e^(x - m), sum e^(x - m) (x - m)) of its tokens of the vocabulary; a
// second kernel joins a row's tiles: lse = m + log s, entropy = log s - t / s.  Few tokens: parts of the logits in fp32, summed and taken in
// by the second kernel.  The maximum is subtracted before anything is scaled, so
// that logits of any finite size keep the accuracy that they have.
// Backward: piece by piece of the vocabulary, the logits again and from them dx_c = g ([c = target] - p) - ge p (log p + entropy),
// rounded to the inputs' type; then the piece's rows of dW = dx^T hidden, and its part of dhidden = dx W in fp32.  A piece's gradients
// are at most 256 MB (up to 524288 rows in bf16, 262144 in fp32), what the memory side caches hold, so that both products read them from
// there, and 8 MB a row.
//
// What bounds it: the matrix units under the clock that their power leaves (bf16: 6144 rows of 130013 tokens, 4096 channels, 5.45 ms, 1.20
// PFLOP/s; gradients of 4096 rows of 32000 tokens 2.75 ms, 1.17, of 2021 of 130013 5.75, 1.12; fp32: gradients of 700 rows of 50021 tokens and 1152 channels 1.26 ms, 0.128
// PFLOP/s); few rows, the weights' bytes (three rows of 150001 tokens 190 us, 6.4 TB/s).
#include <algorithm>

#include "hpd_ffn.h"
#include "hpd_product.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

struct Sums {
  float m, s, t;
};
// (a part without logits above -infinity: m = -infinity, s = 0)
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  const float da = a.s == 0.f ? 0.f : fmaxf(a.m - m, -1e4f), db = b.s == 0.f ? 0.f : fmaxf(b.m - m, -1e4f);
  const float fa = fast_exp2(da * LOG2E), fb = fast_exp2(db * LOG2E);
  return {m, fmaf(a.s, fa, b.s * fb), fmaf(da, a.s, a.t) * fa + fmaf(db, b.s, b.t) * fb};
}

// what the forward product leaves of a row and a tile of the vocabulary
struct RowSums {
  const int32_t* targets;
  float* of_target;  // [rows]: the target's logit (written by the tile that has it)
  float4* parts;     // [rows][tiles]
  int32_t vocab, tiles;
  int64_t rows;
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char* smem) const {
    const int l = at.lane & 31, h = at.lane >> 5;
    float4* const shared = reinterpret_cast<float4*>(smem);  // [WM][BN]
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t row = at.row + 32 * j + l;
      const int32_t target = targets && row < rows ? targets[row] : -1;
      const int64_t behind = (int64_t)target - at.feature;
      const int32_t mine = behind < 0 || behind >= 32 * MI ? -1 : (int32_t)behind;  // the target, counted from the wave's first
      const int64_t inside = vocab - at.feature;  // the wave's tokens that exist
      float x[MI][16];
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[i][r] = sum_of<S>(acc[i][j], r);
      if (inside < 32 * MI) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * i + block_row(r, h) >= inside) x[i][r] = -INFINITY;
      }
      if (__any(mine >= 0)) {  // (hardly ever: a token's target is in one of many tiles)
        float at_target = 0.f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (mine == 32 * i + block_row(r, h)) at_target = x[i][r];
        if (mine >= 0 && mine < inside && (mine >> 2 & 1) == h) of_target[row] = at_target;
      }
      Sums a = {-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) a.m = fmaxf(a.m, x[i][r]);
      // +infinity and NaN (which fmaxf passes over) make s NaN
      const float m = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float d = x[i][r] - m, e = fast_exp2(d * LOG2E);
          a.s += e;
          a.t = fmaf(e, fmaxf(d, -1e4f), a.t);
        }
      __builtin_amdgcn_sched_barrier(0);
      a = join(a, {__shfl_xor(a.m, 32), __shfl_xor(a.s, 32), __shfl_xor(a.t, 32)});
      if (h == 0) shared[at.wave_m * S::BN + (at.wave_n * NI + j) * 32 + l] = make_float4(a.m, a.s, a.t, 0.f);
    }
    __syncthreads();
    const int64_t first = at.row - at.wave_n * NI * 32;
    for (int n = threadIdx.x; n < S::BN; n += 64 * S::WAVES) {
      if (first + n >= rows) continue;
      Sums a = {-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < S::WM; ++w) {
        const float4 v = shared[w * S::BN + n];
        a = w ? join(a, {v.x, v.y, v.z}) : Sums{v.x, v.y, v.z};
      }
      parts[(first + n) * tiles + at.tile_m] = make_float4(a.m, a.s, a.t, 0.f);
    }
  }
};

// A workgroup's threads have parts of a row's sums: the row's outputs.
__device__ __forceinline__ void finish_row(Sums a, float4* of_wave, int64_t row, const float* at_target, const int32_t* targets, int32_t vocab,
                                           float* logprob, float* lse, float* entropy) {
#pragma unroll
  for (int d = 32; d; d >>= 1) a = join(a, {__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)});
  if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = make_float4(a.m, a.s, a.t, 0.f);
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 4; ++w) a = join(a, {of_wave[w].x, of_wave[w].y, of_wave[w].z});
    const float log_s = logf(a.s), total = a.s == 0.f ? -INFINITY : a.m + log_s;
    if (lse) lse[row] = total;
    if (entropy) entropy[row] = a.s == 0.f ? 0.f : log_s - a.t / a.s;
    if (logprob) {
      const int32_t t = targets[row];
      float v = 0.f;
      if (t >= 0 && t < vocab) v = a.s == 0.f ? -INFINITY : (*at_target - a.m) - log_s;
      logprob[row] = v;
    }
  }
  __syncthreads();
}

// a workgroup per row and round (a wave per row: 10 us instead of 5 for 3 rows of 1172 tiles)
__global__ void __launch_bounds__(256) join_rows_kernel(const float4* parts, int32_t tiles, int64_t rows, const float* of_target,
                                                        const int32_t* targets, int32_t vocab, float* logprob, float* lse, float* entropy) {
  __shared__ float4 of_wave[4];
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const float4* const mine = parts + row * tiles;
    Sums a = {-INFINITY, 0.f, 0.f};
    for (int32_t i = threadIdx.x; i < tiles; i += 4 * 256) {
      float4 v[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = i + 256 * n < tiles ? mine[i + 256 * n] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
#pragma unroll
      for (int n = 0; n < 4; ++n) a = join(a, {v[n].x, v[n].y, v[n].z});
    }
    finish_row(a, of_wave, row, of_target + row, targets, vocab, logprob, lse, entropy);
  }
}

// Where a few tokens and a long width would leave CUs without work, the logits' contraction is cut: the logits come as parts in fp32,
// [parts][rows][stride], stride a multiple of 4 (69 rows, 8192 channels and 1119 tokens in fp32: 31 us, 151 in whole sums; 12 rows, 5120 and
// 2057 in bf16: 15, 27).  Four successive ones:
__device__ __forceinline__ void sum_parts(const float* parts, int32_t n_parts, int64_t rows, int64_t stride, int64_t row, int64_t c, float* x) {
  fetch4(parts + row * stride + c, x);
  for (int32_t p = 1; p < n_parts; ++p) {
    float v[4];
    fetch4(parts + (p * rows + row) * stride + c, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += v[e];
  }
}
__global__ void __launch_bounds__(256) rows_of_parts_kernel(const float* parts, int32_t n_parts, int64_t stride, int64_t rows, const int32_t* targets,
                                                            int32_t vocab, float* logprob, float* lse, float* entropy) {
  __shared__ float4 of_wave[4];
  __shared__ float at_target;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int32_t target = logprob ? targets[row] : -1;
    Sums a = {-INFINITY, 0.f, 0.f};
    for (int32_t c = 4 * threadIdx.x; c < vocab; c += 4 * 256) {
      float x[4];
      sum_parts(parts, n_parts, rows, stride, row, c, x);
      Sums b = {-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (c + e >= vocab) x[e] = -INFINITY;
        if (c + e == target) at_target = x[e];
        b.m = fmaxf(b.m, x[e]);
      }
      const float m = b.m == -INFINITY ? 0.f : b.m;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = x[e] - m, p = fast_exp2(d * LOG2E);
        b.s += p;
        b.t = fmaf(p, fmaxf(d, -1e4f), b.t);
      }
      a = join(a, b);
    }
    finish_row(a, of_wave, row, &at_target, targets, vocab, logprob, lse, entropy);
  }
}

// What a row's gradients take from it.
struct RowGradient {
  float L, some, g, ge, H;
  int32_t target;
  __device__ __forceinline__ RowGradient(int64_t row, const int32_t* targets, const float* lse, const float* entropy, const float* g_logprob,
                                         const float* g_entropy, int32_t vocab) {
    const int32_t t = targets ? targets[row] : -1;
    // (a row of nothing but -infinity: no probability anywhere)
    const float row_lse = lse[row];
    L = row_lse == -INFINITY ? 0.f : row_lse;
    some = row_lse == -INFINITY ? 0.f : 1.f;
    ge = g_entropy && some != 0.f ? g_entropy[row] : 0.f;
    H = g_entropy ? entropy[row] : 0.f;
    g = g_logprob ? g_logprob[row] : 0.f;
    if (t < 0 || t >= vocab || some == 0.f) g = 0.f;
    target = t < 0 ? -1 : t;
  }
  // of logit x, without what the target's has besides
  __device__ __forceinline__ float of(float x, bool with_entropy) const {
    const float lp = x - L, p = fast_exp2(lp * LOG2E) * some;
    return -p * (with_entropy && p > 0.f ? fmaf(ge, lp + H, g) : g);
  }
};

// the logits' gradients from parts of the logits, [rows][out_stride], zeros from vocab up to a multiple of 8
template <typename T>
__global__ void __launch_bounds__(256) gradients_of_parts_kernel(const float* parts, int32_t n_parts, int64_t stride, int64_t rows, const int32_t* targets,
                                                                 const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                                                                 int32_t vocab, T* out, int64_t out_stride) {
  const int64_t per = ((int64_t)vocab + 7) / 8 * 2, all = per * rows;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += gridDim.x * 256ll) {
    const int64_t row = i / per, c = (i - row * per) * 4;
    const RowGradient r(row, targets, lse, entropy, g_logprob, g_entropy, vocab);
    float x[4] = {0.f, 0.f, 0.f, 0.f}, v[4];
    if (c < stride) sum_parts(parts, n_parts, rows, stride, row, c, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = r.of(x[e], g_entropy != nullptr);
      if (c + e == r.target) v[e] += r.g;
      if (c + e >= vocab) v[e] = 0.f;
    }
    store4(out + row * out_stride + c, v);
  }
}

// the logits' gradients of a piece of the vocabulary, [rows][stride], zeros from vocab up to stride
template <typename T>
struct LogitGradients {
  const int32_t* targets;
  const float *lse, *entropy, *g_logprob, *g_entropy;
  T* out;
  int64_t stride, rows;
  int32_t first, vocab;  // of the piece, in it
  int32_t whole;         // tokens of the whole vocabulary
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char* smem) const {
    const int l = at.lane & 31, h = at.lane >> 5;
    const Turn<T, 32 * MI> turn(at, smem, S::TURN);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t first_row = at.row + 32 * j;
      asm volatile("" ::: "memory");  // (a block's rows are asked for when they are needed, not all at once)
      const int64_t row = first_row + l < rows ? first_row + l : rows - 1;
      const RowGradient of_row(row, targets, lse, entropy, g_logprob, g_entropy, whole);
      // the lane's target and the end of the piece, counted from the wave's first token
      const int64_t behind = (int64_t)of_row.target - first - at.feature, inside = vocab - at.feature;
      const int32_t mine = of_row.target < 0 || behind < 0 || behind >= 32 * MI ? -1 : (int32_t)behind;
      const bool any = __any(mine >= 0), edge = inside < 32 * MI;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = of_row.of(sum_of<S>(acc[i][j], 4 * q + e), g_entropy != nullptr);
          if (any) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (mine == 32 * i + 8 * q + 4 * h + e) v[e] += of_row.g;
          }
          if (edge) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (32 * i + 8 * q + 4 * h + e >= inside) v[e] = 0.f;
          }
          turn.put4(32 * i + 8 * q, v);
        }
      turn.store(rows - first_row, stride - at.feature, stride, [&](int r) { return out + (first_row + r) * stride + at.feature; });
    }
  }
};

// Both calls make a logit by the same sums (HeadLogitsPlan).  Those of 64 x 64 tiles in fp32 that are not cut are in the order of k, as a plain
// product's are: the lse may come from one, and where a token has nearly all of the probability, 1 - p is as far off as the two orders are
// apart.  With a plain product's lse the gradients of 700 rows of 50021 tokens are off by 1.4e-6 of their norm, with the forward call's by
// 1.1e-6 (in four sums each: 2.5e-6 to 4.1e-6, and 7e-7).  For few rows plain products have other orders, and four sums are nearer with both.
template <>
constexpr bool IN_ORDER<RowSums> = true;
template <>
constexpr bool IN_ORDER<LogitGradients<float>> = true;

template <typename T>
hpd_operand operand(const void* p, int64_t stride, int64_t size) {
  return {{p, p}, stride * (int64_t)sizeof(T), (int32_t)size};
}

template <typename T>
hipError_t forward(const hpd_head_args& a, hipStream_t s) {
  const HeadForwardPlan<T> plan(a.n_rows, a.width, a.vocab);
  const int32_t tiles = (int32_t)plan.tiles;
  float4* const parts = (float4*)a.workspace;
  float* const of_target = (float*)(a.workspace + plan.of_target);
  const hpd_product_args g = {operand<T>(a.weight, a.weight_stride, a.vocab), operand<T>(a.hidden, a.hidden_stride, a.n_rows),
                              a.width, 1, 0, 0};
  const int32_t* const targets = a.logprob ? a.targets : nullptr;
  const dim3 a_row_each((uint32_t)std::min<int64_t>(a.n_rows, 1 << 20));
  if (plan.product.splits > 1) {
    float* const logits = (float*)a.workspace;
    const hipError_t e = launch_product<T, BY_ROWS, BY_ROWS, PLAIN>(plan.product, g, StorePart{logits, round4(a.vocab), a.n_rows, 0}, s);
    if (e != hipSuccess) return e;
    rows_of_parts_kernel<<<a_row_each, dim3(256), 0, s>>>(logits, plan.product.splits, round4(a.vocab), a.n_rows, targets, a.vocab, a.logprob, a.lse, a.entropy);
    return hipGetLastError();
  }
  const hipError_t e = launch_product<T, BY_ROWS, BY_ROWS, PLAIN>(plan.product, g, RowSums{targets, of_target, parts, a.vocab, tiles, a.n_rows}, s);
  if (e != hipSuccess) return e;
  join_rows_kernel<<<a_row_each, dim3(256), 0, s>>>(parts, tiles, a.n_rows, of_target, targets, a.vocab, a.logprob, a.lse, a.entropy);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const hpd_head_backward_args& a, hipStream_t s) {
  const int64_t N = a.n_rows, D = a.width;
  const HeadBackwardPlan<T> plan(N, a.width, a.vocab);
  const int64_t piece = plan.piece;
  T* const dx = (T*)a.workspace;
  float* const parts = (float*)(a.workspace + plan.parts);
  hipError_t e = hipSuccess;
  for (int64_t v0 = 0; v0 < a.vocab && e == hipSuccess; v0 += piece) {
    const int64_t n = std::min<int64_t>(piece, a.vocab - v0);
    const T* const w = (const T*)a.weight + v0 * a.weight_stride;
    if (N > 0) {
      const hpd_product_args g = {operand<T>(w, a.weight_stride, n), operand<T>(a.hidden, a.hidden_stride, N), (int32_t)D, 1, 0, 0};
      if (plan.logits.splits > 1) {
        const int64_t stride = round4(a.vocab), all = (n + 7) / 8 * 2 * N;
        e = launch_product<T, BY_ROWS, BY_ROWS, PLAIN>(plan.logits, g, StorePart{parts, stride, N, 0}, s);
        if (e != hipSuccess) return e;
        gradients_of_parts_kernel<T><<<dim3((uint32_t)std::min<int64_t>((all + 255) / 256, 1 << 16)), dim3(256), 0, s>>>(
            parts, plan.logits.splits, stride, N, a.targets, a.lse, a.entropy, a.g_logprob, a.g_entropy, a.vocab, dx, piece);
        e = hipGetLastError();
      } else {
        e = launch_product<T, BY_ROWS, BY_ROWS, PLAIN>(
            plan.logits, g,
            LogitGradients<T>{a.targets, a.lse, a.entropy, a.g_logprob, a.g_entropy, dx, piece, N, (int32_t)v0, (int32_t)n, a.vocab}, s);
      }
    }
    if (e == hipSuccess && a.d_hidden && N > 0) {
      const hpd_product_args g = {operand<T>(w, a.weight_stride, D), operand<T>(dx, piece, N), (int32_t)n, 1, 0, 0};
      e = launch_product<T, BY_COLUMNS, BY_ROWS, TAIL>(plan.d_hidden, g, StorePart{parts, D, N, v0 > 0}, s);
    }
    if (e == hipSuccess && a.d_weight) {  // (no rows: zeros)
      const hpd_product_args g = {operand<T>(a.hidden, a.hidden_stride, D), operand<T>(dx, piece, n), (int32_t)N, 1, 0, 0};
      const StoreProduct<T> store = {{(T*)a.d_weight + v0 * a.d_weight_stride, nullptr}, {a.d_weight_stride, 0}, n, D, n};
      e = launch_product<T, BY_COLUMNS, BY_COLUMNS, PLAIN>(plan.d_weight, g, store, s);
    }
  }
  if (e == hipSuccess && a.d_hidden && N > 0) e = join_parts(parts, plan.d_hidden.splits, D, N, (T*)a.d_hidden, a.d_hidden_stride, s);
  return e;
}

}  // namespace

int64_t hpd_head_forward_bytes(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab) {
  return dtype == HPD_F32 ? HeadForwardPlan<float>(n_rows, width, vocab).bytes : HeadForwardPlan<hpd::bf16_t>(n_rows, width, vocab).bytes;
}
int64_t hpd_head_backward_bytes(int32_t dtype, int64_t n_rows, int32_t width, int32_t vocab) {
  return dtype == HPD_F32 ? HeadBackwardPlan<float>(n_rows, width, vocab).bytes : HeadBackwardPlan<hpd::bf16_t>(n_rows, width, vocab).bytes;
}
hipError_t hpd_launch_head(const hpd_head_args& a, hipStream_t s) {
  return a.dtype == HPD_F32 ? forward<float>(a, s) : forward<hpd::bf16_t>(a, s);
}
hipError_t hpd_launch_head_backward(const hpd_head_backward_args& a, hipStream_t s) {
  return a.dtype == HPD_F32 ? backward<float>(a, s) : backward<hpd::bf16_t>(a, s);
}
