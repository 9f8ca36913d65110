// The gated feed-forward block and its gradient:
//   g = x Wg^T, u = x Wu^T, h = act(g) u, out = h Wd^T
//   dh = dout Wd, dg = dh u act'(g), du = dh act(g)
//   dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x, dWd = dout^T h
// Forward: one kernel for both projections, activation and product (a tile has the same features of g and u by turns, in
// the same wave), one for the second product.  Backward: one for dh and what follows from it element by element (dg, du and, for
// dWd, h again), one for dx (one contraction over dg and du in turn), one for dWg and dWu together, one for dWd.
//
// What bounds it: many rows, the matrix units under the clock that their power leaves (bf16: 14903 rows, 4096 to 12288 and back, 3.9 ms,
// 1.15 PFLOP/s; gradients of 8191 rows 4.15 ms, 1.19; fp32: gradients of 1801 rows, 1152 to 4008, 0.85 ms, 0.118 PFLOP/s, 85 % of the matrix
// units' time in the largest product); few rows, the weights' bytes (a row 57 us, 5.3 TB/s); in between, a product in one round of
// workgroups (512 rows 175 us); small calls, three launches one after another (333 rows, 256 to 1000, fp32, 21 us).
#include "hpd_ffn.h"
#include "hpd_product.h"

namespace {

// exp(x) by the hardware's exp2: for fp32 with what x log2(e) loses in its rounding made good
template <typename T>
__device__ __forceinline__ float fast_exp(float x) {
  constexpr float L = 1.44269504088896340736f, L_LOW = 1.92596299112661746887e-8f, LN2 = 0.69314718055994530942f;
  const float y = x * L, e = fast_exp2(y);
  if (sizeof(T) == 2) return e;
  const float low = fmaf(x, L, -y) + x * L_LOW;
  // (0 and infinity stay as they are: where y itself is infinite, low is not a number)
  return e > 0.f && e < 3.0e38f ? fmaf(e * LN2, low, e) : e;
}

// act(g) and its derivative (1 / (1 + e) by the reciprocal instruction, good to a step; divisions, and the slope where it is not asked for,
// took 6 of 130 us from the first kernel of 512 rows, 4096 to 12288)
template <typename T, int ACT>
__device__ __forceinline__ void activation(float g, float& a, float& slope) {
  if constexpr (ACT == HPD_ACT_GELU) {
    const float c = sizeof(T) == 2 ? 0.5f + 0.5f * erff(g * 0.70710678118654752f) : 0.5f * erfcf(g * -0.70710678118654752f);
    a = g * c;
    slope = fmaf(g * 0.39894228040143268f, fast_exp<T>(-0.5f * g * g), c);
  } else {
    // silu: g / (1 + exp(-g)); gelu by tanh: g (1 + tanh w) / 2 = g / (1 + exp(-2 w)), w = sqrt(2 / pi) (g + 0.044715 g^3)
    // (the logistic function is 0 or 1 long before |g| = 30, and g^3 stays finite)
    const float c = fminf(fmaxf(g, -30.f), 30.f);
    const float w = ACT == HPD_ACT_SILU ? g : 1.5957691216057308f * c * fmaf(0.044715f * c, c, 1.f);
    const float s = __builtin_amdgcn_rcpf(1.f + fast_exp<T>(-w));
    a = g * s;
    const float dw = ACT == HPD_ACT_SILU ? 1.f : 1.5957691216057308f * fmaf(0.134145f * c, c, 1.f);
    slope = fmaf(a * (1.f - s), dw, s);
  }
}

template <typename T, int ACT>
struct Activate {
  T *h, *gate, *up;  // gate and up may be NULL
  int64_t inner, rows, gate_stride, up_stride;
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char* smem) const {
    const Turn<T, 16 * MI> turn(at, smem, S::TURN);
    const int64_t width = inner - at.feature;
    each<NI>([&](auto j) {
      const int64_t first = at.row + 32 * j, left = rows - first;
      auto put = [&](auto value) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = value([&]() { return sum_of<S>(acc[i][j], 4 * q + e); }, [&]() { return sum_of<S>(acc[i][j], 4 * q + e + 8); });
            turn.put4(16 * i + 8 * q, v);
          }
      };
      put([](auto g, auto u) {
        float a, slope;
        activation<T, ACT>(g(), a, slope);
        return a * u();
      });
      turn.store(left, width, inner, [&](int r) { return h + (first + r) * inner + at.feature; });
      if (gate) {
        put([](auto g, auto) { return g(); });
        turn.store(left, width, gate_stride, [&](int r) { return gate + (first + r) * gate_stride + at.feature; });
      }
      if (up) {
        put([](auto, auto u) { return u(); });
        turn.store(left, width, up_stride, [&](int r) { return up + (first + r) * up_stride + at.feature; });
      }
    });
  }
};

// From dh: dg and du next to each other, h if it is wanted.  g and u come through LDS, where dg and du take their places; two blocks
// at a time, so that both fit.
template <typename T, int ACT>
struct InnerGradients {
  const T *gate, *up;
  T *d_inner, *h;
  int64_t inner, rows, gate_stride, up_stride;
  template <typename S, int MI, int NI>
  __device__ __forceinline__ void operator()(floatx16 (&acc)[MI][NI], const Place& at, char* smem) const {
    constexpr int NB = MI < 2 ? 1 : 2, BYTES = NB * 32 * 32 * (int)sizeof(T);
    static_assert(2 * BYTES <= S::TURN, "g and u");
    using W = Turn<T, 32 * NB>;
    const W of_g(at, smem, S::TURN), of_u(at, smem, S::TURN, BYTES);
    each<NI>([&](auto j) {
      each<MI / NB>([&](auto half) {
        constexpr int i0 = half * NB;
        const int64_t first = at.row + 32 * j, left = rows - first, feature = at.feature + 32 * i0, width = inner - feature;
        const typename W::Rows g_rows = of_g.fetch(left, width, gate_stride, [&](int r) { return gate + (first + r) * gate_stride + feature; });
        const typename W::Rows u_rows = of_u.fetch(left, width, up_stride, [&](int r) { return up + (first + r) * up_stride + feature; });
        of_g.put(g_rows);
        of_u.put(u_rows);
        Four<T> kept[NB][4];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float g[4], u[4], v[4];
            fetch4(of_g.four(32 * i + 8 * q), g);
            fetch4(of_u.four(32 * i + 8 * q), u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float dh = sum_of<S>(acc[i0 + i][j], 4 * q + e);
              float a, slope;
              activation<T, ACT>(g[e], a, slope);
              g[e] = dh * u[e] * slope;
              v[e] = a * u[e];
              u[e] = dh * a;
            }
            of_g.put4(32 * i + 8 * q, g);
            of_u.put4(32 * i + 8 * q, u);
            kept[i][q] = pack4<T>(v);
          }
        of_g.store(left, width, 2 * inner, [&](int r) { return d_inner + (first + r) * 2 * inner + feature; });
        of_u.store(left, width, 2 * inner, [&](int r) { return d_inner + (first + r) * 2 * inner + inner + feature; });
        if (h) {
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<Four<T>*>(of_g.four(32 * i + 8 * q)) = kept[i][q];
          of_g.store(left, width, inner, [&](int r) { return h + (first + r) * inner + feature; });
        }
      });
    });
  }
};

template <typename T>
hpd_operand operand(const void* p, int64_t stride, int64_t size, const void* second = nullptr) {
  return {{p, second ? second : p}, stride * (int64_t)sizeof(T), (int32_t)size};
}

template <typename T, int ACT>
hipError_t forward(const hpd_ffn_forward_args& a, hipStream_t s) {
  const int64_t D = a.cfg.width, F = a.cfg.inner, N = a.n_rows;
  const FfnForwardPlan<T> plan(a.cfg, N);
  T* const h = (T*)a.workspace;
  const hpd_product_args in = {operand<T>(a.w_gate, a.st.w_gate, F, a.w_up), operand<T>(a.x, a.st.x, N), (int32_t)D, 1, 0, 0};
  const Activate<T, ACT> act = {h, (T*)a.gate, (T*)a.up, F, N, a.st.gate, a.st.up};
  const hipError_t e = launch_product<T, BY_ROWS, BY_ROWS, DUAL>(plan.in, in, act, s);
  if (e != hipSuccess) return e;
  const hpd_product_args down = {operand<T>(a.w_down, a.st.w_down, D), operand<T>(h, F, N), (int32_t)F, 1, 0, 0};
  return store_product<T, BY_ROWS, BY_ROWS>(plan.down, down, (float*)(a.workspace + plan.parts), (T*)a.out, a.st.out, s);
}

template <typename T, int ACT>
hipError_t backward(const hpd_ffn_backward_args& a, hipStream_t s) {
  const int64_t D = a.cfg.width, F = a.cfg.inner, N = a.n_rows;
  const FfnBackwardPlan<T> plan(a.cfg, N);
  T* const d_inner = (T*)a.workspace;
  T* const h = (T*)(a.workspace + plan.h);
  hipError_t e = hipSuccess;
  if (N > 0) {
    const hpd_product_args g = {operand<T>(a.w_down, a.st.w_down, F), operand<T>(a.d_out, a.st.d_out, N), (int32_t)D, 1, 0, 0};
    const InnerGradients<T, ACT> grad = {(const T*)a.gate, (const T*)a.up, d_inner, a.d_w_down ? h : nullptr, F, N, a.st.gate, a.st.up};
    e = launch_product<T, BY_COLUMNS, BY_ROWS, PLAIN>(plan.inner, g, grad, s);
  }
  if (e == hipSuccess && a.d_x && N > 0) {
    const hpd_product_args g = {operand<T>(a.w_gate, a.st.w_gate, D, a.w_up), operand<T>(d_inner, 2 * F, N, d_inner + F), (int32_t)F, 1, 0, 0};
    e = store_product<T, BY_COLUMNS, BY_ROWS, SEGMENTS>(plan.dx, g, (float*)(a.workspace + plan.parts), (T*)a.d_x, a.st.d_x, s);
  }
  if (e == hipSuccess && (a.d_w_gate || a.d_w_up)) {  // (no rows: zeros)
    // rows of the result: the gate's features, then the up projection's
    const int64_t skip = a.d_w_gate ? 0 : F, rows = (a.d_w_gate ? F : 0) + (a.d_w_up ? F : 0);
    const hpd_product_args g = {operand<T>(a.x, a.st.x, D), operand<T>(d_inner + skip, 2 * F, rows), (int32_t)N, 1, 0, 0};
    const StoreProduct<T> store = {{(T*)(skip ? a.d_w_up : a.d_w_gate), (T*)a.d_w_up},
                                   {skip ? a.st.d_w_up : a.st.d_w_gate, a.st.d_w_up}, F, D, rows};
    e = launch_product<T, BY_COLUMNS, BY_COLUMNS, PLAIN>(plan.in_weights, g, store, s);
  }
  if (e == hipSuccess && a.d_w_down) {
    const hpd_product_args g = {operand<T>(h, F, F), operand<T>(a.d_out, a.st.d_out, D), (int32_t)N, 1, 0, 0};
    const StoreProduct<T> store = {{(T*)a.d_w_down, nullptr}, {a.st.d_w_down, 0}, D, F, D};
    e = launch_product<T, BY_COLUMNS, BY_COLUMNS, PLAIN>(plan.down_weights, g, store, s);
  }
  return e;
}

}  // namespace

int64_t hpd_ffn_forward_bytes(const hpd_ffn_config& cfg, int64_t n_rows) {
  return cfg.dtype == HPD_F32 ? FfnForwardPlan<float>(cfg, n_rows).bytes : FfnForwardPlan<hpd::bf16_t>(cfg, n_rows).bytes;
}
int64_t hpd_ffn_backward_bytes(const hpd_ffn_config& cfg, int64_t n_rows) {
  return cfg.dtype == HPD_F32 ? FfnBackwardPlan<float>(cfg, n_rows).bytes : FfnBackwardPlan<hpd::bf16_t>(cfg, n_rows).bytes;
}

#define BY_TYPE(call)                                                                                              \
  (a.cfg.dtype == HPD_F32 ? (a.cfg.activation == HPD_ACT_SILU   ? call<float, HPD_ACT_SILU>(a, s)                  \
                             : a.cfg.activation == HPD_ACT_GELU ? call<float, HPD_ACT_GELU>(a, s)                  \
                                                                : call<float, HPD_ACT_GELU_TANH>(a, s))            \
                          : (a.cfg.activation == HPD_ACT_SILU   ? call<hpd::bf16_t, HPD_ACT_SILU>(a, s)            \
                             : a.cfg.activation == HPD_ACT_GELU ? call<hpd::bf16_t, HPD_ACT_GELU>(a, s)            \
                                                                : call<hpd::bf16_t, HPD_ACT_GELU_TANH>(a, s)))
hipError_t hpd_launch_ffn(const hpd_ffn_forward_args& a, hipStream_t s) { return BY_TYPE(forward); }
hipError_t hpd_launch_ffn_backward(const hpd_ffn_backward_args& a, hipStream_t s) { return BY_TYPE(backward); }
