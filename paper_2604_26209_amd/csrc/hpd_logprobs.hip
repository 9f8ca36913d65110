// Log probabilities of given tokens with entropy and the most likely alternatives, and their gradient.
//
// In log2 units, y = x log2(e), with a reference point k, s = sum 2^(y - k), t = sum 2^(y - k) (y - k):
//   lse = (k + log2 s) ln 2,  logprob = (y_target - k - log2 s) ln 2,  entropy = (log2 s - t / s) ln 2.
// One pass over the logits: every lane keeps (k, s, t) of its share; k is a whole number, the lane's maximum rounded up, so
// that y - k is one multiply-add and moving k by d is exact: t' = (t - d s) 2^-d, s' = s 2^-d.  Partial
// results are joined by the same rule.  A k beyond 2^24 would not be whole, and its rounding not small: k starts at -2^22, below
// which a logit counts nothing beside others, and where the largest logit of a wave's share is further from 0 than 2^21 (all
// tokens excluded by a finite value, or a diverged row), the wave goes over it again with the maximum itself as
// reference point, as a sum of two numbers (its cost: 256 x 32000 bf16 logits, half of every row excluded by -1e9: 26.5 -> 30 us;
// nothing where every share has an ordinary logit).  The pass is bound by the bytes of the logits without alternatives, by
// vector instructions with them: 6144 x 130013 bf16 logits, 290 us and 5.5 TB/s without (8.9 instructions a logit), with one
// alternative 294 us and 5.4 TB/s (11.5), with eight 4.6, twenty 4.1, fifty 3.6 TB/s (16, 19, 22 instructions, busy all the time).
//
// Alternatives: a wave keeps its 64 largest (value, index) keys, lane i the i-th.  A vector of logits
// costs one comparison of its maximum with the K-th; what passes is collected and sorted in, 64 at a time.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "hpd_attn_bf16.h"
#include "hpd_finetune.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.69314718055994530942f;
constexpr int UNROLL = 4;          // vectors in flight per lane
constexpr int64_t MAX_GRID = 1 << 20;

// 16 bytes at any address that the element type allows
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  struct __attribute__((packed, aligned(4))) Raw { uint32_t w[4]; };
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r.w[i]);
  }
  static __device__ __forceinline__ Raw pack(const float* f) {
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = __float_as_uint(f[i]);
    return r;
  }
};
template <>
struct Vec<hpd::bf16_t> {
  static constexpr int N = 8;
  struct __attribute__((packed, aligned(2))) Raw { uint32_t w[4]; };
  static __device__ __forceinline__ void unpack(const Raw& r, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(r.w[i] << 16);
      f[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw pack(const float* f) {
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = cvt_pk_bf16(f[2 * i], f[2 * i + 1]);
    return r;
  }
};

// ---- sums
constexpr float NARROW = 2097152.f;          // 2^21: largest logit, in magnitude, up to which a reference point is a whole number
constexpr float NARROW_START = -1048576.f;   // -2^22 / 4
constexpr float OVERFLOWING = -1.0e37f;      // below it y - k may not be finite
constexpr float LOWEST_REFERENCE = -1.25e38f;  // below x log2(e) / 4 of every finite logit
struct Sums {
  float m;      // largest logit
  float r, lo;  // reference point / 4 (finite for every finite logit): r + lo, lo = 0 for a whole number
  float s, t;
};
template <bool WIDE>
__device__ __forceinline__ Sums no_sums() { return {-INFINITY, WIDE ? LOWEST_REFERENCE : NARROW_START, 0.f, 0.f, 0.f}; }
// raises the reference point to 4 (r + lo) >= 4 (a.r + a.lo); narrow: lo and a.lo are 0
template <bool WIDE>
__device__ __forceinline__ void raise(Sums& a, float r, float lo) {
  const float d = fminf(4.f * (WIDE ? (r - a.r) + (lo - a.lo) : r - a.r), 1.0e4f), f = fast_exp2(-d);
  a.t = fmaf(-d, a.s, a.t) * f;
  a.s *= f;
  a.r = r;
  a.lo = lo;
}
// (what the largest logit of a wide share was does not matter any more)
template <bool WIDE>
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  if (a.s == 0.f) a.r = LOWEST_REFERENCE;  // (nothing there: its reference point says nothing)
  if (b.s == 0.f) b.r = LOWEST_REFERENCE;
  const bool first = WIDE && (a.r > b.r || (a.r == b.r && a.lo >= b.lo));
  const float r = WIDE ? (first ? a.r : b.r) : fmaxf(a.r, b.r), lo = WIDE ? (first ? a.lo : b.lo) : 0.f;
  raise<WIDE>(a, r, lo);
  raise<WIDE>(b, r, lo);
  return {WIDE ? a.m : fmaxf(a.m, b.m), r, lo, a.s + b.s, a.t + b.t};
}
template <bool WIDE>
__device__ __forceinline__ Sums join_wave(Sums a) {
#pragma unroll
  for (int d = 32; d; d >>= 1)
    a = join<WIDE>(a, {WIDE ? a.m : __shfl_xor(a.m, d), __shfl_xor(a.r, d), WIDE ? __shfl_xor(a.lo, d) : 0.f, __shfl_xor(a.s, d),
                       __shfl_xor(a.t, d)});
  return a;
}
// (y - k) / 4 of a logit, rounded by its own size however far y and k are from 0
__device__ __forceinline__ float quarter(float x, const Sums& a) { return fmaf(x, 0.25f * LOG2E, -a.r) - a.lo; }
// The logits of one vector.  -infinity counts nothing, NaN and +infinity make s NaN.  WIDE: for shares whose largest logit
// is beyond NARROW in magnitude.
template <int N, bool WIDE>
__device__ __forceinline__ void add_logits(Sums& a, const float* x, float m) {
  a.m = fmaxf(a.m, m);
  if constexpr (WIDE) {
    const float r = m * (0.25f * LOG2E), lo = fmaf(m, 0.25f * LOG2E, -r);
    if (r > a.r || (r == a.r && lo > a.lo)) raise<true>(a, r, lo);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = 4.f * quarter(x[i], a), e = fast_exp2(d);
      a.s += e;
      a.t = fmaf(e, fmaxf(d, -200.f), a.t);
    }
  } else {
    const float y = m * LOG2E;
    if (y > 4.f * a.r) raise<false>(a, 0.25f * ceilf(y), 0.f);
    float low = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) low = fminf(low, x[i]);
    const float k = 4.f * a.r;
    if (__any(low < OVERFLOWING)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = fmaf(x[i], LOG2E, -k), e = fast_exp2(d);
        a.s += e;
        a.t = fmaf(e, fmaxf(d, -200.f), a.t);  // (0 times -infinity)
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = fmaf(x[i], LOG2E, -k), e = fast_exp2(d);
        a.s += e;
        a.t = fmaf(e, d, a.t);
      }
    }
  }
}

// ---- keys: larger = larger logit, then lower index; 0 = none
__device__ __forceinline__ uint64_t make_key(float x, int32_t index) {
  x = x == x ? x + 0.f : -INFINITY;  // (-0 = +0)
  const uint32_t u = __float_as_uint(x);
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return ((uint64_t)o << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
// the value of lane (own ^ M), without the LDS unit
template <int M>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int lane) {
  auto dpp = [](uint32_t x, auto control) __attribute__((always_inline)) -> uint32_t {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(control)::value, 0xf, 0xf, true);
  };
  if constexpr (M == 1) return dpp(v, std::integral_constant<int, 0xB1>{});   // quad_perm 1 0 3 2
  if constexpr (M == 2) return dpp(v, std::integral_constant<int, 0x4E>{});   // quad_perm 2 3 0 1
  if constexpr (M == 4)                                                       // ^ 7 (half mirror), ^ 3 (quad_perm 3 2 1 0)
    return dpp(dpp(v, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1B>{});
  if constexpr (M == 8) return dpp(v, std::integral_constant<int, 0x128>{});  // rotation by 8 in rows of 16
  if constexpr (M == 16) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);  // rows 0 0 2 2, rows 1 1 3 3
    return lane & 16 ? p[0] : p[1];
  }
  if constexpr (M == 32) {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);  // lower halves, upper halves
    return lane & 32 ? p[0] : p[1];
  }
}
template <int M>
__device__ __forceinline__ uint64_t lane_xor(uint64_t k, int lane) {
  return ((uint64_t)lane_xor<M>((uint32_t)(k >> 32), lane) << 32) | lane_xor<M>((uint32_t)k, lane);
}
__device__ __forceinline__ uint64_t read_lane(uint64_t k, int from) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), from) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, from);
}
template <typename K>
__device__ __forceinline__ K larger(K a, K b) { return a > b ? a : b; }

// one stage of a bitonic network over the 64 lanes; UP: the lane bit that marks runs sorted upwards (64: none)
template <int M, int UP, typename K>
__device__ __forceinline__ K stage(K k, int lane) {
  const K o = lane_xor<M>(k, lane);
  const bool low = (lane & M) == 0, up = (lane & UP) != 0;
  return (k > o) == (low != up) ? k : o;
}
template <int N, int M, typename K>
__device__ __forceinline__ K stages(K k, int lane) {  // distances M, M / 2 .. 1 of runs of N
  k = stage<M, N>(k, lane);
  if constexpr (M > 1) k = stages<N, M / 2>(k, lane);
  return k;
}
// a bitonic sequence sorted downwards
template <typename K>
__device__ __forceinline__ K settle(K k, int lane) { return stages<64, 32>(k, lane); }
template <int N = 2, typename K>
__device__ __forceinline__ K sort_down(K k, int lane) {
  k = stages<N, N / 2>(k, lane);
  if constexpr (N < 64) k = sort_down<N * 2>(k, lane);
  return k;
}

// The K largest keys of what a wave has seen: the sorted list, and a buffer of candidates in LDS that is
// sorted into it when it is full.  Candidates are the keys above a bar that rises with what has been seen.
struct Top {
  uint64_t list = 0;  // lane i: the i-th largest
  uint64_t last = 0;  // what a candidate has to exceed, in every lane
  float bar = 0.f;    // its value, once there is one
  bool full = false;
  int count = 0;               // candidates in the buffer
  uint64_t* buffer = nullptr;  // BUFFER keys of this wave
  // (a wave's LDS accesses happen in order; what other lanes have written is behind the compiler's back)
  static __device__ __forceinline__ void order() { asm volatile("" ::: "memory"); }
  // sorts the last 64 candidates in, or what there is
  __device__ __forceinline__ void flush(int K, int lane) {
    const int n = min(count, 64);
    uint64_t* const from = buffer + count - n;
    order();
    const uint64_t c = sort_down(lane < n ? from[lane] : 0, lane);
    order();
    buffer[count - n + lane] = c;  // turned around through LDS: the list and the candidates are one bitonic sequence
    order();
    list = settle(larger(list, from[63 - lane]), lane);
    order();
    count -= n;
    const uint64_t k = read_lane(list, K - 1);
    if (k > last) last = k;
    if (k) {
      full = true;
      bar = key_value(last);
    }
  }
  // one candidate per lane; 0: none
  __device__ __forceinline__ void add(uint64_t key, int K, int lane) {
    const bool in = key > last;
    const uint64_t mask = __ballot(in);
    if (mask == 0) return;
    if (in) buffer[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = key;
    count += __popcll(mask);
  }
  // m: each lane's largest logit of what has been seen or comes next.  The K-th largest of the 64 is one that K logits reach.
  __device__ __forceinline__ void raise_bar(float m, int K, int lane) {
    uint32_t o = (uint32_t)(make_key(m, 0) >> 32);
    if (K == 1) {
      o = larger(o, lane_xor<1>(o, lane));
      o = larger(o, lane_xor<2>(o, lane));
      o = larger(o, lane_xor<4>(o, lane));
      o = larger(o, lane_xor<8>(o, lane));
      o = larger(o, lane_xor<16>(o, lane));
      o = larger(o, lane_xor<32>(o, lane));
    } else {
      o = sort_down(o, lane);
    }
    o = (uint32_t)__builtin_amdgcn_readlane((int)o, K - 1);
    const uint64_t k = ((uint64_t)o << 32) - 1;
    if (k > last) {
      last = k;
      bar = key_value((uint64_t)o << 32);
    }
    full = true;
  }
  // the largest of two sorted lists; other: in LDS
  __device__ __forceinline__ void merge(const uint64_t* other, int lane) { list = settle(larger(list, other[63 - lane]), lane); }
};

constexpr int BUFFER = 64 + 8 * 64 + 64;  // what a flush leaves, a vector of every lane, room for a flush to write 64
struct Shared {
  uint64_t keys[4][BUFFER];  // every wave's candidates, then its list
  Sums sums[4];
};

// results of a row, by one wave (y - k - log2 s: where all logits lie far from 0, log s is less than a step of lse)
__device__ __forceinline__ void finish(const hpd_logprobs_args& a, int64_t row, Sums s, uint64_t list, float x_target,
                                       bool has_target, int lane) {
  const bool none = s.s == 0.f;  // nothing but -infinity
  const float log_s = log2f(s.s);
  auto log_probability = [&](float x) { return none ? -INFINITY : fmaf(quarter(x, s), 4.f * LN2, -log_s * LN2); };
  if (lane == 0) {
    if (a.lse) a.lse[row] = none ? -INFINITY : fmaf(s.r, 4.f * LN2, fmaf(s.lo, 4.f * LN2, log_s * LN2));
    if (a.entropy) a.entropy[row] = none ? 0.f : (log_s - s.t / s.s) * LN2;
    if (a.targets && a.logprob) a.logprob[row] = has_target ? log_probability(x_target) : 0.f;
  }
  if (lane < a.top_k) {
    a.top_id[row * a.top_k + lane] = (int32_t)~(uint32_t)list;
    a.top_logprob[row * a.top_k + lane] = log_probability(key_value(list));
  }
}

// A row's given token and its logit, asked for ahead of the row: two reads one after the other.
template <typename T>
struct Target {
  bool has = false;
  float logit = 0.f;
  __device__ __forceinline__ Target(const hpd_logprobs_args& a, int64_t row, const T* x, bool wanted) {
    const int32_t t = wanted && a.targets ? a.targets[row] : -1;
    has = t >= 0 && t < a.vocab;
    if (has) logit = hpd::to_float(x[t]);
  }
};

// The piece [begin, end) of a row by WV waves, of which this is number w.
template <typename T, bool TOP, bool WIDE>
__device__ __forceinline__ void scan(const T* x, int32_t begin, int32_t end, int w, int WV, int K, int lane, Sums& sums, Top& top) {
  using V = Vec<T>;
  sums = no_sums<WIDE>();
  // one vector per lane, the first logit of which is number `index`; its logits first .. last - 1 count
  auto take = [&](const float* f, int32_t index, int first, int last) __attribute__((always_inline)) {
    float m = f[0];
#pragma unroll
    for (int e = 1; e < V::N; ++e) m = fmaxf(m, f[e]);
    add_logits<V::N, WIDE>(sums, f, m);
    if constexpr (TOP) {
      if (__any(!top.full || !(m < top.bar))) {  // (a vector of NaN too: its keys are those of -infinity)
#pragma unroll
        for (int e = 0; e < V::N; ++e) top.add(e >= first && e < last ? make_key(f[e], index + e) : 0, K, lane);
        while (top.count >= 64) top.flush(K, lane);
      }
    }
  };
  constexpr int32_t STEP = 64 * V::N, RUN = STEP * UNROLL;  // logits of a vector of all lanes, of a turn of the wave
  int32_t at = begin + w * RUN, turns = 0;
  for (; at + RUN <= end; at += WV * RUN, ++turns) {
    typename V::Raw r[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) r[u] = *reinterpret_cast<const typename V::Raw*>(x + at + u * STEP + lane * V::N);
    if constexpr (TOP) {
      if (turns == 0 || turns == 3) {  // (later the candidates themselves raise it, 64 at a time)
        float m = sums.m;
        if (turns == 0) {
#pragma unroll
          for (int u = 0; u < UNROLL; ++u) {
            float f[V::N];
            V::unpack(r[u], f);
#pragma unroll
            for (int e = 0; e < V::N; ++e) m = fmaxf(m, f[e]);
          }
        }
        top.raise_bar(m, K, lane);
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      float f[V::N];
      V::unpack(r[u], f);
      take(f, at + u * STEP + lane * V::N, 0, V::N);
    }
  }
  // The wave's part of a turn that the end cuts.  A lane whose vector is not whole takes the last N logits and leaves out
  // those that are not its own (a piece of fewer than N: one by one).
  if (at < end) {
    typename V::Raw r[UNROLL];
    auto first_of = [&](int u) __attribute__((always_inline)) -> int32_t {  // of the lane's own logits
      return at + u * STEP + lane * V::N;
    };
    auto from_of = [&](int u) __attribute__((always_inline)) -> int32_t { return max(min(first_of(u), end - V::N), begin); };
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (first_of(u) >= end) continue;
      if (end - begin >= V::N) {
        r[u] = *reinterpret_cast<const typename V::Raw*>(x + from_of(u));
      } else {
        T few[V::N] = {};
#pragma unroll
        for (int e = 0; e < V::N; ++e)
          if (begin + e < end) few[e] = x[begin + e];
        r[u] = __builtin_bit_cast(typename V::Raw, few);
      }
    }
    auto logits_of = [&](int u, float* f) __attribute__((always_inline)) {
      V::unpack(r[u], f);
#pragma unroll
      for (int e = 0; e < V::N; ++e)
        if (from_of(u) + e < first_of(u) || from_of(u) + e >= end) f[e] = -INFINITY;
    };
    if constexpr (TOP) {
      float m = sums.m;
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        float f[V::N];
        logits_of(u, f);
#pragma unroll
        for (int e = 0; e < V::N; ++e) m = fmaxf(m, f[e]);
      }
      top.raise_bar(m, K, lane);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (at + u * STEP >= end) break;
      float f[V::N];
      logits_of(u, f);
      take(f, from_of(u), first_of(u) - from_of(u), end - from_of(u));
    }
  }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(256) logprobs_kernel(hpd_logprobs_args a, int32_t parts, int32_t span, int32_t waves) {
  __shared__ Shared sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int K = a.top_k;
  const T* logits = reinterpret_cast<const T*>(a.logits);
  const int64_t per = 4 / waves, items = (a.n_rows * parts + per - 1) / per;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t piece = item * per + (waves == 1 ? wave : 0);
    if (waves == 1 && piece >= a.n_rows) continue;  // (a wave of its own: no barrier below)
    const int64_t row = piece / parts;
    const int32_t part = (int32_t)(piece % parts);
    const T* x = logits + row * a.row_stride;
    const int32_t begin = part * span, end = min(begin + span, a.vocab);
    Sums sums;
    Top top;
    top.buffer = sh.keys[wave];
    const Target<T> target(a, row, x, parts == 1);
    scan<T, TOP, false>(x, begin, end, waves == 1 ? 0 : wave, waves, K, lane, sums, top);
    sums = join_wave<false>(sums);
    if (fabsf(sums.m) > NARROW && sums.m != -INFINITY) {
      Top unused;
      scan<T, false, true>(x, begin, end, waves == 1 ? 0 : wave, waves, K, lane, sums, unused);
      sums = join_wave<true>(sums);
    }
    if constexpr (TOP) {
      while (top.count) top.flush(K, lane);
    }
    if (waves > 1) {
      if (TOP) sh.keys[wave][lane] = top.list;
      if (lane == 0) sh.sums[wave] = sums;
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w) {
          sums = join<true>(sums, sh.sums[w]);
          if (TOP) top.merge(sh.keys[w], lane);
        }
      }
    }
    if (wave == 0 || waves == 1) {
      if (parts == 1) {
        finish(a, row, sums, top.list, target.logit, target.has, lane);
      } else {
        float4* ws = reinterpret_cast<float4*>(a.workspace);
        if (lane == 0) ws[piece] = make_float4(sums.r, sums.lo, sums.s, sums.t);
        if (TOP && lane < K) reinterpret_cast<uint64_t*>(ws + a.n_rows * parts)[piece * K + lane] = top.list;
      }
    }
    if (waves > 1) __syncthreads();
  }
}

// joins the pieces of a row: four waves take every fourth list, the last one the sums as well
template <typename T, bool TOP>
__global__ void __launch_bounds__(256) logprobs_join_kernel(hpd_logprobs_args a, int32_t parts) {
  __shared__ Shared sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int K = a.top_k;
  const float4* ws = reinterpret_cast<const float4*>(a.workspace);
  const uint64_t* lists = reinterpret_cast<const uint64_t*>(ws + a.n_rows * parts);
  for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
    const Target<T> target(a, row, reinterpret_cast<const T*>(a.logits) + row * a.row_stride, wave == 0);
    Sums sums = no_sums<true>();
    if (wave == 3 && lane < parts) {
      const float4 p = ws[row * parts + lane];
      sums = {-INFINITY, p.x, p.y, p.z, p.w};
    }
    Top top;
    if constexpr (TOP) {  // sorted lists, four on their way at a time: the turned one and the wave's are one bitonic sequence
      for (int32_t piece = wave; piece < parts; piece += 16) {
        uint64_t other[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          other[u] = 63 - lane < K && piece + 4 * u < parts ? lists[(row * parts + piece + 4 * u) * K + 63 - lane] : 0;
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (piece + 4 * u < parts) top.list = settle(larger(top.list, other[u]), lane);
      }
      sh.keys[wave][lane] = top.list;
    }
    if (wave == 3) {
      sums = join_wave<true>(sums);
      if (lane == 0) sh.sums[0] = sums;
    }
    __syncthreads();
    if (wave == 0) {
      if constexpr (TOP) {
#pragma unroll
        for (int w = 1; w < 4; ++w) top.merge(sh.keys[w], lane);
      }
      finish(a, row, sh.sums[0], top.list, target.logit, target.has, lane);
    }
    __syncthreads();
  }
}

// d_c = g ([c = target] - p_c) - h p_c (log p_c + H), 4 vectors per lane and turn.  Bound by its bytes: 4096 x 32000 bf16
// logits 92 us, 5.7 TB/s; with the entropy term, 700 x 50021 fp32 ones 51 us, 5.5 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) logprobs_backward_kernel(hpd_logprobs_backward_args a, int32_t pieces) {
  using V = Vec<T>;
  constexpr int32_t RUN = 256 * V::N * UNROLL;
  for (int64_t item = blockIdx.x; item < a.n_rows * pieces; item += gridDim.x) {
    const int64_t row = item / pieces;
    const int32_t begin = (int32_t)(item % pieces) * RUN, end = min(begin + RUN, a.vocab);
    const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
    T* dx = reinterpret_cast<T*>(a.d_logits) + row * a.d_stride;
    const float lse = a.lse[row];
    const int32_t target = a.targets ? a.targets[row] : -1;
    const bool has = target >= 0 && target < a.vocab;
    const float g = a.g_logprob && has ? a.g_logprob[row] : 0.f, hg = a.g_entropy ? a.g_entropy[row] : 0.f;
    const float H = a.g_entropy ? a.entropy[row] : 0.f;
    const bool none = lse == -INFINITY;
    auto gradient = [&](float f, int32_t c) -> float {
      const float lp = f - lse, p = fast_exp2(lp * LOG2E);
      const float d = (c == target ? g : 0.f) - p * fmaf(hg, fmaxf(lp, -1.0e4f) + H, g);
      return none ? 0.f : d;
    };
    if (end - begin == RUN) {
      typename V::Raw r[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u)
        r[u] = *reinterpret_cast<const typename V::Raw*>(x + begin + (u * 256 + threadIdx.x) * V::N);
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int32_t c = begin + (u * 256 + threadIdx.x) * V::N;
        float f[V::N];
        V::unpack(r[u], f);
#pragma unroll
        for (int e = 0; e < V::N; ++e) f[e] = gradient(f[e], c + e);
        *reinterpret_cast<typename V::Raw*>(dx + c) = V::pack(f);
      }
    } else {
      for (int32_t c = begin + threadIdx.x * V::N; c < end; c += 256 * V::N) {
        if (c + V::N <= end) {
          float f[V::N];
          V::unpack(*reinterpret_cast<const typename V::Raw*>(x + c), f);
#pragma unroll
          for (int e = 0; e < V::N; ++e) f[e] = gradient(f[e], c + e);
          *reinterpret_cast<typename V::Raw*>(dx + c) = V::pack(f);
        } else {
          for (int32_t e = c; e < end; ++e) dx[e] = hpd::from_float<T>(gradient(hpd::to_float(x[e]), e));
        }
      }
    }
  }
}

template <typename T>
hipError_t launch(const hpd_logprobs_args& a, const hpd_logprobs_plan& p, hipStream_t s) {
  const int64_t per = 4 / p.waves, items = (a.n_rows * p.parts + per - 1) / per;
  const dim3 grid((unsigned)std::min(items, MAX_GRID));
  if (a.top_k) logprobs_kernel<T, true><<<grid, 256, 0, s>>>(a, p.parts, p.span, p.waves);
  else logprobs_kernel<T, false><<<grid, 256, 0, s>>>(a, p.parts, p.span, p.waves);
  if (p.parts > 1) {
    const dim3 rows((unsigned)std::min(a.n_rows, MAX_GRID));
    if (a.top_k) logprobs_join_kernel<T, true><<<rows, 256, 0, s>>>(a, p.parts);
    else logprobs_join_kernel<T, false><<<rows, 256, 0, s>>>(a, p.parts);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_backward(const hpd_logprobs_backward_args& a, hipStream_t s) {
  constexpr int32_t RUN = 256 * Vec<T>::N * UNROLL;
  const int32_t pieces = (a.vocab + RUN - 1) / RUN;
  logprobs_backward_kernel<T><<<dim3((unsigned)std::min(a.n_rows * pieces, MAX_GRID)), 256, 0, s>>>(a, pieces);
  return hipGetLastError();
}

}  // namespace

hpd_logprobs_plan hpd_plan_logprobs(int32_t dtype, int64_t n_rows, int32_t vocab) {
  const int32_t n = dtype == HPD_F32 ? 4 : 8, run = 64 * n * UNROLL;  // logits that a wave takes at once
  if (vocab <= 2 * run) return {1, vocab, 1};
  // pieces of at least one turn of four waves, at most 64 (one per lane of the joining wave)
  const int64_t want = std::min<int64_t>((1024 + n_rows - 1) / n_rows, std::min<int64_t>(64, (vocab + 4 * run - 1) / (4 * run)));
  if (want <= 1) return {1, vocab, 4};
  const int32_t span = (int32_t)(((vocab + want - 1) / want + run - 1) / run * run);
  return {(vocab + span - 1) / span, span, 4};
}

int64_t hpd_logprobs_bytes(int32_t dtype, int64_t n_rows, int32_t vocab, int32_t top_k) {
  const hpd_logprobs_plan p = hpd_plan_logprobs(dtype, n_rows, vocab);
  return p.parts == 1 ? 0 : n_rows * p.parts * (16 + 8 * (int64_t)top_k);
}

hipError_t hpd_launch_logprobs(int32_t dtype, const hpd_logprobs_args& a, hipStream_t s) {
  const hpd_logprobs_plan p = hpd_plan_logprobs(dtype, a.n_rows, a.vocab);
  return dtype == HPD_F32 ? launch<float>(a, p, s) : launch<hpd::bf16_t>(a, p, s);
}

hipError_t hpd_launch_logprobs_backward(int32_t dtype, const hpd_logprobs_backward_args& a, hipStream_t s) {
  return dtype == HPD_F32 ? launch_backward<float>(a, s) : launch_backward<hpd::bf16_t>(a, s);
}
