// Choice of experts (dpc_gate) and its gradient (dpc_gate_bwd).
//
// A token's scores stand in the registers of LANES lanes, EPL neighbouring
// experts in each; a wavefront holds 64 / LANES tokens and needs no other.
//
// The choice is that of float64 arithmetic, which costs an exponential of some 20
// instructions for every score.  So it is made in float32 first, whose error is
// bounded: where every two neighbours in the order of the best topk + 1 scores,
// and the groups at the border, are further apart than that, the float64 order is
// the same.  Where not, the wavefront does the token again in float64, one token after
// the other.  The weights are float64 arithmetic on the chosen.
//
// Bound by vector issue: 65,536 tokens of 256 bfloat16 scores, 8 of 256 chosen, from 4
// of 8 groups, 36 us where a copy of the bytes takes 8; without groups 30, with neither
// groups nor bias 22 (all float64: 88, a 16-lane float64 loop for the choice: 247).  One
// token 3.2 us.  The gradient: 331,776 tokens of 3 float32 scores 5.7 us (13 MB); 65,536
// of 256, 8 chosen, 50 to 58 in bfloat16 (a copy of the bytes 15) and 79 to 82 in float32
// (29), of 1,024 274 to 296 (57), of 64 18 to 22 (4): elements are loaded and stored one
// by one, and every slot is compared with all of a lane's experts.
//
// How many tokens float32 does not settle is up to the scores: under one in 100 of 256
// experts with a bias of normally distributed numbers, all of them where scores tie or
// all but tie, as without a bias in 16 bits and where sigmoids are near 1.  65,536
// tokens, us:
//   8 of 256, sigmoid, bias 0, logits of spread 1.5, 3, 5.4   float32 34 50 127, bfloat16 82 82 125
//   the same from 4 of 8 groups                               float32 40 56 152, bfloat16 95 95 153
//   16 of 1,024, softmax, spread 1.5; bias normal and 0       float32 167 254, bfloat16 191 490
//   all scores equal, float32, without and with a bias        3 experts 47 79, 16 80 110, 256 106 145
//                                       (scores that differ:  3 experts 8 8, 16 10 13, 256 38 55)
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "dpc.h"
#include "dpc_elem.h"
#include "dpc_internal.h"

namespace {

constexpr int64_t kMaxSlots = (int64_t)1 << 30;
constexpr int kBlock = 256;

struct Gate {
  int ntok, nexpert, topk, sigmoid, groups, per, keep, best, renorm;
  double scale;
  int lanes;      // lanes of a group, if a group is that many whole lanes (1, 2, 4, ...), else 0
  float inverse;  // 1 / per
  // e / per: (e + 1/2) / per is 1/2 / per or more from a whole number, a thousand
  // times what float32 is off by.  (Experts that do not exist are given one, too.)
  __device__ __forceinline__ int group_of(int e) const { return (int)(((float)e + 0.5f) * inverse) & 63; }
};

// ---------------------------------------------------------------------------
// across lanes
// ---------------------------------------------------------------------------
// v of this lane and of the one that step M (1, 2, 4, .. 32) of a reduction pairs
// it with, in any order: all lanes of a group of M hold the same, so that any lane
// of the other group will do.
struct Two {
  unsigned a, b;
};
template <int M>
__device__ __forceinline__ Two both(unsigned v) {
  if constexpr (M == 1) return {v, (unsigned)__builtin_amdgcn_update_dpp(v, v, 0xb1, 0xf, 0xf, false)};        // lanes 1 0 3 2
  else if constexpr (M == 2) return {v, (unsigned)__builtin_amdgcn_update_dpp(v, v, 0x4e, 0xf, 0xf, false)};   // 2 3 0 1
  else if constexpr (M == 4) return {v, (unsigned)__builtin_amdgcn_update_dpp(v, v, 0x141, 0xf, 0xf, false)};  // mirrored in 8
  else if constexpr (M == 8) return {v, (unsigned)__builtin_amdgcn_update_dpp(v, v, 0x140, 0xf, 0xf, false)};  // mirrored in 16
  else if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);  // rows 0 0 2 2 and 1 1 3 3
    return {r[0], r[1]};
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);  // the halves
    return {r[0], r[1]};
  }
}
template <int M, typename V>
__device__ __forceinline__ void both_of(V v, V* x, V* y) {
  unsigned u[sizeof(V) / 4], a[sizeof(V) / 4], b[sizeof(V) / 4];
  __builtin_memcpy(u, &v, sizeof(V));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(V) / 4); ++i) {
    const Two t = both<M>(u[i]);
    a[i] = t.a;
    b[i] = t.b;
  }
  __builtin_memcpy(x, a, sizeof(V));
  __builtin_memcpy(y, b, sizeof(V));
}
// f over LANES lanes, for all of them.
template <int LANES, int M = 1, typename V, typename F>
__device__ __forceinline__ V across(V v, F f) {
  if constexpr (M >= LANES) {
    return v;
  } else {
    V a, b;
    both_of<M>(v, &a, &b);
    return across<LANES, 2 * M>(f(a, b), f);
  }
}

// (numbers: a NaN gives way)
struct Larger {
  __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_fmaxf(a, b); }
  __device__ __forceinline__ double operator()(double a, double b) const { return __builtin_fmax(a, b); }
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; }
};
struct Smaller {
  __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_fminf(a, b); }
  __device__ __forceinline__ double operator()(double a, double b) const { return __builtin_fmin(a, b); }
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const { return a < b ? a : b; }
};
struct Sum {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
struct Or {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const { return a | b; }
};

// What this wavefront has written to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------
// exp(x) within an ulp or so: x = n ln 2 + r with |r| <= ln 2 / 2, the series of
// exp(r) up to r^13 (the rest is below 2^-57).
__device__ __forceinline__ double exp64(double x) {
  x = fmin(fmax(x, -1000.0), 1000.0);  // 0 and infinity beyond
  const double n = rint(x * 1.4426950408889634);
  double r = fma(n, -0.6931471805599453, x);  // ln 2 to 53 bits, and what is left of it
  r = fma(n, -2.3190468138462996e-17, r);
  double p = 1.0 / 6227020800.0;
  constexpr double c[] = {1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0,
                          1.0 / 5040.0,      1.0 / 720.0,      1.0 / 120.0,     1.0 / 24.0,     1.0 / 6.0,
                          0.5,               1.0,              1.0};
#pragma unroll
  for (int i = 0; i < 13; ++i) p = fma(p, r, c[i]);
  return ldexp(p, (int)n);
}
// 1 / x of a normal x: the hardware's estimate (14 bits or more) and three steps of
// Newton's, within an ulp.
__device__ __forceinline__ double inverse64(double x) {
  double r = __builtin_amdgcn_rcp(x);
  r = fma(r, fma(-x, r, 1.0), r);
  r = fma(r, fma(-x, r, 1.0), r);
  return fma(r, fma(-x, r, 1.0), r);
}
__device__ __forceinline__ double sigmoid64(double z) {
  return z < -700.0 ? exp64(z) : inverse64(1.0 + exp64(-z));  // below, 1 + exp(-z) is exp(-z)
}

// The same in float32 by the hardware's exponential and reciprocal.
__device__ __forceinline__ float exp32(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float sigmoid32(float z) { return __builtin_amdgcn_rcpf(1.0f + exp32(-z)); }

// How far a float32 score may be from its exact value.  2^-24 is a rounding.
// Sigmoid: the exponential is off by 1.3 |z| + 2 roundings of itself (its argument's
// and its own), which s (1 - s) makes 0.3 + 0.5 of an absolute one, and the sum and
// the reciprocal add 3 of s: under 4 of them.  Softmax: exponentials off by 2.3 |z -
// top| + 2 roundings and a sum of up to 1,024 of them (16 in a lane, 6 steps across),
// which come to s (2.3 |z - top| + 2.3 sum s |z - top| + 28); s |z - top| <= 0.37, and
// s sum s |z - top| <= 2 for up to 1,024 experts: under 34 of them.  Nearly twice that
// is allowed for; c = s + bias adds one rounding of c, and a key without its last bits
// EPL 2^-23 of it.
__device__ __forceinline__ float score_off_by(bool sigmoid) { return sigmoid ? 0x1p-21f : 0x1p-18f; }
template <int EPL>
__device__ __forceinline__ float off_by(bool sigmoid, float c) {
  return score_off_by(sigmoid) + (EPL + 1) * 0x1p-23f * __builtin_fabsf(c);
}

// A key whose order as a whole number is the number's.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned u = __float_as_uint(v);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number(unsigned key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// LDS of a wavefront: chosen experts [tokens][topk], groups' values [tokens][groups]
// as doubles, and, one after the other, values of groups that are no whole lanes
// ([tokens][nexpert], of the type that chooses), keys [EPL][64] and the values of one
// token as doubles.
__host__ __device__ constexpr size_t chosen_bytes(int tokens, const Gate& g) { return ((size_t)tokens * g.topk * 4 + 15) / 16 * 16; }
__host__ __device__ constexpr size_t group_bytes(int tokens, const Gate& g) {
  return g.groups > 1 ? ((size_t)tokens * g.groups * 8 + 15) / 16 * 16 : 0;
}
template <typename T>
__host__ __device__ constexpr size_t wave_bytes(int tokens, int epl, const Gate& g) {
  const size_t keys = (size_t)epl * 256, one = (size_t)g.nexpert * 8;  // keys: as many bytes as float32 values
  const size_t values = sizeof(T) == 8 ? tokens * one : keys > one ? keys : one;
  return chosen_bytes(tokens, g) + group_bytes(tokens, g) +
         (sizeof(T) == 8 && g.groups == 1 ? 0 : g.groups == 1 ? keys : (values + 15) / 16 * 16);
}

// Which groups stay (bit by bit).  Of a group that is whole lanes (g.lanes) each
// lane has its two best, first and second, -infinity where there is none; else c
// are the lane's values, -infinity where an expert cannot be chosen.  *near: two
// groups at the border are closer than what float32 can tell apart.
template <int LANES, int EPL, typename V>
__device__ __forceinline__ unsigned long long kept_groups(const Gate& g, V first, V second, const V (&c)[EPL], int lane,
                                                          V* values, V* group, bool* near) {
  const int e0 = lane * EPL;
  V size = (V)0;  // magnitudes of a group's best, largest of all groups
  auto put = [&](int q) __attribute__((always_inline)) {
    const bool two = g.best == 2 && second != -(V)INFINITY;
    group[q] = two ? first + second : first;
    if (first != -(V)INFINITY) size = Larger()(size, (V)(__builtin_fabs(first) + (two ? __builtin_fabs(second) : 0.0)));
  };
  auto take = [&](V v) __attribute__((always_inline)) {
    second = Larger()(second, Smaller()(v, first));
    first = Larger()(first, v);
  };
  // the two best of two pairs; all lanes of a group of `some` are here
  auto merge = [&](int some) __attribute__((always_inline)) {
    auto step = [&](auto m) __attribute__((always_inline)) {
      V f[2], n[2];
      both_of<decltype(m)::value>(first, f, f + 1);
      both_of<decltype(m)::value>(second, n, n + 1);
      second = Larger()(Larger()(n[0], n[1]), Smaller()(f[0], f[1]));
      first = Larger()(f[0], f[1]);
    };
    if constexpr (LANES > 1) { if (some > 1) step(std::integral_constant<int, 1>{}); }
    if constexpr (LANES > 2) { if (some > 2) step(std::integral_constant<int, 2>{}); }
    if constexpr (LANES > 4) { if (some > 4) step(std::integral_constant<int, 4>{}); }
    if constexpr (LANES > 8) { if (some > 8) step(std::integral_constant<int, 8>{}); }
    if constexpr (LANES > 16) { if (some > 16) step(std::integral_constant<int, 16>{}); }
  };
  if (g.lanes) {
    merge(g.lanes);
    if (!(lane & (g.lanes - 1)) && e0 < g.nexpert) put(g.group_of(e0));
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i < g.nexpert) values[e0 + i] = c[i];
    wave_sync();
    // as many lanes to a group as there are
    int some = 1;
    while (some * 2 * g.groups <= LANES) some *= 2;
    const int part = lane & (some - 1);
    for (int q = lane / some; q < g.groups; q += LANES / some) {
      first = second = -(V)INFINITY;
      for (int i = part; i < g.per; i += some) take(values[q * g.per + i]);
      merge(some);
      if (part == 0) put(q);
    }
  }
  wave_sync();
  unsigned long long kept = 0;
  V low = (V)INFINITY, high = -(V)INFINITY;  // least of those kept, largest of the others
  for (int q = lane; q < g.groups; q += LANES) {
    const V v = group[q];
    int before = 0;
    for (int o = 0; o < g.groups; ++o) before += group[o] > v || (group[o] == v && o < q);
    if (v == -(V)INFINITY) continue;
    if (before < g.keep) {
      kept |= 1ull << q;
      low = Smaller()(low, v);
    } else {
      high = Larger()(high, v);
    }
  }
  wave_sync();  // read before the next writes
  kept = across<LANES>(kept, Or());
  if constexpr (sizeof(V) == 4) {
    low = across<LANES>(low, Smaller());
    high = across<LANES>(high, Larger());
    size = across<LANES>(size, Larger());
    // a value is off by its terms' errors, what their keys have lost and a rounding
    *near = high != -(V)INFINITY && !(low - high > 4 * score_off_by(g.sigmoid) + (EPL + 4) * 0x1p-22f * size);
  }
  return kept;
}

// -infinity for the experts of the groups that do not stay.
template <int EPL, typename V>
__device__ __forceinline__ void drop(const Gate& g, unsigned long long kept, int e0, V (&c)[EPL]) {
  if (g.lanes) {
    const bool stays = kept >> g.group_of(e0) & 1;
#pragma unroll
    for (int i = 0; i < EPL; ++i) c[i] = stays ? c[i] : -(V)INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (!(kept >> g.group_of(e0 + i) & 1)) c[i] = -(V)INFINITY;
  }
}

// Whether float32 cannot tell the order of two neighbouring keys: equal but for the
// last bits, or (plain: exact numbers) closer than their errors.
template <int EPL>
__device__ __forceinline__ bool close(bool plain, bool sigmoid, unsigned high, unsigned low) {
  high &= ~(EPL - 1u);
  low &= ~(EPL - 1u);
  if (plain) return high == low;
  const float a = number(high), b = number(low);
  return !(a - b > off_by<EPL>(sigmoid, a) + off_by<EPL>(sigmoid, b));
}

// The choice in float64, one expert after the other.
template <int LANES, int EPL>
__device__ __forceinline__ void choose64(const Gate& g, double (&c)[EPL], int lane, double* values, double* group, int* chosen) {
  const int e0 = lane * EPL;
  if (g.groups > 1) {
    double first = -INFINITY, second = -INFINITY;
    if (g.lanes) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        second = Larger()(second, Smaller()(c[i], first));
        first = Larger()(first, c[i]);
      }
    }
    const unsigned long long kept = kept_groups<LANES>(g, first, second, c, lane, values, group, (bool*)nullptr);
    drop(g, kept, e0, c);
  }
  for (int j = 0; j < g.topk; ++j) {
    double top = -INFINITY;
    int at = INT32_MAX;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (c[i] > top) {
        top = c[i];
        at = e0 + i;
      }
    const double best = across<LANES>(top, Larger());
    at = across<LANES>(top == best ? at : INT32_MAX, Smaller());
    if (lane == 0) chosen[j] = at == INT32_MAX ? -1 : at;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i == at) c[i] = -INFINITY;
  }
}

// The same for one token by a whole wavefront, from its logits.
template <typename T, int EPL>
__device__ __forceinline__ void settle(Gate g, const T* pz, const float* bias, double* values, double* group, int* chosen) {
  const int lane = threadIdx.x & 63, e0 = lane * EPL;
  double c[EPL], top = 0.0, inverse = 1.0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) c[i] = e0 + i < g.nexpert ? (double)pz[e0 + i] : -INFINITY;
  if (bias || g.groups > 1) {
    if (!g.sigmoid) {
      top = c[0];
#pragma unroll
      for (int i = 1; i < EPL; ++i) top = Larger()(top, c[i]);
      top = across<64>(top, Larger());
      double sum = 0.0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) sum += exp64(c[i] - top);
      inverse = 1.0 / across<64>(sum, Sum());
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (c[i] != -INFINITY)
        c[i] = (g.sigmoid ? sigmoid64(c[i]) : exp64(c[i] - top) * inverse) + (bias ? (double)bias[e0 + i] : 0.0);
  }
  g.lanes = 0;
  choose64<64>(g, c, lane, values, group, chosen);
}

template <typename T, int LANES, int EPL>
__global__ __launch_bounds__(kBlock) void gate_kernel(Gate g, const T* __restrict__ logits, int64_t ldl,
                                                      const float* __restrict__ bias, int* __restrict__ expert,
                                                      typename ElemAcc<T>::type* __restrict__ weight) {
  typedef typename ElemAcc<T>::type A;
  extern __shared__ __attribute__((aligned(16))) char gate_lds[];
  constexpr int kTokens = 64 / LANES;
  const int lane = threadIdx.x % LANES, mine = (threadIdx.x & 63) / LANES;
  const int64_t t = (blockIdx.y * (int64_t)gridDim.x + blockIdx.x) * (kBlock / LANES) + threadIdx.x / LANES;
  const bool in = t < g.ntok;
  const int e0 = lane * EPL;
  char* lds = gate_lds + (threadIdx.x >> 6) * wave_bytes<T>(kTokens, EPL, g);
  int* chosen = reinterpret_cast<int*>(lds) + mine * g.topk;
  lds += chosen_bytes(kTokens, g);
  double* group = reinterpret_cast<double*>(lds) + mine * g.groups;
  lds += group_bytes(kTokens, g);
  unsigned* keys = reinterpret_cast<unsigned*>(lds);
  A* values = reinterpret_cast<A*>(lds) + mine * g.nexpert;
  const T* pz = logits + (in ? t : 0) * ldl;
  // with neither bias nor groups the order is that of the logits
  const bool plain = !bias && g.groups == 1;

  A z[EPL];
  float b[EPL];
  if (EPL * sizeof(T) >= 16 && e0 + EPL <= g.nexpert) {
    constexpr int VE = Chunk<T>::kElems;
#pragma unroll
    for (int i = 0; i < EPL; i += VE) {
      Chunk<T> ch;
      ch.load(pz + e0 + i);
#pragma unroll
      for (int k = 0; k < VE && i + k < EPL; ++k) z[i + k] = (A)ch.v[k];
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) z[i] = e0 + i < g.nexpert ? (A)pz[e0 + i] : -(A)INFINITY;
  }
  if (!bias) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) b[i] = 0.0f;
  } else if (e0 + EPL <= g.nexpert) {
    __builtin_memcpy(b, bias + e0, sizeof(b));
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) b[i] = e0 + i < g.nexpert ? bias[e0 + i] : 0.0f;
  }

  // A NaN, or in a softmax +infinity: no order.
  bool bad = false;
#pragma unroll
  for (int i = 0; i < EPL; ++i) bad |= __builtin_isunordered((float)z[i], b[i]);
  A top = (A)0;
  if (!g.sigmoid) {
    top = z[0];
#pragma unroll
    for (int i = 1; i < EPL; ++i) top = Larger()(top, z[i]);
    top = across<LANES>(top, Larger());
    bad |= top == (A)INFINITY;
    if (top == -(A)INFINITY) top = (A)0;
  }
  if (__any(bad)) bad = across<LANES>((int)bad, Or());

  bool unsure = sizeof(T) == 8;
  unsigned mine_key = 0;   // with fewer than LANES slots: the key of slot `lane`, and its expert
  int mine_expert = -1;
  if constexpr (sizeof(T) != 8) {
    unsigned key[EPL];
    constexpr unsigned kLow = EPL - 1;  // a key's last bits say which expert of the lane it is
    float c[EPL];
    if (!plain) {
      if (g.sigmoid) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) c[i] = sigmoid32(z[i]);
      } else {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          c[i] = exp32(z[i] - top);
          sum += c[i];
        }
        sum = across<LANES>(sum, Sum());
        const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int i = 0; i < EPL; ++i) c[i] *= inverse;
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) c[i] = z[i] == -INFINITY ? -INFINITY : c[i] + b[i];
      if (g.groups > 1 && !g.lanes) {
        const unsigned long long kept = kept_groups<LANES>(g, 0.0f, 0.0f, c, lane, values, reinterpret_cast<float*>(group), &unsure);
        drop(g, kept, e0, c);
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i) c[i] = z[i] + 0.0f;  // -0 to 0
    }
    // 16-bit logits and the expert's number fit one key together: no two are equal
    const bool whole = sizeof(T) == 2 && plain;
    if (whole) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        unsigned u = 0;
        if constexpr (sizeof(T) == 2) {
          const T v = (T)c[i];
          unsigned short h;
          __builtin_memcpy(&h, &v, 2);
          u = h & 0x8000u ? (unsigned)(unsigned short)~h : h | 0x8000u;
        }
        key[i] = u << 16 | (0xffffu - (unsigned)(e0 + i));
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i) key[i] = (ordered(c[i]) & ~kLow) | (kLow - (unsigned)i);
    }
    // keys up to this are those of -infinity
    const unsigned none = whole && std::is_same_v<T, _Float16> ? 0x03ffffffu : 0x007fffffu;
    // each lane's keys in descending order (exchanges of an odd-even merge sort)
#pragma unroll
    for (int p = 1; p < EPL; p *= 2)
#pragma unroll
      for (int k = p; k >= 1; k /= 2)
#pragma unroll
        for (int j = k % p; j + k < EPL; j += 2 * k)
#pragma unroll
          for (int i = 0; i < k; ++i)
            if (i + j + k < EPL && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
              const unsigned x = key[i + j], y = key[i + j + k];
              key[i + j] = max(x, y);
              key[i + j + k] = min(x, y);
            }
    unsigned head = key[0];
    if (g.groups > 1 && g.lanes) {  // a lane's two best are its first two keys; all of it stays or none
      const float first = key[0] > none ? number(key[0] & ~kLow) : -INFINITY;
      const float second = key[1] > none ? number(key[1] & ~kLow) : -INFINITY;
      const unsigned long long kept = kept_groups<LANES>(g, first, second, c, lane, values, reinterpret_cast<float*>(group), &unsure);
      if (!(kept >> g.group_of(e0) & 1)) head = 0u;
    }
    // The others wait in LDS: key j + 1 of this lane in place j * 64 + lane, 0 behind
    // the last.  The largest of all heads is the next: its lane notes whose it is and
    // goes on to its next key.  Lane j keeps the j-th, if there are as many lanes.
    unsigned* next = keys + (threadIdx.x & 63);
#pragma unroll
    for (int i = 1; i < EPL; ++i) next[(i - 1) * 64] = key[i];
    next[(EPL - 1) * 64] = 0u;
    const bool few = g.topk < LANES;
    unsigned before = 0;
    int taken = 0, rounds = 0;
    for (int j = 0; j <= g.topk; ++j) {
      const unsigned best = across<LANES>(head, Larger());
      if (few) {
        mine_key = lane == j ? best : mine_key;
      } else if (!whole) {
        unsure |= j > 0 && best > none && close<EPL>(plain, g.sigmoid, before, best);
        before = best;
      }
      if (j == g.topk) break;
      if (!few) {
        rounds += best > none;
        if (best <= none && lane == 0) chosen[j] = -1;
      }
      if (head == best && best > none) {
        chosen[j] = few ? e0 : whole ? (int)(0xffffu - (best & 0xffffu)) : e0 + (int)(kLow - (best & kLow));
        head = *next;
        next += 64;
        ++taken;
      }
    }
    if (few) {
      const bool live = lane < g.topk && mine_key > none;
      wave_sync();
      mine_expert = !live ? -1 : whole ? (int)(0xffffu - (mine_key & 0xffffu)) : chosen[lane] + (int)(kLow - (mine_key & kLow));
      if (!whole) {
        const unsigned after = (unsigned)__shfl_down((int)mine_key, 1);
        unsure |= lane < g.topk && after > none && close<EPL>(plain, g.sigmoid, mine_key, after);
        rounds = live;
      }
    }
    // equal ones in two lanes were taken at once
    if (!whole && LANES > 1) unsure |= across<LANES>(few ? taken - rounds : taken, Sum()) != (few ? 0 : rounds);
  }

  // Exactly, where that did not settle it: the whole wavefront does such tokens one
  // by one, 64 at worst (equal scores of up to 16 experts).  (All of the wavefront's
  // tokens at once takes as many registers as to cost the float32 code a third of its
  // wavefronts.)
  double inverse = 1.0;
  if (!g.sigmoid && (!g.renorm || (sizeof(T) == 8 && !plain))) {  // the sum of all exponentials counts
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) sum += exp64((double)z[i] - (double)top);
    sum = across<LANES>(sum, Sum());
    inverse = sum == 0.0 ? 0.0 : 1.0 / sum;
  }
  if constexpr (sizeof(T) == 8) {
    double c[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      c[i] = (double)z[i];
      if (!plain && z[i] != -(A)INFINITY)
        c[i] = (g.sigmoid ? sigmoid64((double)z[i]) : exp64((double)z[i] - (double)top) * inverse) + (double)b[i];
    }
    choose64<LANES>(g, c, lane, values, group, chosen);
  } else {
    unsigned long long left = __ballot(unsure && in && !bad);
    if (left) {
      constexpr int WIDE = LANES * EPL > 64 ? LANES * EPL / 64 : 1;
      wave_sync();  // keys have been read
      const int64_t t0 = t - mine;
      int* first_chosen = chosen - mine * g.topk;
      do {
        const int token = (__ffsll(left) - 1) / LANES;
        left &= ~((~0ull >> (64 - LANES)) << token * LANES);
        settle<T, WIDE>(g, logits + (t0 + token) * ldl, bias, reinterpret_cast<double*>(keys), group - mine * g.groups,
                        first_chosen + token * g.topk);
      } while (left);
      wave_sync();
      const bool again = across<LANES>((int)(unsure && in && !bad), Or());
      if (again && g.topk < LANES) mine_expert = lane < g.topk ? chosen[lane] : -1;
    }
  }
  wave_sync();
  const bool few = sizeof(T) != 8 && g.topk < LANES;

  // weights of the chosen, a slot to a lane (and further ones if there are more)
  auto score = [&](int e) __attribute__((always_inline)) {
    if (bad || !in || e < 0) return 0.0;
    const double v = (double)pz[e];
    return g.sigmoid ? sigmoid64(v) : exp64(v - (double)top) * inverse;
  };
  const int e1 = few ? mine_expert : lane < g.topk ? chosen[lane] : -1;
  const double s1 = score(e1);
  double total = s1;
  for (int j = lane + LANES; j < g.topk; j += LANES) total += score(chosen[j]);
  total = across<LANES>(total, Sum());
  for (int j = lane; in && j < g.topk; j += LANES) {
    const int e = j == lane ? e1 : chosen[j];
    double w = j == lane ? s1 : score(e);
    if (g.renorm && total > 0.0) w = w / total;
    w *= g.scale;
    expert[t * g.topk + j] = bad ? j : e;
    weight[t * g.topk + j] = (A)(bad ? (double)NAN : w);
  }
}

// Scores s of a token's experts from its logits z, in the type of z.
template <int LANES, int EPL, typename A>
__device__ __forceinline__ void scores(const Gate& g, const A (&z)[EPL], A (&s)[EPL]) {
  if (g.sigmoid) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) s[i] = (A)1 / ((A)1 + exp(-z[i]));
    return;
  }
  A top = -(A)INFINITY;
#pragma unroll
  for (int i = 0; i < EPL; ++i) top = fmax(top, z[i]);
  top = across<LANES>(top, Larger());
  if (top == -(A)INFINITY) top = (A)0;  // all closed: every exponential is 0
  A sum = (A)0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    s[i] = exp(z[i] - top);
    sum += s[i];
  }
  sum = across<LANES>(sum, Sum());
  if (sum == (A)0) sum = (A)1;
#pragma unroll
  for (int i = 0; i < EPL; ++i) s[i] /= sum;
}

template <typename T, int LANES, int EPL>
__global__ __launch_bounds__(kBlock) void gate_bwd_kernel(Gate g, const T* __restrict__ logits, int64_t ldl,
                                                          const int* __restrict__ expert,
                                                          const typename ElemAcc<T>::type* __restrict__ dweight,
                                                          T* __restrict__ dlogits, int64_t lddl) {
  typedef typename ElemAcc<T>::type A;
  constexpr int kTokens = kBlock / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t t = (blockIdx.y * (int64_t)gridDim.x + blockIdx.x) * kTokens + threadIdx.x / LANES;
  const bool in = t < g.ntok;
  const int e0 = lane * EPL;
  const T* pz = logits + (in ? t : 0) * ldl;
  A z[EPL], s[EPL], ds[EPL];
  int slots[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) z[i] = in && e0 + i < g.nexpert ? (A)pz[e0 + i] : -(A)INFINITY;
  bool bad = false;  // a NaN, or in a softmax +infinity
#pragma unroll
  for (int i = 0; i < EPL; ++i) bad |= __builtin_isunordered(z[i], z[i]) || (!g.sigmoid && z[i] == (A)INFINITY);
  bad = across<LANES>((int)bad, Or());
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    ds[i] = (A)0;
    slots[i] = 0;
  }
  for (int j = 0; in && j < g.topk; ++j) {
    const int e = expert[t * g.topk + j];
    const A d = dweight[t * g.topk + j];
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e == e0 + i && e < g.nexpert) {
        ds[i] += d;
        slots[i] += 1;
      }
  }
  scores<LANES>(g, z, s);
  A total = (A)0, dot = (A)0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    ds[i] *= (A)g.scale;
    if (!slots[i]) continue;
    total += (A)slots[i] * s[i];
    dot += ds[i] * s[i];
  }
  dot = across<LANES>(dot, Sum());
  A rest = dot;  // sum of ds s
  if (g.renorm) {
    total = across<LANES>(total, Sum());
    const bool tiny = total < (A)(sizeof(A) == 8 ? 0x1p-900 : 0x1p-100);
    if (__any(tiny)) {
      // Scores at the smallest numbers or below, as a bias or a group may choose
      // them: taken against the largest of theirs, since shares are all that counts.
      A top = -(A)INFINITY, high = -(A)INFINITY;  // of all and of the chosen
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        top = fmax(top, z[i]);
        if (slots[i]) high = fmax(high, z[i]);
      }
      if (!g.sigmoid) top = across<LANES>(top, Larger());
      high = across<LANES>(high, Larger());
      // exp(-745.13) is where float64 ends: below, and where none is open, the sum is 0
      const bool some = (g.sigmoid ? high : high - top) >= (A)-745.13;
      const A unit = exp(g.sigmoid ? high : (A)0);
      A sum = (A)0, part = (A)0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        if (!slots[i]) continue;
        if (tiny) s[i] = !some ? (A)0 : g.sigmoid ? (A)1 / (unit + exp(high - z[i])) : exp(z[i] - high);
        sum += (A)slots[i] * s[i];
        part += ds[i] * s[i];
      }
      sum = across<LANES>(sum, Sum());
      part = across<LANES>(part, Sum());
      total = tiny ? sum : total;
      dot = tiny ? part : dot;
    }
    const bool none = total == (A)0;
    const A mean = none ? (A)0 : dot / total;
    rest = (A)0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      ds[i] = none || !slots[i] ? (A)0 : (ds[i] - (A)slots[i] * mean) / total;
      if (slots[i]) rest += ds[i] * s[i];
    }
    rest = tiny ? (A)0 : across<LANES>(rest, Sum());  // 0 but for roundings
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    if (!in || e0 + i >= g.nexpert) continue;
    // 1 - sigmoid(z) is sigmoid(-z)
    A d = g.sigmoid ? ds[i] * s[i] * ((A)1 / ((A)1 + exp(z[i]))) : s[i] * (ds[i] - rest);
    if (bad) d = (A)NAN;
    if (z[i] == -(A)INFINITY) d = (A)0;
    dlogits[t * lddl + e0 + i] = (T)d;
  }
}

// Workgroups of `per` tokens; one dimension of a launch has under 2^32 threads.
dim3 grid_for(int ntok, int per) {
  const int64_t blocks = ((int64_t)ntok + per - 1) / per, wide = 1 << 22;
  return blocks <= wide ? dim3((unsigned)blocks) : dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide));
}

// Calls f<LANES, EPL> for the number of experts; EPL is 16 from 9 experts on, or 8.
template <int MOST, typename F>
void by_width(int nexpert, F f) {
  const auto go = [&](auto lanes, auto epl) { f(lanes, epl); };
  if (nexpert <= 4) return go(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
  if (nexpert <= 8) return go(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
  const std::integral_constant<int, MOST> epl;
  const int lanes = (nexpert + MOST - 1) / MOST;
  if (lanes <= 1) go(std::integral_constant<int, 1>{}, epl);
  else if (lanes <= 2) go(std::integral_constant<int, 2>{}, epl);
  else if (lanes <= 4) go(std::integral_constant<int, 4>{}, epl);
  else if (lanes <= 8) go(std::integral_constant<int, 8>{}, epl);
  else if (lanes <= 16) go(std::integral_constant<int, 16>{}, epl);
  else if (lanes <= 32) go(std::integral_constant<int, 32>{}, epl);
  else go(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
}

template <typename F>
int by_type(dpc_elem elem, F f) {
  (void)hipGetLastError();  // report only what this launch raises
  switch (elem) {
    case DPC_ELEM_F64: f(double{}); break;
    case DPC_ELEM_F32: f(float{}); break;
    case DPC_ELEM_F16: f(_Float16{}); break;
    default: f(__bf16{}); break;
  }
  return dpc_internal_launch_status();
}

int gate_args(dpc_elem elem, const dpc_gate_spec* s, int ntok, Gate* g) {
  if (!elem_ok(elem) || !s || ntok < 0 || s->nexpert < 1 || s->topk < 1 || s->groups < 1 || s->keep < 1 ||
      s->keep > s->groups || (s->best != 1 && s->best != 2) || (s->score != DPC_SCORE_SOFTMAX && s->score != DPC_SCORE_SIGMOID) ||
      !std::isfinite(s->scale))
    return DPC_EINVAL;
  if (s->nexpert > DPC_MAX_EXPERTS || s->topk > DPC_MAX_TOPK || s->groups > DPC_MAX_GATE_GROUPS ||
      (int64_t)ntok * s->topk > kMaxSlots)
    return DPC_ENOTSUP;
  if (s->nexpert % s->groups || s->topk > s->keep * (s->nexpert / s->groups)) return DPC_EINVAL;
  *g = Gate{ntok, s->nexpert, s->topk, s->score == DPC_SCORE_SIGMOID, s->groups, s->nexpert / s->groups, s->keep, s->best,
            s->renorm != 0, s->scale, 0, 1.0f / (float)(s->nexpert / s->groups)};
  return DPC_OK;
}

}  // namespace

extern "C" int dpc_gate(void* stream, dpc_elem elem, const dpc_gate_spec* spec, int ntok, const void* logits, int64_t ldl,
                        const float* bias, int* expert, void* weight) {
  Gate g;
  const int st = gate_args(elem, spec, ntok, &g);
  if (st != DPC_OK) return st;
  if (ntok == 0) return DPC_OK;
  const size_t ws = elem == DPC_ELEM_F64 ? 8 : 4;
  if (!logits || !expert || !weight || ldl < g.nexpert || !elem_aligned(logits, elem_size(elem)) || !elem_aligned(bias, 4) ||
      !elem_aligned(expert, 4) || !elem_aligned(weight, ws))
    return DPC_EINVAL;
  return by_type(elem, [&](auto tt) {
    typedef decltype(tt) T;
    by_width<16>(g.nexpert, [&](auto l, auto e) {
      constexpr int LANES = decltype(l)::value, EPL = decltype(e)::value, TOKENS = kBlock / LANES;
      Gate with = g;
      const int lanes = g.per / EPL;
      with.lanes = g.per % EPL == 0 && lanes <= LANES && (lanes & (lanes - 1)) == 0 ? lanes : 0;
      const size_t lds = wave_bytes<T>(64 / LANES, EPL, with) * (kBlock / 64);
      hipLaunchKernelGGL((gate_kernel<T, LANES, EPL>), grid_for(ntok, TOKENS), dim3(kBlock), lds,
                         static_cast<hipStream_t>(stream), with, (const T*)logits, ldl, bias, expert,
                         (typename ElemAcc<T>::type*)weight);
    });
  });
}

extern "C" int dpc_gate_bwd(void* stream, dpc_elem elem, const dpc_gate_spec* spec, int ntok, const void* logits, int64_t ldl,
                            const int* expert, const void* dweight, void* dlogits, int64_t lddl) {
  Gate g;
  const int st = gate_args(elem, spec, ntok, &g);
  if (st != DPC_OK) return st;
  if (ntok == 0) return DPC_OK;
  const size_t ws = elem == DPC_ELEM_F64 ? 8 : 4;
  if (!logits || !expert || !dweight || !dlogits || ldl < g.nexpert || lddl < g.nexpert ||
      !elem_aligned(logits, elem_size(elem)) || !elem_aligned(dlogits, elem_size(elem)) || !elem_aligned(expert, 4) ||
      !elem_aligned(dweight, ws))
    return DPC_EINVAL;
  return by_type(elem, [&](auto tt) {
    typedef decltype(tt) T;
    by_width<8>(g.nexpert, [&](auto l, auto e) {
      constexpr int LANES = decltype(l)::value, EPL = decltype(e)::value, TOKENS = kBlock / LANES;
      hipLaunchKernelGGL((gate_bwd_kernel<T, LANES, EPL>), grid_for(ntok, TOKENS), dim3(kBlock), 0,
                         static_cast<hipStream_t>(stream), g, (const T*)logits, ldl, expert,
                         (const typename ElemAcc<T>::type*)dweight, (T*)dlogits, lddl);
    });
  });
}
