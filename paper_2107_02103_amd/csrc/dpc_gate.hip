// Choice of experts (dpc_gate) and its gradient (dpc_gate_bwd).
//
// A token's scores stand in the registers of LANES lanes, EPL neighbouring
// experts in each; a wavefront holds 64 / LANES tokens and needs no other.
//
// The choice is that of float64 arithmetic, which costs an exponential of some 20
// instructions for every score.  So it is made in float32 first, whose error is
// bounded: where every two neighbours in the order of the best topk + 1 scores,
// and the groups at the border, are further apart than that, the float64 order is
// the same.  Where not (a token in a hundred, or exact ties), the wavefront does
// it again in float64.  The weights are float64 arithmetic on the chosen scores.
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
};

// ---------------------------------------------------------------------------
// across lanes
// ---------------------------------------------------------------------------
// v of the lane that step M (1, 2, 4, .. 32) of a reduction pairs this one with:
// all lanes of a group of M hold the same, so that any lane of the other group will do.
template <int M>
__device__ __forceinline__ unsigned partner(unsigned v) {
  if constexpr (M == 1) return __builtin_amdgcn_update_dpp(v, v, 0xb1, 0xf, 0xf, false);        // lanes 1 0 3 2
  else if constexpr (M == 2) return __builtin_amdgcn_update_dpp(v, v, 0x4e, 0xf, 0xf, false);   // 2 3 0 1
  else if constexpr (M == 4) return __builtin_amdgcn_update_dpp(v, v, 0x141, 0xf, 0xf, false);  // mirrored in 8
  else if constexpr (M == 8) return __builtin_amdgcn_update_dpp(v, v, 0x140, 0xf, 0xf, false);  // mirrored in 16
  else return (unsigned)__shfl_xor((int)v, M);
}
template <int M, typename V>
__device__ __forceinline__ V partner_of(V v) {
  if constexpr (sizeof(V) == 4) {
    unsigned u;
    __builtin_memcpy(&u, &v, 4);
    u = partner<M>(u);
    __builtin_memcpy(&v, &u, 4);
  } else {
    unsigned u[2];
    __builtin_memcpy(u, &v, 8);
    u[0] = partner<M>(u[0]);
    u[1] = partner<M>(u[1]);
    __builtin_memcpy(&v, u, 8);
  }
  return v;
}
// f over LANES lanes, for all of them.
template <int LANES, int M = 1, typename V, typename F>
__device__ __forceinline__ V across(V v, F f) {
  if constexpr (M >= LANES) return v;
  else return across<LANES, 2 * M>(f(v, partner_of<M>(v)), f);
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
__device__ __forceinline__ double sigmoid64(double z) { return 1.0 / (1.0 + exp64(-z)); }

// The same in float32 by the hardware's exponential and reciprocal.
__device__ __forceinline__ float exp32(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float sigmoid32(float z) { return __builtin_amdgcn_rcpf(1.0f + exp32(-z)); }

// How far a float32 score may be from its exact value.  2^-24 is a rounding.
// Sigmoid: the exponential is off by |z| + 2 roundings of itself (its argument's and
// its own), which s (1 - s) makes 0.23 + 0.5 of an absolute one, and the sum and the
// reciprocal add 3 of s.  Softmax: exponentials off by |z - top| + 2 roundings and
// a sum of up to 1,024 of them (16 in a lane, 6 steps across), which come to s (|z -
// top| + sum s |z - top| + 28), and s |z - top| <= 0.37, s sum s |z - top| <= s ln
// (1,024 / s) + .. <= 3: under 32 of them.  Both under 2^-19; c = s + bias adds one
// rounding of c, a key without its last bits EPL 2^-23 of it: `most` is the largest
// magnitude among the token's c.
template <int EPL>
__device__ __forceinline__ float off_by(float most) { return 0x1p-19f + (EPL + 1) * 0x1p-23f * most; }

// A key whose order as a whole number is the number's.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float number(unsigned key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// LDS of a wavefront: chosen experts [tokens][topk], then for groups values
// [tokens][nexpert] and groups' values [tokens][groups], as doubles.
__host__ __device__ constexpr size_t chosen_bytes(int tokens, int topk) { return ((size_t)tokens * topk * 4 + 15) / 16 * 16; }
__host__ __device__ constexpr size_t wave_bytes(int tokens, const Gate& g) {
  return chosen_bytes(tokens, g.topk) + (g.groups > 1 ? (size_t)tokens * (g.nexpert + g.groups) * 8 : 0);
}

// Which groups stay (bit by bit) of values c, -infinity where an expert cannot be
// chosen; *near: two at the border are closer than what float32 can tell apart.
template <int LANES, int EPL, typename V>
__device__ __forceinline__ unsigned long long kept_groups(const Gate& g, const V (&c)[EPL], int lane, V* values, V off,
                                                          bool* near) {
  const int e0 = lane * EPL;
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (e0 + i < g.nexpert) values[e0 + i] = c[i];
  wave_sync();
  V* group = values + g.nexpert;
  // as many lanes to a group as there are
  int some = 1;
  while (some * 2 * g.groups <= LANES) some *= 2;
  const int part = lane & (some - 1);
  for (int q = lane / some; q < g.groups; q += LANES / some) {
    V first = -(V)INFINITY, second = -(V)INFINITY;
    for (int i = part; i < g.per; i += some) {
      const V v = values[q * g.per + i];
      second = Larger()(second, Smaller()(v, first));
      first = Larger()(first, v);
    }
    // (the lanes of a group are in this together; the two best of two pairs)
    auto merge = [&](V of, V os) {
      second = Larger()(Larger()(second, os), Smaller()(first, of));
      first = Larger()(first, of);
    };
    if constexpr (LANES > 1) { if (some > 1) merge(partner_of<1>(first), partner_of<1>(second)); }
    if constexpr (LANES > 2) { if (some > 2) merge(partner_of<2>(first), partner_of<2>(second)); }
    if constexpr (LANES > 4) { if (some > 4) merge(partner_of<4>(first), partner_of<4>(second)); }
    if constexpr (LANES > 8) { if (some > 8) merge(partner_of<8>(first), partner_of<8>(second)); }
    if constexpr (LANES > 16) { if (some > 16) merge(partner_of<16>(first), partner_of<16>(second)); }
    if (part == 0) group[q] = g.best == 2 && second != -(V)INFINITY ? first + second : first;
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
    *near = high != -(V)INFINITY && !(low - high > 8 * off);
  }
  return kept;
}

// The order in float64, one expert after the other.
template <int LANES, int EPL>
__device__ __forceinline__ void choose64(const Gate& g, double (&c)[EPL], int lane, int* chosen) {
  const int e0 = lane * EPL;
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
  char* lds = gate_lds + (threadIdx.x >> 6) * wave_bytes(kTokens, g);
  int* chosen = reinterpret_cast<int*>(lds) + mine * g.topk;
  double* values = reinterpret_cast<double*>(lds + chosen_bytes(kTokens, g.topk)) + (size_t)mine * (g.nexpert + g.groups);
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
      for (int k = 0; k < VE && i + k < EPL; ++k) z[i + k] = in ? (A)ch.v[k] : -(A)INFINITY;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) z[i] = in && e0 + i < g.nexpert ? (A)pz[e0 + i] : -(A)INFINITY;
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) b[i] = bias && e0 + i < g.nexpert ? bias[e0 + i] : 0.0f;

  // A NaN, or in a softmax +infinity: no order.  The sum of a finite number's
  // difference to itself is 0.
  int bad = 0;
  A top = -(A)INFINITY;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    bad |= z[i] != z[i] || b[i] != b[i] || (!g.sigmoid && z[i] == (A)INFINITY);
    top = Larger()(top, z[i]);
  }
  bad = across<LANES>(bad, Or());
  if (!g.sigmoid) {
    top = across<LANES>(top, Larger());
    if (top == -(A)INFINITY) top = (A)0;
  }

  bool unsure = sizeof(T) == 8;
  if constexpr (sizeof(T) != 8) {
    // keys: 0 for what cannot be chosen
    unsigned key[EPL];
    constexpr unsigned kLow = EPL - 1;  // a key's last bits say which expert of the lane it is
    float c[EPL], off = 0.0f;
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
      for (int i = 0; i < EPL; ++i) {
        c[i] = z[i] == -INFINITY ? -INFINITY : c[i] + b[i];
        if (c[i] != -INFINITY) off = Larger()(off, __builtin_fabsf(c[i]));
      }
      off = off_by<EPL>(across<LANES>(off, Larger()));
      if (g.groups > 1) {
        bool near = false;
        const unsigned long long kept = kept_groups<LANES>(g, c, lane, reinterpret_cast<float*>(values), off, &near);
        unsure = near;
#pragma unroll
        for (int i = 0; i < EPL; ++i)
          if (!(kept >> (min(e0 + i, g.nexpert - 1) / g.per) & 1)) c[i] = -INFINITY;
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
        unsigned u;
        if constexpr (sizeof(T) == 2) {
          const T v = (T)z[i];
          unsigned short h;
          __builtin_memcpy(&h, &v, 2);
          // +0 and -0 are equal
          u = h == 0x8000u ? 0x8000u : h & 0x8000u ? (unsigned)(unsigned short)~h : h | 0x8000u;
        }
        key[i] = c[i] == -INFINITY ? 0u : u << 16 | (0xffffu - (unsigned)(e0 + i));
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        key[i] = c[i] == -INFINITY ? 0u : (ordered(c[i]) & ~kLow) | (kLow - (unsigned)i);
    }
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
    // the largest of all heads is the next: its lane goes on to its next key
    unsigned before = 0;
    for (int j = 0; j <= g.topk; ++j) {
      const unsigned best = across<LANES>(key[0], Larger());
      if (!whole && j > 0) {
        // neighbours: equal but for the last bits, or closer than their errors
        const unsigned a = before & ~kLow, d = best & ~kLow;
        unsure |= best != 0 && (plain ? a == d : !(number(a) - number(d) > 4 * off));
      }
      if (j == g.topk) break;
      const bool hit = key[0] == best && best != 0;
      if (!whole && LANES > 1) {  // equal ones in two lanes
        const unsigned long long hits = __ballot(hit) >> (mine * LANES) & (~0ull >> (64 - LANES));
        unsure |= (hits & (hits - 1)) != 0;
      }
      if (hit) {
        chosen[j] = whole ? (int)(0xffffu - (best & 0xffffu)) : e0 + (int)(kLow - (best & kLow));
#pragma unroll
        for (int i = 0; i + 1 < EPL; ++i) key[i] = key[i + 1];
        key[EPL - 1] = 0u;
      } else if (best == 0 && lane == 0) {
        chosen[j] = -1;
      }
      before = best;
    }
  }

  // Exactly, where that did not settle it.
  const bool all = !g.sigmoid && !g.renorm;  // the sum of all exponentials counts
  double sum = 1.0;
  const bool again = __any(unsure && in && !bad);
  if (all || (again && !plain && !g.sigmoid)) {
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) sum += exp64((double)z[i] - (double)top);
    sum = across<LANES>(sum, Sum());
    if (sum == 0.0) sum = 1.0;
  }
  if (again) {
    double c[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      c[i] = (double)z[i];
      if (!plain && z[i] != -(A)INFINITY)
        c[i] = (g.sigmoid ? sigmoid64((double)z[i]) : exp64((double)z[i] - (double)top) / sum) + (double)b[i];
    }
    wave_sync();
    if (g.groups > 1) {
      const unsigned long long kept = kept_groups<LANES>(g, c, lane, values, 0.0, nullptr);
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (!(kept >> (min(e0 + i, g.nexpert - 1) / g.per) & 1)) c[i] = -INFINITY;
    }
    choose64<LANES>(g, c, lane, chosen);
  }
  wave_sync();

  // weights of the chosen, a slot to a lane
  double total = 0.0;
  for (int j = lane; j < g.topk; j += LANES) {
    const int e = chosen[j];
    if (e >= 0 && !bad && in) total += g.sigmoid ? sigmoid64((double)pz[e]) : exp64((double)pz[e] - (double)top) / sum;
  }
  total = across<LANES>(total, Sum());
  for (int j = lane; in && j < g.topk; j += LANES) {
    const int e = bad ? j : chosen[j];
    double w = 0.0;
    if (bad) {
      w = NAN;
    } else if (e >= 0) {
      const double s = g.sigmoid ? sigmoid64((double)pz[e]) : exp64((double)pz[e] - (double)top) / sum;
      w = g.scale * (g.renorm ? total > 0.0 ? s / total : 0.0 : s);
    }
    expert[t * g.topk + j] = e;
    weight[t * g.topk + j] = (A)w;
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
  scores<LANES>(g, z, s);
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
  A total = (A)0, dot = (A)0;
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (slots[i]) {
      total += (A)slots[i] * s[i];
      dot += ds[i] * s[i];
    }
  total = across<LANES>(total, Sum());
  dot = across<LANES>(dot, Sum());
  const A scale = (A)g.scale;
  A rest = scale * dot;  // sum of ds s
  if (g.renorm) {
    const A mean = total == (A)0 ? (A)0 : dot / total;
#pragma unroll
    for (int i = 0; i < EPL; ++i) ds[i] = total == (A)0 || !slots[i] ? (A)0 : scale * ((ds[i] - (A)slots[i] * mean) / total);
    rest = (A)0;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) ds[i] *= scale;
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    if (!in || e0 + i >= g.nexpert) continue;
    A d = g.sigmoid ? ds[i] * s[i] * ((A)1 - s[i]) : s[i] * (ds[i] - rest);
    if (z[i] == -(A)INFINITY) d = (A)0;
    dlogits[t * lddl + e0 + i] = (T)d;
  }
}

// Workgroups of `per` tokens; one dimension of a launch has under 2^32 threads.
dim3 grid_for(int ntok, int per) {
  const int64_t blocks = ((int64_t)ntok + per - 1) / per, wide = 1 << 22;
  return blocks <= wide ? dim3((unsigned)blocks) : dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide));
}

// Calls f<LANES, EPL> for the number of experts.
template <typename F>
void by_width(int nexpert, F f) {
  if (nexpert <= 4) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
  else if (nexpert <= 8) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
  else if (nexpert <= 16) f(std::integral_constant<int, 2>{}, std::integral_constant<int, 8>{});
  else if (nexpert <= 32) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
  else if (nexpert <= 64) f(std::integral_constant<int, 8>{}, std::integral_constant<int, 8>{});
  else if (nexpert <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
  else if (nexpert <= 256) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 8>{});
  else if (nexpert <= 512) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
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
            s->renorm != 0, s->scale};
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
    by_width(g.nexpert, [&](auto l, auto e) {
      constexpr int LANES = decltype(l)::value, EPL = decltype(e)::value, TOKENS = kBlock / LANES;
      const size_t lds = wave_bytes(64 / LANES, g) * (kBlock / 64);
      hipLaunchKernelGGL((gate_kernel<T, LANES, EPL>), grid_for(ntok, TOKENS), dim3(kBlock), lds,
                         static_cast<hipStream_t>(stream), g, (const T*)logits, ldl, bias, expert,
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
    by_width(g.nexpert, [&](auto l, auto e) {
      constexpr int LANES = decltype(l)::value, EPL = decltype(e)::value, TOKENS = kBlock / LANES;
      hipLaunchKernelGGL((gate_bwd_kernel<T, LANES, EPL>), grid_for(ntok, TOKENS), dim3(kBlock), 0,
                         static_cast<hipStream_t>(stream), g, (const T*)logits, ldl, expert,
                         (const typename ElemAcc<T>::type*)dweight, (T*)dlogits, lddl);
    });
  });
}
