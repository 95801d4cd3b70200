// Choice of experts (dpc_gate) and its gradient (dpc_gate_bwd).
//
// A token's scores stand in the registers of LANES lanes, EPL neighbouring
// experts in each; a wavefront holds 64 / LANES tokens.  Everything that decides
// a choice is float64.
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

template <int LANES, typename V, typename F>
__device__ __forceinline__ V across(V v, F f) {
#pragma unroll
  for (int m = LANES >> 1; m; m >>= 1) v = f(v, __shfl_xor(v, m));
  return v;
}

// Scores s of a token's experts from its logits z, in the type A of z.
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
  top = across<LANES>(top, [](A a, A b) { return fmax(a, b); });
  if (top == -(A)INFINITY) top = (A)0;  // all closed: every exponential is 0
  A sum = (A)0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    s[i] = exp(z[i] - top);
    sum += s[i];
  }
  sum = across<LANES>(sum, [](A a, A b) { return a + b; });
  if (sum == (A)0) sum = (A)1;
#pragma unroll
  for (int i = 0; i < EPL; ++i) s[i] /= sum;
}

template <typename T, int LANES, int EPL>
__global__ __launch_bounds__(kBlock) void gate_kernel(Gate g, const T* __restrict__ logits, int64_t ldl,
                                                      const float* __restrict__ bias, int* __restrict__ expert,
                                                      typename ElemAcc<T>::type* __restrict__ weight) {
  typedef typename ElemAcc<T>::type W;
  extern __shared__ double gate_lds[];
  constexpr int kTokens = kBlock / LANES;
  const int lane = threadIdx.x % LANES, mine = threadIdx.x / LANES;
  const int64_t t = (blockIdx.y * (int64_t)gridDim.x + blockIdx.x) * kTokens + mine;
  const bool in = t < g.ntok;
  const int e0 = lane * EPL;
  double* chosen = gate_lds + (size_t)mine * g.topk;              // scores of the chosen
  double* values = gate_lds + (size_t)kTokens * g.topk + (size_t)mine * (g.nexpert + g.groups);  // c, then groups
  const T* pz = logits + (in ? t : 0) * ldl;

  double s[EPL], c[EPL], z[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) z[i] = in && e0 + i < g.nexpert ? (double)pz[e0 + i] : -INFINITY;
  scores<LANES>(g, z, s);
  int bad = 0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    c[i] = s[i];
    if (bias && e0 + i < g.nexpert) c[i] += (double)bias[e0 + i];
    bad |= c[i] != c[i];
    if (z[i] == -INFINITY) c[i] = -INFINITY;
  }
  bad = across<LANES>(bad, [](int a, int b) { return a | b; });

  if (g.groups > 1) {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i < g.nexpert) values[e0 + i] = c[i];
    __syncthreads();
    double* group = values + g.nexpert;
    for (int q = lane; q < g.groups; q += LANES) {
      double first = -INFINITY, second = -INFINITY;
      for (int i = 0; i < g.per; ++i) {
        const double v = values[q * g.per + i];
        second = fmax(second, fmin(v, first));
        first = fmax(first, v);
      }
      group[q] = g.best == 2 && second != -INFINITY ? first + second : first;
    }
    __syncthreads();
    unsigned long long kept = 0;
    for (int q = lane; q < g.groups; q += LANES) {
      const double v = group[q];
      int before = 0;
      for (int o = 0; o < g.groups; ++o) before += group[o] > v || (group[o] == v && o < q);
      if (before < g.keep && v != -INFINITY) kept |= 1ull << q;
    }
    kept = across<LANES>(kept, [](unsigned long long a, unsigned long long b) { return a | b; });
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i < g.nexpert && !(kept >> ((e0 + i) / g.per) & 1)) c[i] = -INFINITY;
  }

  double total = 0.0;
  for (int j = 0; j < g.topk; ++j) {
    double top = -INFINITY, score = 0.0;
    int at = INT32_MAX;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (c[i] > top) {
        top = c[i];
        at = e0 + i;
        score = s[i];
      }
#pragma unroll
    for (int m = LANES >> 1; m; m >>= 1) {
      const double other = __shfl_xor(top, m), os = __shfl_xor(score, m);
      const int oa = __shfl_xor(at, m);
      if (other > top || (other == top && oa < at)) {
        top = other;
        at = oa;
        score = os;
      }
    }
    total += score;
    if (lane == 0) chosen[j] = score;
    if (in && lane == 0) expert[t * g.topk + j] = bad ? j : at == INT32_MAX ? -1 : at;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i == at) c[i] = -INFINITY;
  }
  __syncthreads();
  for (int j = lane; in && j < g.topk; j += LANES) {
    const double w = g.scale * (g.renorm ? total > 0.0 ? chosen[j] / total : 0.0 : chosen[j]);
    weight[t * g.topk + j] = (W)(bad ? (double)NAN : w);
  }
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
  const auto add = [](A a, A b) { return a + b; };
  total = across<LANES>(total, add);
  dot = across<LANES>(dot, add);
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
  else if (nexpert <= 32) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
  else if (nexpert <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
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
      const size_t lds = (size_t)TOKENS * (g.topk + (g.groups > 1 ? g.nexpert + g.groups : 0)) * sizeof(double);
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
