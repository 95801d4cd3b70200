// Tokens sorted by expert and back (the routing calls of dpc.h).
//
// Plan: a stable counting sort of nslot expert numbers.  With h[e][c] the
// number of slots of expert e in part c of the slots (parts in order), the
// row of a slot is
//   sum_{e' < e, c} h[e'][c] + sum_{c' < c} h[e][c'] + (slots of e before it in c).
// A part is what one wavefront walks, 64 slots at a time: lanes with the same
// expert find each other by one ballot per bit of the expert's number, and
// their rank is the number of such lanes below.  No atomics: the order is the
// same on every call.  Bound by latency: 3 us for a few slots, 12 to 16 us for
// 331,776 in three launches of 1,024 slots to a workgroup (with 4,096 31 us).
//
// Rows: the gather, the combine and its gradient move each row once and do
// one or two FMA per element, so they are bound by HBM bandwidth (or by the
// latency of two dependent loads, plan then row, for a few tokens).  A row is
// cut into 16-byte chunks, and the lanes of a wavefront take the chunks of one
// row, or of several rows if a row has fewer than 33.  The last chunk of a row
// whose width is no multiple of a chunk overlaps the one before it, so that
// odd widths run at the same loads.  65,536 tokens of 8 KiB to 4 experts each,
// 11% of the choices dropped: gather 524 us (2.7 GB by counters: 5.1 TB/s),
// combine 459 (2.5 GB: 5.4), gradient 917 (4.6 GB: 5.0); a copy of 2 GiB runs at
// 4.9 TB/s.  float64: 262,144 rows of 1,600 1,268, 1,240 and 1,896 us (5.3, 5.4, 5.3).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "dpc.h"
#include "dpc_elem.h"
#include "dpc_internal.h"

namespace {

constexpr int64_t kMaxSlots = (int64_t)1 << 30;
constexpr int kMaxWidth = INT32_MAX - 127;  // a lane's next element (64 on) and a width rounded up to chunks are ints

// ---------------------------------------------------------------------------
// plan
// ---------------------------------------------------------------------------
// Up to here one workgroup makes the whole plan.  With 64 experts, us: 4,096
// slots 9.4 so and 13.6 in three launches, 8,192 14.4 and 14.1, 16,384 24.3 and
// 14.1 (2 experts 6.9, 10.5; 9.5, 10.6; 14.8, 10.9).
constexpr int kOneBlockSlots = 8192;
constexpr int kPartSlots = 1024;       // slots of a workgroup beyond that, at least
constexpr int kMaxBlocks = 1024;
constexpr int kPlanWaves = 4;          // wavefronts of a workgroup of the three-launch plan

inline int plan_blocks(int64_t nslot) {
  const int64_t b = (nslot + kPartSlots - 1) / kPartSlots;
  return (int)(b < kMaxBlocks ? b : kMaxBlocks);
}
// slots of a workgroup: every wavefront gets whole groups of 64
inline int64_t plan_part(int64_t nslot, int blocks) {
  const int64_t unit = 64 * kPlanWaves;
  return ((nslot + blocks - 1) / blocks + unit - 1) / unit * unit;
}

// Walks slots [lo, hi) of one wavefront, 64 at a time in order, calling
// f(slot, expert, lanes of the same expert) for the lanes with a kept slot.
template <typename F>
__device__ __forceinline__ void walk(const int* __restrict__ expert, int64_t lo, int64_t hi, int nexpert, F f) {
  const int lane = threadIdx.x & 63;
  const int bits = nexpert > 1 ? 32 - __clz(nexpert - 1) : 0;
  for (int64_t s0 = lo; s0 < hi; s0 += 64) {
    const int64_t s = s0 + lane;
    const int e = s < hi ? expert[s] : -1;
    const bool kept = (unsigned)e < (unsigned)nexpert;
    unsigned long long same = __ballot(kept);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((e >> b) & 1);
      same &= (e >> b) & 1 ? set : ~set;
    }
    f(s, s < hi, e, kept, same);
  }
}

// Counts of the experts among the slots [lo, hi) of one wavefront, in LDS.
__device__ __forceinline__ void count(const int* expert, int64_t lo, int64_t hi, int nexpert, int* cnt) {
  const int lane = threadIdx.x & 63;
  walk(expert, lo, hi, nexpert, [&](int64_t, bool, int e, bool kept, unsigned long long same) {
    // the lowest lane of each expert adds for all of them: one lane per address
    if (kept && (same & ((1ull << lane) - 1)) == 0) cnt[e] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  });
}

// Rows of the slots [lo, hi) of one wavefront; next[e]: its next row of expert e.
__device__ __forceinline__ void place(const int* expert, int64_t lo, int64_t hi, int nexpert, int* next, int* rows,
                                      int* pos) {
  const int lane = threadIdx.x & 63;
  walk(expert, lo, hi, nexpert, [&](int64_t s, bool in, int e, bool kept, unsigned long long same) {
    const int before = __popcll(same & ((1ull << lane) - 1));
    const int first = kept ? next[e] : 0;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (kept) {
      if (before == 0) next[e] = first + __popcll(same);
      rows[first + before] = (int)s;
    }
    if (in) pos[s] = kept ? first + before : -1;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  });
}

// Exclusive prefix sums of v[0 .. n) in LDS by the whole workgroup, total
// returned; tmp holds one int per wavefront.
__device__ __forceinline__ int block_scan(int* v, int n, int* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int carry = 0;
  for (int i0 = 0; i0 < n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    const int mine = i < n ? v[i] : 0;
    int sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    if (lane == 63) tmp[wave] = sum;
    __syncthreads();
    int before = carry, all = carry;
    for (int w = 0; w < waves; ++w) {
      if (w < wave) before += tmp[w];
      all += tmp[w];
    }
    if (i < n) v[i] = before + sum - mine;
    carry = all;
    __syncthreads();
  }
  return carry;
}

// Few slots: one workgroup.  LDS: counts [waves][nexpert], totals [nexpert],
// one int per wavefront.
__global__ __launch_bounds__(1024) void plan_one_kernel(int nslot, int nexpert, const int* __restrict__ expert,
                                                        int* __restrict__ offsets, int* __restrict__ rows,
                                                        int* __restrict__ pos) {
  extern __shared__ int plan_lds[];
  const int waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int* cnt = plan_lds;
  int* tot = cnt + waves * nexpert;
  int* tmp = tot + nexpert;
  const int part = ((nslot + waves - 1) / waves + 63) & ~63;
  const int lo = wave * part < nslot ? wave * part : nslot;
  const int hi = lo + part < nslot ? lo + part : nslot;
  for (int i = threadIdx.x; i < waves * nexpert; i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  count(expert, lo, hi, nexpert, cnt + wave * nexpert);
  __syncthreads();
  for (int e = threadIdx.x; e < nexpert; e += blockDim.x) {
    int run = 0;
    for (int w = 0; w < waves; ++w) {
      const int c = cnt[w * nexpert + e];
      cnt[w * nexpert + e] = run;
      run += c;
    }
    tot[e] = run;
  }
  __syncthreads();
  const int kept = block_scan(tot, nexpert, tmp);
  for (int e = threadIdx.x; e < nexpert; e += blockDim.x) {
    const int first = tot[e];
    offsets[e] = first;
    for (int w = 0; w < waves; ++w) cnt[w * nexpert + e] += first;
  }
  if (threadIdx.x == 0) offsets[nexpert] = kept;
  for (int r = kept + threadIdx.x; r < nslot; r += blockDim.x) rows[r] = -1;
  __syncthreads();
  place(expert, lo, hi, nexpert, cnt + wave * nexpert, rows, pos);
}

// Many slots, first launch: hist[e][block] = slots of expert e in the block's part.
__global__ __launch_bounds__(64 * kPlanWaves) void plan_count_kernel(int64_t nslot, int64_t part, int nexpert,
                                                                     const int* __restrict__ expert,
                                                                     int* __restrict__ hist) {
  extern __shared__ int plan_lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int i = threadIdx.x; i < kPlanWaves * nexpert; i += blockDim.x) plan_lds[i] = 0;
  __syncthreads();
  const int64_t first = blockIdx.x * part + wave * (part / kPlanWaves);
  const int64_t lo = first < nslot ? first : nslot;
  const int64_t hi = lo + part / kPlanWaves < nslot ? lo + part / kPlanWaves : nslot;
  count(expert, lo, hi, nexpert, plan_lds + wave * nexpert);
  __syncthreads();
  for (int e = threadIdx.x; e < nexpert; e += blockDim.x) {
    int sum = 0;
    for (int w = 0; w < kPlanWaves; ++w) sum += plan_lds[w * nexpert + e];
    hist[(int64_t)e * gridDim.x + blockIdx.x] = sum;
  }
}

// Second launch, one workgroup per expert: hist[e] to its exclusive prefix
// sums over the blocks, total[e] to their sum.
__global__ __launch_bounds__(256) void plan_scan_kernel(int blocks, int* __restrict__ hist, int* __restrict__ total) {
  __shared__ int v[kMaxBlocks];
  __shared__ int tmp[4];
  int* h = hist + (int64_t)blockIdx.x * blocks;
  for (int i = threadIdx.x; i < blocks; i += blockDim.x) v[i] = h[i];
  __syncthreads();
  const int sum = block_scan(v, blocks, tmp);
  for (int i = threadIdx.x; i < blocks; i += blockDim.x) h[i] = v[i];
  if (threadIdx.x == 0) total[blockIdx.x] = sum;
}

// Third launch: rows and positions of the block's part.
__global__ __launch_bounds__(64 * kPlanWaves) void plan_place_kernel(int64_t nslot, int64_t part, int nexpert,
                                                                     const int* __restrict__ expert,
                                                                     const int* __restrict__ hist,
                                                                     const int* __restrict__ total,
                                                                     int* __restrict__ offsets, int* __restrict__ rows,
                                                                     int* __restrict__ pos) {
  extern __shared__ int plan_lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int* cnt = plan_lds;
  int* off = cnt + kPlanWaves * nexpert;
  int* tmp = off + nexpert;
  for (int i = threadIdx.x; i < kPlanWaves * nexpert; i += blockDim.x) cnt[i] = 0;
  for (int e = threadIdx.x; e < nexpert; e += blockDim.x) off[e] = total[e];
  __syncthreads();
  const int kept = block_scan(off, nexpert, tmp);
  const int64_t first = blockIdx.x * part + wave * (part / kPlanWaves);
  const int64_t lo = first < nslot ? first : nslot;
  const int64_t hi = lo + part / kPlanWaves < nslot ? lo + part / kPlanWaves : nslot;
  count(expert, lo, hi, nexpert, cnt + wave * nexpert);
  __syncthreads();
  for (int e = threadIdx.x; e < nexpert; e += blockDim.x) {
    int run = off[e] + hist[(int64_t)e * gridDim.x + blockIdx.x];
    for (int w = 0; w < kPlanWaves; ++w) {
      const int c = cnt[w * nexpert + e];
      cnt[w * nexpert + e] = run;
      run += c;
    }
    if (blockIdx.x == 0) offsets[e] = off[e];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) offsets[nexpert] = kept;
  for (int64_t r = kept + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; r < nslot; r += (int64_t)gridDim.x * blockDim.x)
    rows[r] = -1;
  __syncthreads();
  place(expert, lo, hi, nexpert, cnt + wave * nexpert, rows, pos);
}

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------
struct Shape {
  int64_t nslot;
  int ntok, topk, width;
  int lanes_log2;  // lanes of a row
};

// Rows of 192 MiB and more (with their addresses and strides multiples of 16
// bytes) are read and written past the caches: they would not be found there
// by the call that uses them next.  Gather, combine and its gradient in a row:
//   rows of 67 MB  68 us, past the caches 87;  105 MB 129 and 142;
//   rows of 268 MB 284 us, past the caches 253;  319 MB 410 and 393.
// Unaligned rows share cache lines between chunks (134 MB 146 us, 172).
constexpr int64_t kOnceBytes = (int64_t)192 << 20;

constexpr int kBlock = 256;

// weight times an element: a product in the type of sums, rounded to it before it
// is rounded to the element's type (one fused multiply would round once, and
// differ from what a caller gets from the two operations)
template <typename T>
__device__ __forceinline__ T times(typename ElemAcc<T>::type w, T v) {
  typename ElemAcc<T>::type p = w * (typename ElemAcc<T>::type)v;
  if constexpr (sizeof(T) == 2) asm("" : "+v"(p));  // the product is a value of its own
  return (T)p;
}

template <typename T, bool WEIGHT, bool ONCE>
__global__ __launch_bounds__(kBlock) void combine_kernel(Shape sh, const T* __restrict__ x, int64_t ldx,
                                                         const typename ElemAcc<T>::type* __restrict__ weight,
                                                         const int* __restrict__ pos, T* __restrict__ y, int64_t ldy) {
  typedef typename ElemAcc<T>::type A;
  constexpr int VE = Chunk<T>::kElems;
  const int lanes = 1 << sh.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int64_t groups = ((int64_t)gridDim.x * kBlock) >> sh.lanes_log2;
  const int nch = (sh.width + VE - 1) / VE;
  for (int64_t t = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh.lanes_log2; t < sh.ntok; t += groups) {
    const int* pt = pos + t * sh.topk;
    T* py = y + t * ldy;
    if (sh.width < VE) {
      for (int c = lane; c < sh.width; c += lanes) {
        A acc = (A)0;
        for (int j = 0; j < sh.topk; ++j) {
          const int r = pt[j];
          if ((unsigned)r >= (unsigned)sh.nslot) continue;
          const A v = (A)x[(int64_t)r * ldx + c];
          acc += WEIGHT ? weight[t * sh.topk + j] * v : v;
        }
        py[c] = (T)acc;
      }
      continue;
    }
    for (int c = lane; c < nch; c += lanes) {
      const int at = c * VE < sh.width - VE ? c * VE : sh.width - VE;
      A acc[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) acc[i] = (A)0;
      for (int j = 0; j < sh.topk; ++j) {
        const int r = pt[j];
        if ((unsigned)r >= (unsigned)sh.nslot) continue;
        Chunk<T> ch;
        const T* px = x + (int64_t)r * ldx + at;
        if (ONCE) ch.load_once(px);
        else ch.load(px);
        const A w = WEIGHT ? weight[t * sh.topk + j] : (A)1;
#pragma unroll
        for (int i = 0; i < VE; ++i) acc[i] += WEIGHT ? w * (A)ch.v[i] : (A)ch.v[i];
      }
      Chunk<T> out;
#pragma unroll
      for (int i = 0; i < VE; ++i) out.v[i] = (T)acc[i];
      if (ONCE) out.store_once(py + at);
      else out.store(py + at);
    }
  }
}

// Sends dy to the rows of its token (times their weights), and with DOT takes
// the dot product of each row with it.  Token by token, J of a token's rows at
// a time: a token's dy is read from memory once, whatever its number of rows.
template <typename T, bool WEIGHT, bool DOT, int J, bool ONCE>
__global__ __launch_bounds__(kBlock) void send_kernel(
    Shape sh, const T* __restrict__ x, int64_t ldx, const typename ElemAcc<T>::type* __restrict__ weight,
    const int* __restrict__ rows, const int* __restrict__ pos, const T* __restrict__ dy, int64_t lddy,
    T* __restrict__ dx, int64_t lddx, typename ElemAcc<T>::type* __restrict__ dweight) {
  typedef typename ElemAcc<T>::type A;
  constexpr int VE = Chunk<T>::kElems;
  const int lanes = 1 << sh.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int64_t groups = ((int64_t)gridDim.x * kBlock) >> sh.lanes_log2;
  const int nch = (sh.width + VE - 1) / VE;
  // whole wavefronts stay in the loop: the sums below are taken across lanes
  const int64_t rounds = (sh.ntok + groups - 1) / groups;
  int64_t t = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh.lanes_log2;
  for (int64_t i = 0; i < rounds; ++i, t += groups) {
    const bool in = t < sh.ntok;
    const T* pdy = dy + (in ? t : 0) * lddy;
    for (int j0 = 0; j0 < sh.topk; j0 += J) {
      const int64_t s0 = (in ? t : 0) * sh.topk + j0;
      int r[J];
      bool live[J], any = false;
      A w[J], dot[J];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const bool mine = in && j0 + j < sh.topk;
        r[j] = mine ? pos[s0 + j] : -1;
        live[j] = (unsigned)r[j] < (unsigned)sh.nslot;
        any |= live[j];
        w[j] = (A)1;
        if (WEIGHT) w[j] = live[j] ? weight[s0 + j] : (A)0;
        dot[j] = (A)0;
      }
      if (any && sh.width < VE) {
        for (int c = lane; c < sh.width; c += lanes) {
          const T d = pdy[c];
#pragma unroll
          for (int j = 0; j < J; ++j) {
            if (!live[j]) continue;
            if (DOT) dot[j] += (A)d * (A)x[(int64_t)r[j] * ldx + c];
            if (dx) dx[(int64_t)r[j] * lddx + c] = WEIGHT ? times<T>(w[j], d) : d;
          }
        }
      } else if (any) {
        for (int c = lane; c < nch; c += lanes) {
          const int at = c * VE < sh.width - VE ? c * VE : sh.width - VE;
          Chunk<T> d, v[J];
          d.load(pdy + at);
          if (DOT) {
#pragma unroll
            for (int j = 0; j < J; ++j)
              if (live[j]) {
                const T* px = x + (int64_t)r[j] * ldx + at;
                if (ONCE) v[j].load_once(px);
                else v[j].load(px);
              }
#pragma unroll
            for (int j = 0; j < J; ++j) {
              if (!live[j]) continue;
#pragma unroll
              for (int k = 0; k < VE; ++k) {
                // elements that the chunk before holds too count there
                const A p = (A)d.v[k] * (A)v[j].v[k];
                dot[j] += at + k >= c * VE ? p : (A)0;
              }
            }
          }
          if (dx) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
              if (!live[j]) continue;
              Chunk<T> out = d;
              if (WEIGHT) {
#pragma unroll
                for (int k = 0; k < VE; ++k) out.v[k] = times<T>(w[j], d.v[k]);
              }
              T* px = dx + (int64_t)r[j] * lddx + at;
              if (ONCE) out.store_once(px);
              else out.store(px);
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (j0 + j >= sh.topk) break;
        if (DOT) {
          for (int m = lanes >> 1; m; m >>= 1) dot[j] += __shfl_xor(dot[j], m);
          if (in && lane == 0) dweight[s0 + j] = dot[j];
        }
        // the empty rows: row s0 + j is looked at here
        if (dx && in && (unsigned)rows[s0 + j] >= (unsigned)sh.nslot) {
          for (int c = lane; c < sh.width; c += lanes) dx[(s0 + j) * lddx + c] = (T)0;
        }
      }
    }
  }
}

int log2_lanes(int width, size_t es) {
  const int chunk = (int)(16 / es);
  const int nch = (width + chunk - 1) / chunk;
  int l = 0;
  while (l < 6 && (1 << l) < nch) ++l;
  return l;
}

unsigned grid_for(int64_t items, int lanes_log2) {
  const int64_t per = kBlock >> lanes_log2;
  const int64_t blocks = (items + per - 1) / per;
  const int64_t most = 1 << 20;  // beyond, workgroups take several items
  return (unsigned)(blocks < most ? blocks : most);
}

// DPC_OK and the shape of a call on rows, or why it is refused
int row_shape(dpc_elem elem, int ntok, int topk, int width, Shape* sh) {
  if (!elem_ok(elem) || ntok < 0 || topk < 1 || width < 1) return DPC_EINVAL;
  if (topk > DPC_MAX_TOPK || (int64_t)ntok * topk > kMaxSlots || width > kMaxWidth) return DPC_ENOTSUP;
  *sh = Shape{(int64_t)ntok * topk, ntok, topk, width, log2_lanes(width, elem_size(elem))};
  return DPC_OK;
}

// whether the chunks of all rows start at multiples of 16 bytes
bool chunks_aligned(dpc_elem elem, const Shape& sh, const void* a, int64_t lda, const void* b, int64_t ldb) {
  const size_t es = elem_size(elem);
  return sh.width * es % 16 == 0 && (!a || (elem_aligned(a, 16) && lda * es % 16 == 0)) &&
         (!b || (elem_aligned(b, 16) && ldb * es % 16 == 0));
}
bool past_caches(dpc_elem elem, const Shape& sh) {
  return sh.nslot * sh.width * (int64_t)elem_size(elem) >= kOnceBytes;
}

bool rows_ok(dpc_elem elem, const void* p, int64_t ld, int width) {
  return p && elem_aligned(p, elem_size(elem)) && ld >= width;
}
bool weight_ok(dpc_elem elem, const void* p) { return elem_aligned(p, elem == DPC_ELEM_F64 ? 8 : 4); }

// Calls f with the element type, whether there are weights and whether the rows
// go past the caches
template <typename F>
int by_type(dpc_elem elem, bool weight, bool once, F f) {
  (void)hipGetLastError();  // report only what this launch raises
  const auto with = [&](auto t) {
    if (weight) once ? f(t, std::true_type{}, std::true_type{}) : f(t, std::true_type{}, std::false_type{});
    else once ? f(t, std::false_type{}, std::true_type{}) : f(t, std::false_type{}, std::false_type{});
  };
  switch (elem) {
    case DPC_ELEM_F64: with(double{}); break;
    case DPC_ELEM_F32: with(float{}); break;
    case DPC_ELEM_F16: with(_Float16{}); break;
    default: with(__bf16{}); break;
  }
  return dpc_internal_launch_status();
}

int send(void* stream, dpc_elem elem, const Shape& sh, const void* x, int64_t ldx, const void* weight, const int* rows,
         const int* pos, const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dweight) {
  const bool once = past_caches(elem, sh) && chunks_aligned(elem, sh, dweight ? x : nullptr, ldx, dx, lddx);
  return by_type(elem, weight != nullptr, once, [&](auto t, auto w, auto o) {
    typedef decltype(t) T;
    typedef typename ElemAcc<T>::type A;
    constexpr bool W = decltype(w)::value, ONCE = decltype(o)::value;
    const auto kernel = sh.topk == 1 ? (dweight ? send_kernel<T, W, true, 1, ONCE> : send_kernel<T, W, false, 1, ONCE>)
                                     : (dweight ? send_kernel<T, W, true, 4, ONCE> : send_kernel<T, W, false, 4, ONCE>);
    hipLaunchKernelGGL(kernel, dim3(grid_for(sh.ntok, sh.lanes_log2)), dim3(kBlock), 0,
                       static_cast<hipStream_t>(stream), sh, (const T*)x, ldx, (const A*)weight, rows, pos,
                       (const T*)dy, lddy, (T*)dx, lddx, (A*)dweight);
  });
}

}  // namespace

extern "C" size_t dpc_route_workspace_bytes(int ntok, int topk, int nexpert) {
  if (ntok < 0 || topk < 1 || topk > DPC_MAX_TOPK || nexpert < 1 || nexpert > DPC_MAX_EXPERTS) return 0;
  const int64_t nslot = (int64_t)ntok * topk;
  if (nslot > kMaxSlots) return 0;
  const size_t blocks = nslot <= kOneBlockSlots ? 0 : plan_blocks(nslot);
  return ((blocks + 1) * nexpert * sizeof(int) + 255) / 256 * 256;
}

extern "C" int dpc_route_plan(void* stream, int ntok, int topk, int nexpert, const int* expert, void* workspace,
                              size_t workspace_bytes, int* offsets, int* rows, int* pos) {
  if (ntok < 0 || topk < 1 || nexpert < 1) return DPC_EINVAL;
  const int64_t nslot = (int64_t)ntok * topk;
  if (topk > DPC_MAX_TOPK || nexpert > DPC_MAX_EXPERTS || nslot > kMaxSlots) return DPC_ENOTSUP;
  if (!offsets || !elem_aligned(offsets, 4)) return DPC_EINVAL;
  if (nslot > 0) {
    if (!expert || !rows || !pos || !workspace || !elem_aligned(workspace, 16) || !elem_aligned(expert, 4) ||
        !elem_aligned(rows, 4) || !elem_aligned(pos, 4))
      return DPC_EINVAL;
    if (workspace_bytes < dpc_route_workspace_bytes(ntok, topk, nexpert)) return DPC_EINVAL;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();  // report only what these launches raise
  if (nslot <= kOneBlockSlots) {
    const int waves = nslot <= 256 ? 4 : 16;
    const size_t lds = ((size_t)(waves + 1) * nexpert + waves) * sizeof(int);
    hipLaunchKernelGGL(plan_one_kernel, dim3(1), dim3(64 * waves), lds, s, (int)nslot, nexpert, expert, offsets, rows,
                       pos);
    return dpc_internal_launch_status();
  }
  const int blocks = plan_blocks(nslot);
  const int64_t part = plan_part(nslot, blocks);
  int* hist = static_cast<int*>(workspace);
  int* total = hist + (size_t)blocks * nexpert;
  const dim3 block(64 * kPlanWaves);
  hipLaunchKernelGGL(plan_count_kernel, dim3(blocks), block, (size_t)kPlanWaves * nexpert * sizeof(int), s, nslot, part,
                     nexpert, expert, hist);
  hipLaunchKernelGGL(plan_scan_kernel, dim3(nexpert), dim3(256), 0, s, blocks, hist, total);
  hipLaunchKernelGGL(plan_place_kernel, dim3(blocks), block,
                     ((size_t)(kPlanWaves + 1) * nexpert + kPlanWaves) * sizeof(int), s, nslot, part, nexpert, expert,
                     hist, total, offsets, rows, pos);
  return dpc_internal_launch_status();
}

extern "C" int dpc_route_gather(void* stream, dpc_elem elem, int ntok, int topk, int width, const void* x, int64_t ldx,
                                const void* weight, const int* rows, const int* pos, void* y, int64_t ldy) {
  Shape sh;
  const int st = row_shape(elem, ntok, topk, width, &sh);
  if (st != DPC_OK) return st;
  if (ntok == 0) return DPC_OK;
  if (!rows_ok(elem, x, ldx, width) || !rows_ok(elem, y, ldy, width) || !weight_ok(elem, weight) || !rows ||
      !pos || !elem_aligned(rows, 4) || !elem_aligned(pos, 4))
    return DPC_EINVAL;
  return send(stream, elem, sh, nullptr, 0, weight, rows, pos, x, ldx, y, ldy, nullptr);
}

extern "C" int dpc_route_combine(void* stream, dpc_elem elem, int ntok, int topk, int width, const void* x, int64_t ldx,
                                 const void* weight, const int* pos, void* y, int64_t ldy) {
  Shape sh;
  const int st = row_shape(elem, ntok, topk, width, &sh);
  if (st != DPC_OK) return st;
  if (ntok == 0) return DPC_OK;
  if (!rows_ok(elem, x, ldx, width) || !rows_ok(elem, y, ldy, width) || !weight_ok(elem, weight) || !pos ||
      !elem_aligned(pos, 4))
    return DPC_EINVAL;
  const bool once = past_caches(elem, sh) && chunks_aligned(elem, sh, x, ldx, y, ldy);
  return by_type(elem, weight != nullptr, once, [&](auto t, auto w, auto o) {
    typedef decltype(t) T;
    hipLaunchKernelGGL((combine_kernel<T, decltype(w)::value, decltype(o)::value>), dim3(grid_for(ntok, sh.lanes_log2)), dim3(kBlock), 0,
                       static_cast<hipStream_t>(stream), sh, (const T*)x, ldx,
                       (const typename ElemAcc<T>::type*)weight, pos, (T*)y, ldy);
  });
}

extern "C" int dpc_route_combine_bwd(void* stream, dpc_elem elem, int ntok, int topk, int width, const void* x,
                                     int64_t ldx, const void* weight, const int* rows, const int* pos, const void* dy,
                                     int64_t lddy, void* dx, int64_t lddx, void* dweight) {
  Shape sh;
  const int st = row_shape(elem, ntok, topk, width, &sh);
  if (st != DPC_OK) return st;
  if (ntok == 0) return DPC_OK;
  if (!dx && !dweight) return DPC_EINVAL;
  if (!rows_ok(elem, dy, lddy, width) || (dweight && !rows_ok(elem, x, ldx, width)) ||
      (dx && !rows_ok(elem, dx, lddx, width)) || !weight_ok(elem, weight) || !weight_ok(elem, dweight) || !rows ||
      !pos || !elem_aligned(rows, 4) || !elem_aligned(pos, 4))
    return DPC_EINVAL;
  return send(stream, elem, sh, x, ldx, weight, rows, pos, dy, lddy, dx, lddx, dweight);
}
