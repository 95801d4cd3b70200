// Vectors of ids (dpc_embed) and the gradient of their table (dpc_embed_bwd).
//
// Lookup: a copy of rows with one product per element; the table of a few ids
// stays in the caches, and the call is bound by what it writes.
//
// Gradient: tokens are sorted by id (dpc_sort.h, up to 10 bits of the id a
// pass), so that an id's tokens are a run of positions.  The positions are cut into
// parts.  A group of lanes sums the runs of its part, in order; a run inside one
// part is written out, of a run that crosses into another part both keep the
// sum of their piece, which a second kernel joins.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "dpc.h"
#include "dpc_elem.h"
#include "dpc_internal.h"
#include "dpc_sort.h"

namespace {

constexpr int kMaxCount = 1 << 30;          // tokens, ids
constexpr int kMaxWidth = INT32_MAX - 127;  // a lane's next element (64 on) and a width rounded up to chunks are ints
constexpr int kBlock = 256;

int log2_lanes(int width, size_t es) {
  const int chunk = (int)(16 / es);
  const int nch = (width + chunk - 1) / chunk;
  int l = 0;
  while (l < 6 && (1 << l) < nch) ++l;
  return l;
}

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kBlock) void embed_kernel(int ntok, int nid, int width, int lanes_log2,
                                                       const int* __restrict__ ids, const T* __restrict__ table, int64_t ldt,
                                                       typename ElemAcc<T>::type scale, T* __restrict__ y, int64_t ldy) {
  constexpr int VE = Chunk<T>::kElems;
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int64_t groups = ((int64_t)gridDim.x * kBlock) >> lanes_log2;
  const int nch = (width + VE - 1) / VE;
  for (int64_t t = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lanes_log2; t < ntok; t += groups) {
    const int id = ids[t];
    const bool live = (unsigned)id < (unsigned)nid;
    const T* px = table + (int64_t)(live ? id : 0) * ldt;
    T* py = y + t * ldy;
    if (width < VE) {
      for (int c = lane; c < width; c += lanes) py[c] = live ? times<T>(scale, px[c]) : (T)0;
      continue;
    }
    for (int c = lane; c < nch; c += lanes) {
      const int at = c * VE < width - VE ? c * VE : width - VE;
      Chunk<T> ch;
      ch.load(px + at);
#pragma unroll
      for (int i = 0; i < VE; ++i) ch.v[i] = live ? times<T>(scale, ch.v[i]) : (T)0;
      ch.store(py + at);
    }
  }
}

// ---------------------------------------------------------------------------
// tokens sorted by id
// ---------------------------------------------------------------------------
// One pass over `bits` bits of the ids from `shift` on.  The first pass drops
// ids outside [0, nid); later ones sort what the pass before has left.
struct IdJob {
  const int* __restrict__ from_id;   // ids in the order of the pass before
  const int* __restrict__ from_tok;  // their tokens; NULL: the order of the tokens
  const int* __restrict__ left;      // how many there are; NULL: all
  int* __restrict__ to_id;
  int* __restrict__ to_tok;
  int* __restrict__ kept;
  int nid, shift, mask;
  __device__ __forceinline__ int key(int64_t s) const {
    const int id = from_id[s];
    return (unsigned)id < (unsigned)nid ? id >> shift & mask : -1;
  }
  __device__ __forceinline__ int64_t size(int64_t n) const { return left ? min((int64_t)*left, n) : n; }
  __device__ __forceinline__ void put(int64_t s, int, int row) const {
    if (row < 0) return;
    to_id[row] = from_id[s];
    to_tok[row] = from_tok ? from_tok[s] : (int)s;
  }
  __device__ __forceinline__ void first(int, int) const {}
  __device__ __forceinline__ void total(int n) const { *kept = n; }
  __device__ __forceinline__ void empty(int64_t) const {}
};

struct Passes {
  int count, bits;
};
inline Passes passes_for(int nid) {
  int bits = 1;
  while (bits < 31 && (1 << bits) < nid) ++bits;
  const int count = (bits + 9) / 10;
  return Passes{count, (bits + count - 1) / count};
}

// ---------------------------------------------------------------------------
// sums of runs
// ---------------------------------------------------------------------------
struct Runs {
  const int* __restrict__ id;   // of each position, ascending
  const int* __restrict__ tok;
  const int* __restrict__ kept; // positions
  int nid, width, part, parts, slabs, lanes_log2;
};

// Chunk of a lane: its first element, or -1.  Widths under a chunk: an element.
template <typename T>
__device__ __forceinline__ int chunk_at(const Runs& r, int slab, int lane) {
  constexpr int VE = Chunk<T>::kElems;
  const int c = (slab << r.lanes_log2) + lane;
  if (r.width < VE) return c < r.width ? c : -1;
  const int nch = (r.width + VE - 1) / VE;
  return c >= nch ? -1 : c * VE < r.width - VE ? c * VE : r.width - VE;
}

template <typename TD, int VE, typename S>
__device__ __forceinline__ void write_row(TD* p, int at, bool narrow, const S (&sum)[VE], S scale) {
#pragma unroll
  for (int i = 0; i < VE; ++i)
    if (i == 0 || !narrow) p[at + i] = (TD)(sum[i] * scale);
}

// partial sums: [parts][2][width], 0: the run that comes from the part before,
// 1: a run that starts here and goes on
template <typename T, typename TD>
__global__ __launch_bounds__(kBlock) void runs_kernel(Runs r, const T* __restrict__ dy, int64_t lddy,
                                                      typename ElemAcc<T>::type scale,
                                                      typename ElemAcc<T>::type* __restrict__ partial,
                                                      TD* __restrict__ dtable, int64_t ldt) {
  typedef typename ElemAcc<T>::type A;
  constexpr int VE = Chunk<T>::kElems;
  const int lane = threadIdx.x & ((1 << r.lanes_log2) - 1);
  const int64_t item = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> r.lanes_log2;
  if (item >= (int64_t)r.parts * r.slabs) return;
  const int part = (int)(item / r.slabs), slab = (int)(item % r.slabs);
  const int64_t n = *r.kept, p0 = (int64_t)part * r.part, p1 = min(n, p0 + r.part);
  const int at = chunk_at<T>(r, slab, lane);
  if (p0 >= p1 || at < 0) return;
  const bool narrow = r.width < VE;
  const int before = p0 > 0 ? r.id[p0 - 1] : -1, after = p1 < n ? r.id[p1] : -1;
  A sum[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) sum[i] = (A)0;
  int cur = r.id[p0];
  auto flush = [&](int64_t end) {
    const bool open_left = cur == before, open_right = end == p1 && cur == after;
    if (!open_left && !open_right) {
      write_row<TD>(dtable + cur * ldt, at, narrow, sum, scale);
    } else {
      // a run that fills the part and goes on both ways counts as one from the left
      A* to = partial + ((int64_t)part * 2 + (open_left ? 0 : 1)) * r.width;
      write_row<A>(to, at, narrow, sum, (A)1);
    }
  };
  for (int64_t p = p0; p < p1; ++p) {
    const int id = r.id[p];
    if (id != cur) {
      flush(p);
      cur = id;
#pragma unroll
      for (int i = 0; i < VE; ++i) sum[i] = (A)0;
    }
    const T* px = dy + (int64_t)r.tok[p] * lddy + at;
    if (narrow) {
      sum[0] += (A)px[0];
    } else {
      Chunk<T> ch;
      ch.load(px);
#pragma unroll
      for (int i = 0; i < VE; ++i) sum[i] += (A)ch.v[i];
    }
  }
  flush(p1);
}

// First position from lo on (of n) whose id is above v.
__device__ __forceinline__ int64_t behind(const int* id, int64_t lo, int64_t n, int v) {
  int64_t hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (id[mid] > v) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

template <typename T, typename TD>
__global__ __launch_bounds__(kBlock) void join_kernel(Runs r, typename ElemAcc<T>::type scale,
                                                      const typename ElemAcc<T>::type* __restrict__ partial,
                                                      TD* __restrict__ dtable, int64_t ldt) {
  constexpr int VE = Chunk<T>::kElems;
  const int lane = threadIdx.x & ((1 << r.lanes_log2) - 1);
  const int64_t item = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> r.lanes_log2;
  if (item >= (int64_t)r.parts * r.slabs) return;
  const int part = (int)(item / r.slabs), slab = (int)(item % r.slabs);
  const int64_t n = *r.kept, p0 = (int64_t)part * r.part, p1 = min(n, p0 + r.part);
  const int at = chunk_at<T>(r, slab, lane);
  if (p1 >= n || p0 >= p1 || at < 0) return;
  const int v = r.id[p1 - 1];
  if (r.id[p1] != v || (p0 > 0 && r.id[p0 - 1] == v)) return;  // the run ends here, or starts before
  const bool narrow = r.width < VE;
  const int last = (int)((behind(r.id, p1, n, v) - 1) / r.part);
  double sum[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) sum[i] = i == 0 || !narrow ? (double)partial[((int64_t)part * 2 + 1) * r.width + at + i] : 0.0;
  for (int q = part + 1; q <= last; ++q) {
#pragma unroll
    for (int i = 0; i < VE; ++i)
      if (i == 0 || !narrow) sum[i] += (double)partial[(int64_t)q * 2 * r.width + at + i];
  }
  write_row<TD>(dtable + v * ldt, at, narrow, sum, (double)scale);
}

// Zeros in the rows of ids without tokens.
template <typename TD>
__global__ __launch_bounds__(kBlock) void absent_kernel(Runs r, TD* __restrict__ dtable, int64_t ldt) {
  const int64_t n = *r.kept;
  const int lane = threadIdx.x & 63;
  const int64_t waves = (int64_t)gridDim.x * (kBlock / 64);
  for (int64_t v = (int64_t)blockIdx.x * (kBlock / 64) + threadIdx.x / 64; v < r.nid; v += waves) {
    const int64_t at = behind(r.id, 0, n, (int)v);
    if (at > 0 && r.id[at - 1] == v) continue;
    for (int c = lane; c < r.width; c += 64) dtable[v * ldt + c] = (TD)0;
  }
}

// What a gradient needs of the workspace, in order.
struct Layout {
  Passes passes;
  int part, parts, slabs, lanes_log2;
  size_t id[2], tok[2], kept, sort, partial, bytes;
};
Layout layout_for(dpc_elem elem, int ntok, int nid, int width) {
  Layout l;
  l.passes = passes_for(nid);
  l.lanes_log2 = log2_lanes(width, elem_size(elem));
  const int VE = (int)(16 / elem_size(elem)), nch = width < VE ? width : (width + VE - 1) / VE;
  l.slabs = (int)(((int64_t)nch + (1 << l.lanes_log2) - 1) >> l.lanes_log2);
  const int64_t part = ((int64_t)ntok * l.slabs + 4095) / 4096;
  l.part = (int)(part < 16 ? 16 : part > 1024 ? 1024 : part);
  l.parts = (int)(((int64_t)ntok + l.part - 1) / l.part);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  for (int b = 0; b < 2; ++b) {
    l.id[b] = take((size_t)ntok * 4);
    l.tok[b] = take((size_t)ntok * 4);
  }
  l.kept = take(4 * sizeof(int));
  l.sort = take(sort_workspace_bytes(ntok, 1 << l.passes.bits));
  l.partial = take((size_t)l.parts * 2 * width * (elem == DPC_ELEM_F64 ? 8 : 4));
  l.bytes = at;
  return l;
}

// Calls f with a value of the element type.
template <typename F>
void by_elem(dpc_elem elem, F f) {
  switch (elem) {
    case DPC_ELEM_F64: f(double{}); break;
    case DPC_ELEM_F32: f(float{}); break;
    case DPC_ELEM_F16: f(_Float16{}); break;
    default: f(__bf16{}); break;
  }
}

int embed_sizes(dpc_elem elem, int ntok, int nid, int width) {
  if (!elem_ok(elem) || ntok < 0 || nid < 1 || width < 1) return DPC_EINVAL;
  return ntok > kMaxCount || nid > kMaxCount || width > kMaxWidth ? DPC_ENOTSUP : DPC_OK;
}

}  // namespace

extern "C" int dpc_embed(void* stream, dpc_elem elem, int ntok, int nid, int width, const int* ids, const void* table,
                         int64_t ldt, double scale, void* y, int64_t ldy) {
  const int st = embed_sizes(elem, ntok, nid, width);
  if (st != DPC_OK) return st;
  if (!std::isfinite(scale)) return DPC_EINVAL;
  if (ntok == 0) return DPC_OK;
  if (!ids || !table || !y || ldt < width || ldy < width || !elem_aligned(ids, 4) ||
      !elem_aligned(table, elem_size(elem)) || !elem_aligned(y, elem_size(elem)))
    return DPC_EINVAL;
  (void)hipGetLastError();  // report only what this launch raises
  by_elem(elem, [&](auto tt) {
    typedef decltype(tt) T;
    const int l = log2_lanes(width, sizeof(T));
    const int64_t per = kBlock >> l, blocks = (ntok + per - 1) / per, most = 1 << 20;
    hipLaunchKernelGGL(embed_kernel<T>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kBlock), 0,
                       static_cast<hipStream_t>(stream), ntok, nid, width, l, ids, (const T*)table, ldt,
                       (typename ElemAcc<T>::type)scale, (T*)y, ldy);
  });
  return dpc_internal_launch_status();
}

extern "C" size_t dpc_embed_bwd_workspace_bytes(dpc_elem elem, int ntok, int nid, int width) {
  if (embed_sizes(elem, ntok, nid, width) != DPC_OK) return 0;
  return layout_for(elem, ntok, nid, width).bytes;
}

extern "C" int dpc_embed_bwd(void* stream, dpc_elem elem, dpc_elem elem_d, int ntok, int nid, int width, const int* ids,
                             const void* dy, int64_t lddy, double scale, void* workspace, size_t workspace_bytes,
                             void* dtable, int64_t lddt) {
  const int st = embed_sizes(elem, ntok, nid, width);
  if (st != DPC_OK) return st;
  if (!std::isfinite(scale) || (elem_d != elem && elem_d != DPC_ELEM_F32)) return DPC_EINVAL;
  if (!dtable || lddt < width || !elem_aligned(dtable, elem_size(elem_d)) || !workspace || !elem_aligned(workspace, 16) ||
      (ntok > 0 && (!ids || !dy || lddy < width || !elem_aligned(ids, 4) || !elem_aligned(dy, elem_size(elem)))))
    return DPC_EINVAL;
  const Layout l = layout_for(elem, ntok, nid, width);
  if (workspace_bytes < l.bytes) return DPC_EINVAL;
  char* ws = static_cast<char*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();  // report only what these launches raise
  const auto at = [&](size_t where) { return reinterpret_cast<int*>(ws + where); };
  const int* id = ids;
  const int* tok = nullptr;
  const int* left = nullptr;
  for (int p = 0; p < l.passes.count; ++p) {
    int* kept = at(l.kept) + p;
    const IdJob job{id, tok, left, at(l.id[p & 1]), at(l.tok[p & 1]), kept, nid, p * l.passes.bits, (1 << l.passes.bits) - 1};
    launch_sort(s, ntok, 1 << l.passes.bits, job, ws + l.sort);
    id = job.to_id;
    tok = job.to_tok;
    left = kept;
  }
  const Runs r{id, tok, left, nid, width, l.part, l.parts, l.slabs, l.lanes_log2};
  const int64_t threads = ((int64_t)l.parts * l.slabs) << l.lanes_log2;
  const dim3 grid((unsigned)((threads + kBlock - 1) / kBlock));
  by_elem(elem, [&](auto tt) {
    typedef decltype(tt) T;
    typedef typename ElemAcc<T>::type A;
    const auto go = [&](auto dd) {
      typedef decltype(dd) TD;
      if (ntok > 0) {
        hipLaunchKernelGGL((runs_kernel<T, TD>), grid, dim3(kBlock), 0, s, r, (const T*)dy, lddy, (A)scale,
                           (A*)(ws + l.partial), (TD*)dtable, lddt);
        hipLaunchKernelGGL((join_kernel<T, TD>), grid, dim3(kBlock), 0, s, r, (A)scale, (const A*)(ws + l.partial),
                           (TD*)dtable, lddt);
      }
      const int64_t blocks = ((int64_t)nid + 3) / 4, most = 1 << 20;
      hipLaunchKernelGGL(absent_kernel<TD>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kBlock), 0, s, r,
                         (TD*)dtable, lddt);
    };
    if (elem_d == elem) go(T{});
    else go(float{});
  });
  return dpc_internal_launch_status();
}
