// Vectors of ids (dpc_embed) and the gradient of their table (dpc_embed_bwd).
//
// Lookup: a copy of rows with one product per element; the table of a few ids
// stays in the caches, and the call is bound by what it writes: 1,048,576 float32 rows
// of 240 for 3 ids 174 us (5.8 TB/s).  A vocabulary's rows are read, too: 16,384 bfloat16
// rows of 4,096 for 65,536 ids 54 us (a copy of the bytes 56), 131,072 of them 308 (335).
//
// Gradient: tokens are sorted by id (dpc_sort.h, up to 10 bits of the id a
// pass), so that an id's tokens are a run of positions.  The positions are cut into
// parts.  A group of lanes sums the runs of its part, in order and in float64; a
// run inside one part is written out, of a run that crosses into another part both
// keep the sum of their piece, which a second kernel joins.  331,776 float32 rows of
// 240 for 2 ids 76 us: sort 11, runs 61 (the rows at 5.2 TB/s), joins 11 (the kernels
// one by one); 16,384 bfloat16 rows of 4,096 for 65,536 ids 174: sort 29, runs and zeros
// 132 (671 MB at 5.1 TB/s), joins 14.
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
// One dimension of a launch has under 2^32 threads.
inline dim3 rows_grid(int64_t blocks) {
  const int64_t wide = 1 << 23;
  return blocks <= wide ? dim3((unsigned)blocks) : dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide));
}

constexpr int kRowsAtOnce = 4;  // rows whose loads a group of lanes has under way

// Results of 192 MiB and more (with addresses and strides multiples of 16 bytes)
// go past the caches: they would not be found there by the call that uses them.
constexpr int64_t kOnceBytes = (int64_t)192 << 20;

template <typename T, bool ONCE>
__global__ __launch_bounds__(kBlock) void embed_kernel(int ntok, int nid, int width, int lanes_log2,
                                                       const int* __restrict__ ids, const T* __restrict__ table, int64_t ldt,
                                                       typename ElemAcc<T>::type scale, T* __restrict__ y, int64_t ldy) {
  constexpr int VE = Chunk<T>::kElems, R = kRowsAtOnce;
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int nch = (width + VE - 1) / VE;
  const int64_t block = blockIdx.y * (int64_t)gridDim.x + blockIdx.x;
  const int64_t t0 = ((block * kBlock + threadIdx.x) >> lanes_log2) * R;
  if (t0 >= ntok) return;
  const T* px[R];
  bool live[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int id = ids[t0 + j < ntok ? t0 + j : ntok - 1];
    live[j] = (unsigned)id < (unsigned)nid;
    px[j] = table + (int64_t)(live[j] ? id : 0) * ldt;
  }
  if (width < VE) {
    for (int c = lane; c < width; c += lanes)
#pragma unroll
      for (int j = 0; j < R; ++j)
        if (t0 + j < ntok) y[(t0 + j) * ldy + c] = live[j] ? times<T>(scale, px[j][c]) : (T)0;
    return;
  }
  for (int c = lane; c < nch; c += lanes) {
    const int at = c * VE < width - VE ? c * VE : width - VE;
    Chunk<T> ch[R];
#pragma unroll
    for (int j = 0; j < R; ++j) ch[j].load(px[j] + at);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (t0 + j >= ntok) break;
#pragma unroll
      for (int i = 0; i < VE; ++i) ch[j].v[i] = live[j] ? times<T>(scale, ch[j].v[i]) : (T)0;
      T* py = y + (t0 + j) * ldy + at;
      if (ONCE) ch[j].store_once(py);
      else ch[j].store(py);
    }
  }
}

// The same for results without gaps between rows of whole chunks, as one array of
// chunks: every store of a wavefront is 1 KiB in a piece, whole cache lines.  (Row by
// row 1,048,576 rows of 960 bytes take 194 us.)
constexpr int kFlat = 4;  // chunks of a lane

template <typename T, bool ONCE>
__global__ __launch_bounds__(kBlock) void embed_flat_kernel(unsigned chunks, unsigned nch, double inverse, int nid,
                                                            const int* __restrict__ ids, const T* __restrict__ table,
                                                            int64_t ldt, typename ElemAcc<T>::type scale, T* __restrict__ y) {
  constexpr int VE = Chunk<T>::kElems;
  const unsigned f0 = blockIdx.x * (kBlock * kFlat) + (threadIdx.x & ~63u) * kFlat + (threadIdx.x & 63);
  Chunk<T> ch[kFlat];
  bool live[kFlat];
#pragma unroll
  for (int u = 0; u < kFlat; ++u) {
    const unsigned f = min(f0 + u * 64, chunks - 1);
    // f / nch: (f + 1/2) / nch is 1/2 / nch or more from a whole number
    const unsigned t = (unsigned)(((double)f + 0.5) * inverse);
    const int id = ids[t];
    live[u] = (unsigned)id < (unsigned)nid;
    ch[u].load(table + (int64_t)(live[u] ? id : 0) * ldt + (f - t * nch) * VE);
  }
#pragma unroll
  for (int u = 0; u < kFlat; ++u) {
    if (f0 + u * 64 >= chunks) break;
#pragma unroll
    for (int i = 0; i < VE; ++i) ch[u].v[i] = live[u] ? times<T>(scale, ch[u].v[i]) : (T)0;
    T* py = y + (int64_t)(f0 + u * 64) * VE;
    if (ONCE) ch[u].store_once(py);
    else ch[u].store(py);
  }
}

// ---------------------------------------------------------------------------
// tokens sorted by id
// ---------------------------------------------------------------------------
// One pass over `bits` bits of the ids from `shift` on.  The first pass drops
// ids outside [0, nid); later ones sort what the pass before has left.
struct IdJob {
  static constexpr int kPart = 512;  // 100,000 tokens of as many ids 61.7 us in all, with 256 62.8, with 1,024 70.0
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
  int nid, width, part, parts, slabs, lanes_log2, join_slabs, join_log2;
  int zero_slabs, zero_wide;    // columns of the zeros of a wavefront: chunks zero_wide s and more of slab s
};

// First element of chunk c, or -1.  Widths under a chunk: element c.
template <typename T>
__device__ __forceinline__ int chunk_at(const Runs& r, int c) {
  constexpr int VE = Chunk<T>::kElems;
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

// First position (of n) whose id is v or above.
__device__ __forceinline__ int64_t reaches(const int* id, int64_t n, int64_t v) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (id[mid] >= v) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Zeros in chunks [c0, c1) of the rows of the ids of [64 k, 64 k + 64) that have no
// token, by one wavefront: each lane looks for one id.
template <typename TD>
__device__ __forceinline__ void absent(const Runs& r, int64_t k, int c0, int c1, int64_t n, TD* dtable, int64_t ldt) {
  constexpr int VE = Chunk<TD>::kElems;
  const int lane = threadIdx.x & 63;
  const int64_t v = k * 64 + lane;
  const int64_t at = v < r.nid ? reaches(r.id, n, v) : 0;
  const bool none = v < r.nid && (at >= n || r.id[at] != v);
  Chunk<TD> zero;
#pragma unroll
  for (int i = 0; i < VE; ++i) zero.v[i] = (TD)0;
  for (unsigned long long left = __ballot(none); left; left &= left - 1) {
    TD* p = dtable + (k * 64 + __ffsll(left) - 1) * ldt;
    if (r.width < VE) {
      if (lane < r.width) p[lane] = (TD)0;
    } else {
      for (int c = c0 + lane; c < c1; c += 64) zero.store(p + (c * VE < r.width - VE ? c * VE : r.width - VE));
    }
  }
}

// Sums of the runs of each part, and zeros in the rows of ids without tokens (the
// workgroups from run_blocks on): one launch, since neither waits for the other.
// partial sums: [parts][2][width], 0: the run that comes from the part before,
// 1: a run that starts here and goes on.
// kAtOnce rows of a part are under way at a time, whichever ids they belong to.
// KIND kNarrow: rows of less than a chunk, an element to a lane (a branch inside would
// cut the loads of chunks in pieces: 494,073 float16 rows of 240 take 133 us for 58 then); kWide:
// a row takes a whole wavefront, and what is known of positions is scalar.
enum Kind { kNarrow, kChunks, kWide };
constexpr int kAtOnce = 8;
constexpr int kZeroWaves = 4096;

template <typename T, typename TD, Kind KIND>
__global__ __launch_bounds__(kBlock) void runs_kernel(Runs r, unsigned run_blocks, const T* __restrict__ dy, int64_t lddy,
                                                      double scale, double* __restrict__ partial,
                                                      TD* __restrict__ dtable, int64_t ldt) {
  constexpr int VE = Chunk<T>::kElems;
  constexpr bool WIDE = KIND == kWide, narrow = KIND == kNarrow;
  const int64_t n = *r.kept;
  if (blockIdx.x >= run_blocks) {
    const int64_t item = (int64_t)(blockIdx.x - run_blocks) * (kBlock / 64) + threadIdx.x / 64, k = item / r.zero_slabs;
    const int nch = (r.width + Chunk<TD>::kElems - 1) / Chunk<TD>::kElems;
    const int c0 = (int)(item % r.zero_slabs) * r.zero_wide;
    if (k * 64 < r.nid) absent<TD>(r, k, c0, min(nch - c0, r.zero_wide) + c0, n, dtable, ldt);
    return;
  }
  const int lane = threadIdx.x & ((1 << r.lanes_log2) - 1);
  const int64_t item = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> r.lanes_log2;
  if (item >= (int64_t)r.parts * r.slabs) return;
  int part = (int)(item / r.slabs);
  const int slab = (int)(item % r.slabs);
  if (WIDE) part = __builtin_amdgcn_readfirstlane(part);
  const int64_t p0 = (int64_t)part * r.part, p1 = min(n, p0 + r.part);
  const int at = chunk_at<T>(r, (slab << r.lanes_log2) + lane);
  if (p0 >= p1 || (!WIDE && at < 0)) return;
  const int before = p0 > 0 ? r.id[p0 - 1] : -1, after = p1 < n ? r.id[p1] : -1;
  double sum[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) sum[i] = 0.0;
  int cur = r.id[p0];
  auto flush = [&](int64_t end) __attribute__((always_inline)) {
    const bool open_left = cur == before, open_right = end == p1 && cur == after;
    if (at < 0) return;
    if (!open_left && !open_right) {
      write_row<TD>(dtable + cur * ldt, at, narrow, sum, scale);
    } else {
      // a run that fills the part and goes on both ways counts as one from the left
      write_row<double>(partial + ((int64_t)part * 2 + (open_left ? 0 : 1)) * r.width, at, narrow, sum, 1.0);
    }
  };
  // The rows behind these are on their way while these are added, and the ids behind
  // those while they are.
  struct Ids {
    int id[kAtOnce], tok[kAtOnce];
  };
  auto look = [&](int64_t p, Ids& to) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int64_t q = p + k < p1 ? p + k : p1 - 1;
      to.id[k] = r.id[q];
      to.tok[k] = r.tok[q];
    }
  };
  auto fetch = [&](const Ids& of, Chunk<T> (&to)[kAtOnce]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const T* px = dy + (int64_t)of.tok[k] * lddy + max(at, 0);
      if constexpr (narrow) to[k].v[0] = px[0];
      else to[k].load(px);
    }
  };
  Ids now, next;
  Chunk<T> ch[kAtOnce], behind[kAtOnce];
  look(p0, now);
  fetch(now, ch);
  if (p0 + kAtOnce < p1) look(p0 + kAtOnce, next);
  for (int64_t p = p0; p < p1; p += kAtOnce) {
    const bool more = p + kAtOnce < p1;
    Ids later;
    if (more) {
      fetch(next, behind);
      look(min(p + 2 * kAtOnce, p1 - 1), later);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (p + k >= p1) break;
      if (now.id[k] != cur) {
        flush(p + k);
        cur = now.id[k];
#pragma unroll
        for (int i = 0; i < VE; ++i) sum[i] = 0.0;
      }
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (i == 0 || !narrow) sum[i] += (double)ch[k].v[i];
    }
    if (more) {
      now = next;
      next = later;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) ch[k] = behind[k];
    }
  }
  flush(p1);
}

// Sums of the runs that cross parts, 2^join_log2 chunks of a row at a time.  A
// group of lanes looks at the part where such a run starts; of up to kAlone parts
// it joins them itself, of up to kLong all groups of its wavefront do, longer ones
// are joined by the whole workgroup, one after the other.  Few columns to a
// workgroup: a run of hundreds of parts would take the CU's whole bandwidth else
// (331,776 rows of 960 bytes for 2 ids: whole rows 56 us).
constexpr int kJoinBlock = 512, kAlone = 8, kLong = 512;

// Partial sums of parts first, first + step, ... up to last; the run starts in `part`.
template <int VE, bool NARROW>
__device__ __forceinline__ void add_parts(const Runs& r, const double* partial, int part, int first, int step, int last,
                                          int at, double (&sum)[VE]) {
  constexpr int U = NARROW ? 8 : 32 / VE, N = NARROW ? 1 : VE;
  for (int64_t q = first; q <= last; q += U * step) {
    double v[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t w = min(q + u * step, (int64_t)last);
      __builtin_memcpy(v[u], partial + (w * 2 + (w == part)) * r.width + at, N * sizeof(double));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (q + u * step <= last) sum[i] += v[u][i];
  }
}

template <typename T, typename TD>
__global__ __launch_bounds__(kJoinBlock) void join_kernel(Runs r, double scale, const double* __restrict__ partial,
                                                          TD* __restrict__ dtable, int64_t ldt) {
  constexpr int VE = Chunk<T>::kElems;
  __shared__ double sums[kJoinBlock * VE];
  __shared__ int list[kJoinBlock][3], listed;
  const int lane = threadIdx.x & ((1 << r.join_log2) - 1), sub = threadIdx.x >> r.join_log2;
  const int subs = kJoinBlock >> r.join_log2;
  const int64_t n = *r.kept;
  const bool narrow = r.width < VE;
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  auto add = [&](int part, int first, int step, int last, int at, double (&sum)[VE]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VE; ++i) sum[i] = 0.0;
    if (narrow) add_parts<VE, true>(r, partial, part, first, step, last, at, sum);
    else add_parts<VE, false>(r, partial, part, first, step, last, at, sum);
  };
  // neighbouring groups take neighbouring parts of the same columns
  const int64_t item = (int64_t)blockIdx.x * subs + sub;
  const int slab = (int)(item / r.parts), part = (int)(item % r.parts);
  const int at = slab < r.join_slabs ? chunk_at<T>(r, (slab << r.join_log2) + lane) : -1;
  const int64_t p0 = (int64_t)part * r.part, p1 = p0 + r.part;
  int mine = part;  // last part of the run that starts in `part` and goes on, if one does
  if (slab < r.join_slabs && p1 < n) {
    const int v = r.id[p1 - 1];
    if (r.id[p1] == v && (p0 == 0 || r.id[p0 - 1] != v)) {  // starts here and goes on
      // Part q belongs to the run if its first position does: last does, past does
      // not.  Each lane of the group tries one: the next parts, then cuts of the rest.
      const int lanes = 1 << r.join_log2, end = (int)((n + r.part - 1) / r.part);
      const auto how_many = [&](int q) {  // of the lanes' q, which ascend, belong to the run
        const unsigned long long yes = __ballot(q < end && r.id[(int64_t)q * r.part] == v);
        return __popcll(yes >> (threadIdx.x & 63 & ~(lanes - 1)) & (~0ull >> (64 - lanes)));
      };
      int last = part + 1, past = end;
      const int next = how_many(last + 1 + lane);
      last += next;
      if (next < lanes) past = last + 1;
      while (past - last > 1) {
        const int wide = past - last;
        const auto cut = [&](int i) { return last + (int)((int64_t)wide * (i + 1) / (lanes + 1)); };
        const int yes = how_many(cut(lane));
        past = yes < lanes ? cut(yes) : past;
        last = yes > 0 ? cut(yes - 1) : last;
      }
      mine = last;
      if (last - part >= kLong) {
        if (lane == 0) {
          int* entry = list[atomicAdd(&listed, 1)];
          entry[0] = sub;
          entry[1] = last;
          entry[2] = v;
        }
      } else if (at >= 0 && last - part < kAlone) {
        double sum[VE];
        add(part, part, 1, last, at, sum);
        write_row<TD>(dtable + v * ldt, at, narrow, sum, scale);
      }
    }
  }
  // runs of some length: every group of the wavefront, one after the other
  const int wave_subs = 64 >> r.join_log2;
  for (unsigned long long left = __ballot(lane == 0 && mine - part >= kAlone && mine - part < kLong); left; left &= left - 1) {
    const int from = __ffsll(left) - 1;
    const int first = __shfl(part, from), last = __shfl(mine, from), at_it = __shfl(at, from + lane);
    double sum[VE];
    if (at_it >= 0) add(first, first + ((threadIdx.x & 63) >> r.join_log2), wave_subs, last, at_it, sum);
    else
#pragma unroll
      for (int i = 0; i < VE; ++i) sum[i] = 0.0;
    for (int m = 1 << r.join_log2; m < 64; m <<= 1)
#pragma unroll
      for (int i = 0; i < VE; ++i) sum[i] += __shfl_xor(sum[i], m);
    if ((int)(threadIdx.x & 63) < 1 << r.join_log2 && at_it >= 0)
      write_row<TD>(dtable + (int64_t)r.id[(int64_t)last * r.part] * ldt, at_it, narrow, sum, scale);
  }
  __syncthreads();
  for (int l = 0; l < listed; ++l) {
    const int64_t it = (int64_t)blockIdx.x * subs + list[l][0];
    const int first = (int)(it % r.parts), last = list[l][1];
    const int at_it = chunk_at<T>(r, ((int)(it / r.parts) << r.join_log2) + lane);
    double sum[VE];
    if (at_it >= 0) add(first, first + sub, subs, last, at_it, sum);
#pragma unroll
    for (int i = 0; i < VE; ++i) sums[i * kJoinBlock + threadIdx.x] = at_it >= 0 ? sum[i] : 0.0;
    for (int d = subs / 2; d; d >>= 1) {
      __syncthreads();
      if (sub < d)
#pragma unroll
        for (int i = 0; i < VE; ++i) sums[i * kJoinBlock + threadIdx.x] += sums[i * kJoinBlock + threadIdx.x + (d << r.join_log2)];
    }
    __syncthreads();
    if (sub == 0 && at_it >= 0) {
#pragma unroll
      for (int i = 0; i < VE; ++i) sum[i] = sums[i * kJoinBlock + threadIdx.x];
      write_row<TD>(dtable + list[l][2] * ldt, at_it, narrow, sum, scale);
    }
    __syncthreads();
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
  // About 4,096 wavefronts in all; 2,048, two to a SIMD, where ids have many tokens,
  // since of long runs every part is read again when they are joined (runs and joins
  // of 494,073 float16 rows of 240 for 21 ids 85 us; with 1,536 wavefronts 93, with 3,072
  // 88).  8 to 1,024 rows to a part, 32 and more where a row takes a wavefront.
  const int lanes = 1 << l.lanes_log2, least = lanes / 2 < 8 ? 8 : lanes / 2;
  const int64_t all = (int64_t)(ntok / nid >= 256 ? 2048 : 4096) * 64;
  const int64_t part = ((int64_t)ntok * l.slabs * lanes + all - 1) / all;
  l.part = (int)(part < least ? least : part > 1024 ? 1024 : part);
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
  l.sort = take(sort_workspace_bytes<IdJob>(ntok, 1 << l.passes.bits));
  l.partial = take((size_t)l.parts * 2 * width * sizeof(double));
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
  const size_t es = elem_size(elem);
  const int l = log2_lanes(width, es);
  const int64_t per = (int64_t)(kBlock >> l) * kRowsAtOnce;
  const bool once = (int64_t)ntok * width * (int64_t)es >= kOnceBytes && width * es % 16 == 0 && ldy * es % 16 == 0 &&
                    elem_aligned(y, 16);
  const int64_t nch = (int64_t)width * es / 16, chunks = ntok * nch;
  if (width * es % 16 == 0 && ldy == width && chunks < (int64_t)1 << 31) {
    by_elem(elem, [&](auto tt) {
      typedef decltype(tt) T;
      hipLaunchKernelGGL((once ? embed_flat_kernel<T, true> : embed_flat_kernel<T, false>),
                         dim3((unsigned)((chunks + kBlock * kFlat - 1) / (kBlock * kFlat))), dim3(kBlock), 0,
                         static_cast<hipStream_t>(stream), (unsigned)chunks, (unsigned)nch, 1.0 / (double)nch, nid, ids,
                         (const T*)table, ldt, (typename ElemAcc<T>::type)scale, (T*)y);
    });
    return dpc_internal_launch_status();
  }
  by_elem(elem, [&](auto tt) {
    typedef decltype(tt) T;
    hipLaunchKernelGGL((once ? embed_kernel<T, true> : embed_kernel<T, false>), rows_grid((ntok + per - 1) / per),
                       dim3(kBlock), 0, static_cast<hipStream_t>(stream), ntok, nid, width, l, ids, (const T*)table, ldt,
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
  const int most_log2 = elem_size(elem) == 8 ? 3 : 2;
  const int join_log2 = l.lanes_log2 < most_log2 ? l.lanes_log2 : most_log2;
  const int chunk = (int)(16 / elem_size(elem)), nch = width < chunk ? width : (width + chunk - 1) / chunk;
  const int64_t join_slabs = ((int64_t)nch + (1 << join_log2) - 1) >> join_log2;
  // Zeros: 64 rows of ids to a wavefront, and as many of their columns as makes about
  // kZeroWaves of them (21 float32 rows of 6,920 for 258 ids 15 us; whole rows 68).
  const int64_t id_waves = ((int64_t)nid + 63) / 64, VE = 16 / (int64_t)elem_size(elem_d), units = (width + 64 * VE - 1) / (64 * VE);
  const int64_t cuts = id_waves < kZeroWaves ? kZeroWaves / id_waves : 1;
  const int64_t zero_units = (units + cuts - 1) / cuts;
  const int zero_slabs = (int)((units + zero_units - 1) / zero_units);
  const Runs r{id, tok, left, nid, width, l.part, l.parts, l.slabs, l.lanes_log2, (int)join_slabs, join_log2, zero_slabs,
               (int)(zero_units * 64)};
  const int64_t threads = ((int64_t)l.parts * l.slabs) << l.lanes_log2;
  const unsigned run_blocks = (unsigned)((threads + kBlock - 1) / kBlock);
  const unsigned absent_blocks = (unsigned)((id_waves * zero_slabs + kBlock / 64 - 1) / (kBlock / 64));
  by_elem(elem, [&](auto tt) {
    typedef decltype(tt) T;
    const auto go = [&](auto dd) {
      typedef decltype(dd) TD;
      double* partial = reinterpret_cast<double*>(ws + l.partial);
      hipLaunchKernelGGL((width < Chunk<T>::kElems ? runs_kernel<T, TD, kNarrow>
                          : l.lanes_log2 == 6        ? runs_kernel<T, TD, kWide>
                                                     : runs_kernel<T, TD, kChunks>),
                         dim3(run_blocks + absent_blocks), dim3(kBlock), 0, s, r, run_blocks, (const T*)dy, lddy, scale,
                         partial, (TD*)dtable, lddt);
      if (l.parts > 1)
        hipLaunchKernelGGL((join_kernel<T, TD>), dim3((unsigned)((((l.parts * join_slabs) << join_log2) + kJoinBlock - 1) / kJoinBlock)), dim3(kJoinBlock),
                           0, s, r, scale, partial, (TD*)dtable, lddt);
    };
    if (elem_d == elem) go(T{});
    else go(float{});
  });
  return dpc_internal_launch_status();
}
