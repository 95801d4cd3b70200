// Layers in microscaled 4-bit floating point (dpc_quant_mx4, dpc_values_mx4,
// dpc_matmul_mx4, dpc_linear_mx4).
//
// Codes: a block of 32 elements is held by 4 lanes, 8 in each; its scale follows
// from its own largest magnitude, so that a row is read once, in any order.  Bound by
// HBM bandwidth: 32,768 bfloat16 rows of 4,096 65 us (5.2 TB/s), 1,048,576 float32 rows
// of 1,600 1,540 (5.0); one row 2.5 us.  Their values back in 52 us (6.6 TB/s).
//
// Product: y[r][c] = sum_i xq[t][i] wq[g][c][i] + bias[g][c] on the matrix cores,
// which take 128 columns of codes and the scales of their 4 blocks at a time.  A
// step is 256 columns, 128 bytes of codes and 8 of scales of a row.  Which block
// stands in which lane of a product is free as long as both sides agree: quarter q
// of the lanes takes blocks 2 q and 2 q + 1 of the step in its two products, whose
// scales are neighbouring bytes.  W's rows are the rows and x's rows the columns of
// a tile: a lane of a result holds four channels of one row of y.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "dpc.h"
#include "dpc_elem.h"
#include "dpc_groups.h"
#include "dpc_internal.h"
#include "dpc_mx4_tiles.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30;      // rows of codes
constexpr int64_t kMaxProduct = (int64_t)1 << 27;   // rows of a product (a launch has under 2^32 threads)
constexpr int kMaxChannels = 1 << 24;
constexpr int kBlock = 256;
constexpr int64_t kOnceBytes = (int64_t)192 << 20;  // rows of that size are written past the caches

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// codes
// ---------------------------------------------------------------------------
// The scale byte of a block whose largest magnitude (as float32) is a, and the
// scale as a number, 0 where the codes are 0.
__device__ __forceinline__ unsigned scale_byte(float a, float* scale) {
  const unsigned bits = __float_as_uint(a);
  unsigned e = ((bits + (1u << 21)) >> 23) - 2;  // rounded up from 1.75 on
  const bool finite = bits < 0x7f800000u, live = finite && a >= 0x1p-100f;
  *scale = live ? __uint_as_float(e << 23) : 0.0f;
  return live ? e : finite ? 0u : 255u;
}

// The largest of magnitudes, NaN if one is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The same over the 4 lanes of a block.
__device__ __forceinline__ float block_max(float a) {
  a = larger(a, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(a), 0xb1, 0xf, 0xf, false)));  // lanes 1 0 3 2
  return larger(a, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(a), 0x4e, 0xf, 0xf, false)));  // 2 3 0 1
}

// 8 elements to 8 codes.
__device__ __forceinline__ unsigned codes_of(const float (&v)[8], float scale) {
  unsigned q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], scale, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], scale, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], scale, 2);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], scale, 3);
  return scale > 0.0f ? q : 0u;
}

// The scale byte of the block of these 4 lanes, and the scale as a number.
__device__ __forceinline__ unsigned code_step(const float (&v)[8], float* factor) {
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = larger(a, __builtin_fabsf(v[i]));
  return scale_byte(block_max(a), factor);
}

// 8 elements of a row of `ncols` from column c on, zeros past its end.
template <typename T>
__device__ __forceinline__ void take8(const T* px, int c, int ncols, float (&v)[8]) {
  if (c + 8 <= ncols) {
    T t[8];
    __builtin_memcpy(t, px + c, sizeof(t));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < ncols ? (float)px[c + i] : 0.0f;
  }
}

constexpr int kQuantSteps = 4;  // steps of a row that 32 lanes take

// 8 rows to a workgroup, kQuantSteps steps of each.  Rows go on in z: one
// dimension of a launch has under 2^32 threads.
constexpr int64_t kWide = 1 << 22;
dim3 rows_grid(int64_t rows, int ncols) {
  const int64_t blocks = (rows + kBlock / 32 - 1) / (kBlock / 32), wide = blocks < kWide ? blocks : kWide;
  const int steps = DPC_MX4_LD(ncols) / 256;
  return dim3((unsigned)wide, (unsigned)((steps + kQuantSteps - 1) / kQuantSteps), (unsigned)((blocks + wide - 1) / wide));
}
__device__ __forceinline__ int64_t row_of_lane() {
  return (blockIdx.z * (int64_t)gridDim.x + blockIdx.x) * (kBlock / 32) + threadIdx.x / 32;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void quant_kernel(int64_t nrows_all, int nrows, int ncols, const T* __restrict__ x,
                                                       int64_t ldx, uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
  const int lane = threadIdx.x & 31, steps = DPC_MX4_LD(ncols) / 256;
  const int64_t r = row_of_lane();
  if (r >= nrows_all) return;
  const int s0 = blockIdx.y * kQuantSteps;
  const int64_t group = r / nrows, row = r - group * nrows;
  const T* px = x + r * ldx;
  float v[kQuantSteps][8];
#pragma unroll
  for (int k = 0; k < kQuantSteps; ++k) take8(px, (s0 + k) * 256 + lane * 8, ncols, v[k]);
#pragma unroll
  for (int k = 0; k < kQuantSteps; ++k) {
    if (s0 + k >= steps) break;
    float factor;
    const unsigned e = code_step(v[k], &factor);
    *reinterpret_cast<unsigned*>(q + (r * steps + s0 + k) * 128 + lane * 4) = codes_of(v[k], factor);
    if ((lane & 3) == 0) scale[((group * steps + s0 + k) * nrows + row) * 8 + (lane >> 2)] = (uint8_t)e;
  }
}

// Values: a lane makes chunks of 16 bytes, kChunks of a row on their way; 2^lanes_log2
// lanes to a row, so that neighbouring lanes write neighbouring chunks.
constexpr int kChunks = 4;

template <typename T, bool ONCE>
__global__ __launch_bounds__(kBlock) void values_kernel(int64_t nrows_all, int nrows, int ncols, int lanes_log2,
                                                        const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale,
                                                        T* __restrict__ y, int64_t ldy) {
  constexpr int VE = Chunk<T>::kElems;
  typedef std::conditional_t<VE == 8, unsigned, std::conditional_t<VE == 4, uint16_t, uint8_t>> Codes;
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1), steps = DPC_MX4_LD(ncols) / 256;
  const int64_t r = (blockIdx.z * (int64_t)gridDim.x + blockIdx.x) * (kBlock >> lanes_log2) + (threadIdx.x >> lanes_log2);
  if (r >= nrows_all) return;
  const int64_t group = r / nrows, row = r - group * nrows;
  const int c0 = (int)blockIdx.y * kChunks * lanes + lane, nch = (ncols + VE - 1) / VE;
  unsigned code[kChunks], e[kChunks];
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    const int at = min(c0 + k * lanes, nch - 1) * VE;  // first column
    code[k] = *reinterpret_cast<const Codes*>(q + r * steps * 128 + at / 2);
    e[k] = scale[((group * steps + at / 256) * nrows + row) * 8 + at / 32 % 8];
  }
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    const int at = (c0 + k * lanes) * VE;
    if (at >= ncols) break;
    // 2^(E - 127): in float32 a number below the least normal one for E = 0
    typename ElemAcc<T>::type f;
    if constexpr (sizeof(T) == 8) f = __longlong_as_double(e[k] == 255 ? 0x7ff8000000000000ll : (long long)(e[k] + 896) << 52);
    else f = __uint_as_float(e[k] == 0 ? 0x00400000u : e[k] == 255 ? 0x7fc00000u : e[k] << 23);
    Chunk<T> out;
#define DPC_PAIR(p)                                                             \
  if constexpr (2 * p < VE) {                                                   \
    const v2f two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[k], 1.0f, p); \
    out.v[2 * p] = (T)(two[0] * f);                                             \
    out.v[2 * p + 1] = (T)(two[1] * f);                                         \
  }
    DPC_PAIR(0) DPC_PAIR(1) DPC_PAIR(2) DPC_PAIR(3)
#undef DPC_PAIR
    T* py = y + r * ldy + at;
    if (at + VE <= ncols) {
      if (ONCE) out.store_once(py);
      else out.store(py);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (at + i < ncols) py[i] = out.v[i];
    }
  }
}

// Calls f with a value of the element type.
template <typename F>
int by_elem(dpc_elem elem, F f) {
  (void)hipGetLastError();  // report only what this launch raises
  switch (elem) {
    case DPC_ELEM_F64: f(double{}); break;
    case DPC_ELEM_F32: f(float{}); break;
    case DPC_ELEM_F16: f(_Float16{}); break;
    default: f(__bf16{}); break;
  }
  return dpc_internal_launch_status();
}

int quant(hipStream_t s, dpc_elem elem, int ngroup, int nrows, int ncols, const void* x, int64_t ldx, uint8_t* q,
          uint8_t* scale) {
  const int64_t rows = (int64_t)ngroup * nrows;
  return by_elem(elem, [&](auto t) {
    typedef decltype(t) T;
    hipLaunchKernelGGL(quant_kernel<T>, rows_grid(rows, ncols), dim3(kBlock), 0, s, rows, nrows, ncols, (const T*)x, ldx, q,
                       scale);
  });
}

// ---------------------------------------------------------------------------
// product
// ---------------------------------------------------------------------------
struct Product {
  int ntok, topk, m, n, k, steps, ngroup;
  const uint8_t* qx;
  const uint8_t* sx;
  const int* rows;
  const int* offsets;
  const uint8_t* qw;
  const uint8_t* sw;
  const float* bias;
};

// Tiles of `size` rows that find_tile can be asked for.
inline int64_t most_tiles(const Product& p, int size) { return mx4_most_tiles(p.m, p.ngroup, p.offsets != nullptr, size); }

inline bool few_rows(const Product& p) { return mx4_few_rows(p.m, p.n, p.ngroup, p.offsets != nullptr); }

// One product of 16 rows of W and 16 rows of x, 128 columns: codes a and b of this
// lane's block, whose scale is byte K of sa and sb.
template <int K>
__device__ __forceinline__ v4f mfma4(v4i a, v4i b, v4f c, int sa, int sb) {
  const v8i a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, K, sa, K, sb);
}

// Where chunk c of the 8 of row r lies in LDS, and the chunk that lies in slot `slot`
// of it: even chunks first, since the lanes of one read take chunks 0, 2, 4, 6 or
// 1, 3, 5, 7 of 16 rows, then turned with the row, so that 8 lanes that read at once
// meet all banks.  In order, c ^ (r & 7), half of a read's clocks were conflicts:
// 270 us for 265 at 8192 x 8192 x 8192, 10.3 for 9.8 at 2048 x 2048 x 2048.
__device__ __forceinline__ int place_of(int c, int r) { return ((c >> 1 | (c & 1) << 2) ^ (r & 7)) << 4; }
__device__ __forceinline__ int chunk_at(int slot, int r) {
  const int c = slot ^ (r & 7);
  return (c & 3) << 1 | c >> 2;
}

template <typename TY>
__device__ __forceinline__ TY result(float sum, float bias) {
  float f = sum + bias;
  if constexpr (sizeof(TY) == 2) asm("" : "+v"(f));  // the sum is rounded to float32 before
  return (TY)f;
}

// Few rows: 16 rows times 16 channels of y for each `share` wavefronts of a
// workgroup of 8, which take the steps of K in turn and whose sums are added in
// LDS, in order.  W is read once for each 16 rows of an expert, up to 8 KiB of it
// under way in every wavefront: bound by that read, or for short rows by latency.
// TX is the type of rows that the workgroup codes itself (into LDS), or uint8_t for
// rows that are codes already.
constexpr int kFewWaves = 8, kFewAhead = 4;

template <typename TX, typename TY>
__global__ __launch_bounds__(64 * kFewWaves) void few_product_kernel(Product p, int share, const TX* __restrict__ x,
                                                                     int64_t ldx, TY* __restrict__ y, int64_t ldy) {
  constexpr bool kCoded = sizeof(TX) == 1;
  extern __shared__ __attribute__((aligned(16))) uint8_t codes[];  // codes made here [rows][steps][128], then scales [steps][rows][8]
  __shared__ float sums[kFewWaves][256];
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile t = find_tile(p, 16, blockIdx.y + gridDim.y * blockIdx.z);
  if (t.row0 >= t.end) return;
  const int tiles = kFewWaves / share;  // channel tiles of the workgroup
  const int c0 = (blockIdx.x * tiles + wave / share) * 16, part = wave % share;
  const int steps = p.steps, group = max(t.group, 0), high = t.end - t.row0;
  // Codes: 4 lanes to 64 bytes of a row, moved to the lanes of a product by to_rows;
  // in the first load of a step the even chunks, in the second the odd ones.
  const uint8_t* pw = p.qw + ((int64_t)group * p.n + min(c0 + (lane >> 2), p.n - 1)) * steps * 128 + (lane & 3) * 32;
  const uint8_t* psw = p.sw + ((int64_t)group * steps * p.n + min(c0 + l16, p.n - 1)) * 8 + quad * 2;
  auto token = [&](int r) __attribute__((always_inline)) { return t.group < 0 ? -1 : token_of(p, min(t.row0 + r, t.end - 1)); };
  const uint8_t *pq = nullptr, *psq = nullptr;
  if (kCoded) {
    pq = (const uint8_t*)x + (int64_t)max(token(lane >> 2), 0) * steps * 128 + (lane & 3) * 32;
    psq = p.sx + (int64_t)max(token(l16), 0) * 8 + quad * 2;
  }
  v4i w[kFewAhead][2], q[kFewAhead][2];
  int ew[kFewAhead], eq[kFewAhead];
  auto fetch = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int s = min(s0 + u * share, steps - 1);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        w[u][k] = *reinterpret_cast<const v4i*>(pw + s * 128 + k * 16);
        if (kCoded) q[u][k] = *reinterpret_cast<const v4i*>(pq + s * 128 + k * 16);
      }
      ew[u] = *reinterpret_cast<const uint16_t*>(psw + (int64_t)s * p.n * 8);
      if (kCoded) eq[u] = *reinterpret_cast<const uint16_t*>(psq + (int64_t)s * p.ntok * 8);
    }
  };
  fetch(part);
  const int held = min(high, 16);
  const uint8_t* scales = codes + held * steps * 128;
  if constexpr (!kCoded) {
    // 32 lanes to a step of a row, as in quant_kernel
    const int l32 = threadIdx.x & 31, chunk = l32 >> 2;
    int row = 0, s = threadIdx.x >> 5;
    for (;; s += 64 * kFewWaves / 32) {
      for (; s >= steps && row < held; ++row) s -= steps;
      if (row >= held) break;
      float v[8], factor;
      take8(x + (int64_t)max(token(row), 0) * ldx, s * 256 + l32 * 8, p.k, v);
      const unsigned e = code_step(v, &factor);
      *reinterpret_cast<unsigned*>(codes + (row * steps + s) * 128 + place_of(chunk, row) + (l32 & 3) * 4) = codes_of(v, factor);
      if ((l32 & 3) == 0) codes[held * steps * 128 + (s * held + row) * 8 + chunk] = (uint8_t)e;
    }
    __syncthreads();
  }
  const int mine = min(l16, held - 1);  // rows of the tile past its end repeat its last one
  v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = part; s0 < steps; s0 += share * kFewAhead) {
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int s = s0 + u * share;
      if (s >= steps) break;
      v4i b[2];
      int e;
      if constexpr (kCoded) {
#pragma unroll
        for (int k = 0; k < 2; ++k) b[k] = to_rows(q[u][k]);
        e = eq[u];
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          b[k] = *reinterpret_cast<const v4i*>(codes + (mine * steps + s) * 128 + place_of(quad * 2 + k, mine));
        e = *reinterpret_cast<const uint16_t*>(scales + (s * held + mine) * 8 + quad * 2);
      }
      acc = mfma4<0>(to_rows(w[u][0]), b[0], acc, ew[u], e);
      acc = mfma4<1>(to_rows(w[u][1]), b[1], acc, ew[u], e);
    }
    if (s0 + share * kFewAhead < steps) fetch(s0 + share * kFewAhead);
  }
  // this lane: row l16, channels 4 quad .. 4 quad + 3
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[wave][l16 * 16 + quad * 4 + i] = acc[i];
  __syncthreads();
  for (int e = threadIdx.x; e < tiles * 256; e += 64 * kFewWaves) {
    const int tile = e >> 8, row = e >> 4 & 15, c = (blockIdx.x * tiles + tile) * 16 + (e & 15), r = t.row0 + row;
    if (r >= t.end || c >= p.n) continue;
    float sum = 0.0f;
    for (int v = 0; v < share; ++v) sum += sums[tile * share + v][e & 255];
    y[(int64_t)r * ldy + c] = token(row) < 0 ? (TY)0 : result<TY>(sum, p.bias ? p.bias[(int64_t)group * p.n + c] : 0.0f);
  }
}

// LDS of rows that the workgroup codes.
inline size_t few_bytes(const Product& p) { return (size_t)(p.m < 16 ? p.m : 16) * p.steps * 136; }

template <typename TX, typename TY>
void launch_few(hipStream_t s, const Product& p, const TX* x, int64_t ldx, TY* y, int64_t ldy) {
  const int64_t tiles = most_tiles(p, 16);
  const unsigned gy = (unsigned)(tiles < 32768 ? tiles : 32768);
  // wavefronts that share a tile: about 16 in all for each of 256 CUs
  const int64_t wide = (p.n + 15) / 16;
  int share = kFewWaves;
  while (share > 1 && wide * tiles * share > 4096) share /= 2;
  hipLaunchKernelGGL((few_product_kernel<TX, TY>),
                     dim3((unsigned)((wide * share + kFewWaves - 1) / kFewWaves), gy, (unsigned)((tiles + gy - 1) / gy)),
                     dim3(64 * kFewWaves), sizeof(TX) == 1 ? 0 : few_bytes(p), s, p, share, x, ldx, y, ldy);
}

// Tiles of BM rows times BN channels, K in steps of 256 columns: codes and scales
// of both operands go from memory to LDS without passing registers, the next
// step's while the matrix cores work on this one's.  A row of a step is 8 chunks of
// 16 bytes, one block each; where each lies, place_of says.  The scales of a
// row are 8 bytes in a row, of which a lane reads the two of its chunks.
//
// 8192 x 8192 x 8192 in 257 to 276 us late in a row of 3,000 (4.0 to 4.3e15 operations a
// second; random codes in registers alone 7.2e15: 153 us), 269 to 374 in the first 23 of
// a row, 274 to 298 one by one with pauses; 32,768 rows for 16 experts' 4096 x 4096 333
// to 378 past the first 50, 364 to 486 in the first 23, 383 to 408 with pauses.  Of 285
// us the products alone take 196: the largest tile's reads (1,024 clocks a step), loads
// (512) and products (2,048) overlap in part.  Tried without gain: reads in the order of
// use one to three fragments ahead (287 to 292), the next half step's while this one is
// multiplied (451: spills), four wavefronts of 128 x 128 (297), 64 x 128 (398), workgroups
// that go on to their next tile with its first step under way (298: spills).
template <typename TY, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void product_tiled_kernel(Product p, int col_tiles, TY* __restrict__ y,
                                                                     int64_t ldy) {
  constexpr int VE = 16 / sizeof(TY);
  constexpr int kWaves = WM * WN, TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
  constexpr int kStep = 128, kRows = BM + BN;
  constexpr int kLoads = kRows / 8 / kWaves;       // 8 rows of codes each
  constexpr int kScaleLoads = (kRows / 32 + kWaves - 1) / kWaves;  // 32 rows of scales each
  static_assert(kLoads * kWaves * 8 == kRows && kRows % 32 == 0, "every load is whole");
  // codes, then scales: of two arrays the compiler would wait for every load before
  // it reads one
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][kRows * (kStep + 8)];
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;

  // consecutive workgroups go to different XCDs: each XCD gets a run of tiles
  // of its own, in bands of 8 row tiles, so that its L2 serves tiles that share
  // rows; the runs are cut from the tiles that exist, for equal work
  const int row_tiles = count_tiles(p, BM);
  const int total = row_tiles * col_tiles, per = (total + 7) / 8;
  const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= total) return;
  const int band = id / (8 * col_tiles), in = id - band * 8 * col_tiles;
  const int high = min(8, row_tiles - band * 8);
  const int ct = in / high, rt = band * 8 + in % high;

  const Tile t = find_tile(p, BM, rt);
  if (t.row0 >= t.end) return;
  const int c0 = ct * BN;

  if (t.group < 0) {  // rows of no expert
    const int high_rows = t.end - t.row0, wide = min(BN, p.n - c0);
    for (int e = threadIdx.x; e < high_rows * wide; e += 64 * kWaves)
      y[(int64_t)(t.row0 + e / wide) * ldy + c0 + e % wide] = (TY)0;
    return;
  }

  v4f acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  // this lane's rows of the loads: x rows first, then rows of W
  const uint8_t* src[kLoads];
  int dst[kLoads];
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int r8 = (wave * kLoads + l) * 8, r = r8 + (lane >> 3);
    const int chunk = chunk_at(lane & 7, r < BM ? r : turn_of<VE>(r));
    const uint8_t* row;
    if (r < BM) {
      const int tok = token_of(p, min(t.row0 + r, t.end - 1));
      row = p.qx + (int64_t)(tok < 0 ? 0 : tok) * p.steps * kStep;
    } else {
      row = p.qw + ((int64_t)t.group * p.n + min(c0 + r - BM, p.n - 1)) * p.steps * kStep;
    }
    src[l] = row + chunk * 16;
    dst[l] = r8 * kStep;
  }
  // and of the scales: 4 bytes each, two lanes to a row
  const uint8_t* ssrc[kScaleLoads];
  int64_t sstep[kScaleLoads];
#pragma unroll
  for (int l = 0; l < kScaleLoads; ++l) {
    const int r = min((l * kWaves + wave) * 32, kRows - 32) + (lane >> 1);
    if (r < BM) {
      const int tok = token_of(p, min(t.row0 + r, t.end - 1));
      ssrc[l] = p.sx + (int64_t)(tok < 0 ? 0 : tok) * 8;
      sstep[l] = (int64_t)p.ntok * 8;
    } else {
      ssrc[l] = p.sw + ((int64_t)t.group * p.steps * p.n + min(c0 + r - BM, p.n - 1)) * 8;
      sstep[l] = (int64_t)p.n * 8;
    }
    ssrc[l] += (lane & 1) * 4;
  }
  auto fetch = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      __builtin_amdgcn_global_load_lds((GlobalPtr)src[l], (LdsPtr)(&lds[buf][dst[l]]), 16, 0, 0);
      src[l] += kStep;
    }
#pragma unroll
    for (int l = 0; l < kScaleLoads; ++l) {
      const int r32 = l * kWaves + wave;  // of every wavefront there is one, of some there may be one more
      if (r32 * 32 < kRows) __builtin_amdgcn_global_load_lds((GlobalPtr)ssrc[l], (LdsPtr)(&lds[buf][kRows * kStep + r32 * 256]), 4, 0, 0);
      ssrc[l] += sstep[l];
    }
  };
  fetch(0);
  for (int s = 0; s < p.steps; ++s) {
    // vmcnt(0), lgkmcnt(0): this step's rows are in LDS, the step before has
    // been read; the barrier says so for every wavefront
    __builtin_amdgcn_s_waitcnt(0x0070);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + 1 < p.steps) fetch((s + 1) & 1);
    const uint8_t* xs = &lds[s & 1][wm * TM * kStep];
    const uint8_t* ws = &lds[s & 1][(BM + wn * TN) * kStep];
    const uint8_t* xe = &lds[s & 1][kRows * kStep + wm * TM * 8 + quad * 2];
    const uint8_t* we = &lds[s & 1][kRows * kStep + (BM + wn * TN) * 8 + quad * 2];
    v4i a[2][NI], b[2][MI];
    int ea[NI], eb[MI];
#pragma unroll
    for (int j = 0; j < NI; ++j)
      ea[j] = *reinterpret_cast<const uint16_t*>(we + (channel_of<VE>(j, 0) + channel_of<VE>(0, l16)) * 8);
#pragma unroll
    for (int i = 0; i < MI; ++i) eb[i] = *reinterpret_cast<const uint16_t*>(xe + (i * 16 + l16) * 8);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int slot = place_of(quad * 2 + k, l16);
#pragma unroll
      for (int j = 0; j < NI; ++j)
        a[k][j] = *reinterpret_cast<const v4i*>(ws + (channel_of<VE>(j, 0) + channel_of<VE>(0, l16)) * kStep + slot);
#pragma unroll
      for (int i = 0; i < MI; ++i) b[k][i] = *reinterpret_cast<const v4i*>(xs + (i * 16 + l16) * kStep + slot);
    }
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mfma4<0>(a[0][j], b[0][i], acc[i][j], ea[j], eb[i]);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mfma4<1>(a[1][j], b[1][i], acc[i][j], ea[j], eb[i]);
    // LDS reads of the second half between the products of the first
    constexpr int kReads = NI + MI, kSpaced = 2 * kReads <= MI * NI ? 2 : 1;
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * kReads, 0);
#pragma unroll
    for (int q = 0; q < kReads; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, kSpaced, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 2 * MI * NI - kSpaced * kReads, 0);
    asm volatile("" ::: "memory");
  }

  // this lane's results: row l16 of each row tile, runs of VE channels from
  // first, first + 4 VE, ...
  constexpr int kRuns = NI * 4 / VE;
  const int first = c0 + wn * TN + quad * VE;
  const bool whole = c0 + BN <= p.n;
  float bias[kRuns][VE];
#pragma unroll
  for (int g = 0; g < kRuns; ++g)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int c = min(first + g * 4 * VE + e, p.n - 1);
      bias[g][e] = p.bias ? p.bias[(int64_t)t.group * p.n + c] : 0.0f;
    }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = t.row0 + wm * TM + i * 16 + l16;
    const int tok = token_of(p, min(r, t.end - 1));
    TY* py = y + (int64_t)r * ldy + first;
#pragma unroll
    for (int g = 0; g < kRuns; ++g) {
      TY out[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        out[e] = result<TY>(acc[i][(g * VE + e) / 4][(g * VE + e) % 4], bias[g][e]);
        if (tok < 0) out[e] = (TY)0;  // a row of the group that no slot owns
      }
      const int left = r >= t.end ? 0 : whole ? VE : p.n - (first + g * 4 * VE);
      put_run(py + g * 4 * VE, out, left);
    }
  }
}

template <typename TY, int BM, int BN, int WM, int WN>
void launch_tiled(hipStream_t s, const Product& p, TY* y, int64_t ldy) {
  const int col_tiles = (p.n + BN - 1) / BN;
  const unsigned per = ((unsigned)most_tiles(p, BM) * (unsigned)col_tiles + 7) / 8;
  hipLaunchKernelGGL((product_tiled_kernel<TY, BM, BN, WM, WN>), dim3(per * 8), dim3(64 * WM * WN), 0, s, p, col_tiles,
                     y, ldy);
}

template <typename TY>
void launch_product(hipStream_t s, const Product& p, TY* y, int64_t ldy) {
  if (few_rows(p)) return launch_few(s, p, p.qx, 0, y, ldy);
  switch (mx4_tile(p.m, p.n, p.steps, p.ngroup, p.offsets != nullptr)) {
    case 0: return launch_tiled<TY, 256, 256, 2, 4>(s, p, y, ldy);
    case 1: return launch_tiled<TY, 128, 128, 2, 2>(s, p, y, ldy);
    case 2: return launch_tiled<TY, 128, 64, 2, 2>(s, p, y, ldy);
    default: return launch_tiled<TY, 64, 64, 2, 2>(s, p, y, ldy);
  }
}

int product(hipStream_t s, dpc_elem elem_y, const Product& p, void* y, int64_t ldy) {
  return by_elem(elem_y, [&](auto t) { launch_product(s, p, (decltype(t)*)y, ldy); });
}

// Codes and product in one, for layers of few channels over many rows: the codes
// of kCodedRows rows pass through LDS step by step and never see memory.  While a
// step is coded and multiplied, the next one's elements are on their way to
// registers.  Wavefront w makes channels 32 w .. 32 w + 31, with W's rows straight
// from L2 (every workgroup reads all of W).  Chunks of codes lie as in the tiles above.
constexpr int kCodedRows = 32, kCodedWaves = 8;

// A lane's 8 results of a row in the type of y, runs at c, c + 4 VE, ... of n.
template <typename TY>
__device__ __forceinline__ void put_row(TY* y, int c, int n, const v4f (&acc)[2], const float (&bias)[8], bool exists, bool owned) {
  constexpr int VE = 16 / sizeof(TY);
#pragma unroll
  for (int g = 0; g < 8 / VE; ++g) {
    TY out[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int at = g * VE + e;
      out[e] = owned ? result<TY>(acc[at / 4][at % 4], bias[at]) : (TY)0;
    }
    put_run(y + c + g * 4 * VE, out, exists ? n - c - g * 4 * VE : 0);
  }
}

template <typename TX>
__global__ __launch_bounds__(64 * kCodedWaves, 4) void coded_product_kernel(Product p, dpc_elem elem_y, const TX* __restrict__ x,
                                                                            int64_t ldx, void* __restrict__ y, int64_t ldy) {
  constexpr int kRows = kCodedRows, MI = kRows / 16, kPass = kRows * 32 / (64 * kCodedWaves);  // rows that 32 lanes code
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][kRows * 136];          // codes, then scales
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile t = find_tile(p, kRows, blockIdx.x);
  if (t.row0 >= t.end) return;
  const int steps = p.steps, group = max(t.group, 0);
  const int ve = elem_y == DPC_ELEM_F64 ? 2 : elem_y == DPC_ELEM_F32 ? 4 : 8;
  auto channel = [&](int j, int r) __attribute__((always_inline)) {
    return ve == 2 ? channel_of<2>(j, r) : ve == 4 ? channel_of<4>(j, r) : channel_of<8>(j, r);
  };
  // 32 lanes to a row: rows half, half + 16, ...
  const int half = threadIdx.x >> 5, l32 = threadIdx.x & 31;
  const TX* px[kPass];
#pragma unroll
  for (int a = 0; a < kPass; ++a) {
    const int tok = t.group < 0 ? -1 : token_of(p, min(t.row0 + half + 16 * a, t.end - 1));
    px[a] = x + (int64_t)max(tok, 0) * ldx + l32 * 8;
  }
  const uint8_t *pw[2], *psw[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    pw[j] = p.qw + ((int64_t)group * p.n + min(wave * 32 + channel(j, lane >> 2), p.n - 1)) * steps * 128 + (lane & 3) * 32;
    psw[j] = p.sw + ((int64_t)group * steps * p.n + min(wave * 32 + channel(j, l16), p.n - 1)) * 8 + quad * 2;
  }
  const bool work = wave * 32 < p.n;  // this wavefront has channels
  auto take = [&](int s, TX (&held)[kPass][8]) __attribute__((always_inline)) {
    if (s * 256 + 256 <= p.k) {
#pragma unroll
      for (int a = 0; a < kPass; ++a)
#pragma unroll
        for (int c = 0; c < 8; c += Chunk<TX>::kElems) {
          Chunk<TX> ch;
          ch.load_once(px[a] + s * 256 + c);
#pragma unroll
          for (int i = 0; i < Chunk<TX>::kElems; ++i) held[a][c + i] = ch.v[i];
        }
    } else {
#pragma unroll
      for (int a = 0; a < kPass; ++a)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = s * 256 + l32 * 8 + i;
          const TX v = px[a][min(c, p.k - 1) - l32 * 8];
          held[a][i] = c < p.k ? v : (TX)0;
        }
    }
  };
  v4f acc[MI][2];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  TX held[kPass][8];
  take(0, held);
  for (int s = 0; s < steps; ++s) {
    uint8_t* to = lds[s & 1];
    v4i w[2][2];
    int ew[2];
    if (work) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int k = 0; k < 2; ++k) w[k][j] = *reinterpret_cast<const v4i*>(pw[j] + s * 128 + k * 16);
        ew[j] = *reinterpret_cast<const uint16_t*>(psw[j] + (int64_t)s * p.n * 8);
      }
    }
#pragma unroll
    for (int a = 0; a < kPass; ++a) {
      const int row = half + 16 * a, chunk = l32 >> 2;
      float v[8], factor;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)held[a][i];
      const unsigned e = code_step(v, &factor);
      *reinterpret_cast<unsigned*>(to + row * 128 + place_of(chunk, row) + (l32 & 3) * 4) = codes_of(v, factor);
      if ((l32 & 3) == 0) to[kRows * 128 + row * 8 + chunk] = (uint8_t)e;
    }
    if (s + 1 < steps) take(s + 1, held);
    // the codes of this step are written (its buffer was read two steps ago, before
    // the barrier in between); loads stay under way
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (!work) continue;
    v4i a[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j) a[k][j] = to_rows(w[k][j]);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int row = i * 16 + l16;
      const int ex = *reinterpret_cast<const uint16_t*>(to + kRows * 128 + row * 8 + quad * 2);
      const v4i b0 = *reinterpret_cast<const v4i*>(to + row * 128 + place_of(quad * 2, l16));
      const v4i b1 = *reinterpret_cast<const v4i*>(to + row * 128 + place_of(quad * 2 + 1, l16));
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        acc[i][j] = mfma4<0>(a[0][j], b0, acc[i][j], ew[j], ex);
        acc[i][j] = mfma4<1>(a[1][j], b1, acc[i][j], ew[j], ex);
      }
    }
  }
  if (!work) return;
  float bias[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int c = min(wave * 32 + channel(q / 4, quad * 4 + q % 4), p.n - 1);
    bias[q] = p.bias ? p.bias[(int64_t)group * p.n + c] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = t.row0 + i * 16 + l16, c = wave * 32 + quad * ve;
    const bool exists = r < t.end, owned = exists && t.group >= 0 && token_of(p, r) >= 0;
    auto put = [&](auto* py) __attribute__((always_inline)) {
      put_row(py + (int64_t)r * ldy, c, p.n, acc[i], bias, exists, owned);
    };
    switch (elem_y) {
      case DPC_ELEM_F64: put((double*)y); break;
      case DPC_ELEM_F32: put((float*)y); break;
      case DPC_ELEM_F16: put((_Float16*)y); break;
      default: put((__bf16*)y); break;
    }
  }
}

// Whether that kernel takes a layer: rows of 1,024 elements or more, so many of them
// that in two kernels the codes would leave the caches in between.  Times, us, 240
// channels, one kernel and two:
//   float32, 1,600 columns     8,192 rows 17.6 18.3, 32,768 60.1 52.0, 131,072 223 259, 1,048,576 1,824 2,025
//   bfloat16, 1,600 columns    8,192 rows 14.7 15.4, 32,768 40.7 39.7, 131,072 147 161, 1,048,576 1,138 1,223
//   bfloat16, 8,192 columns    8,192 rows 53.1 46.0, 16,384 75.6 107, 131,072 551 786
//   bfloat16, 240 columns      8,192 rows 7.1 7.7, 131,072 56.3 44.0, 1,048,576 465 342
//   float64, 1,600 columns     16,384 rows 74.7 46.4, 131,072 605 458
// Coding takes most of its instructions: with 64 rows to a workgroup (W moved to the
// lanes of a product half as often) registers spill (2,563 us in the first line), with
// two steps of elements under way it is no faster (1,920).
inline bool one_kernel(const Product& p, dpc_elem elem_x) {
  return p.topk == 1 && p.n <= 256 && p.k >= 1024 && (int64_t)p.m * p.k >= (int64_t)1 << 27 && elem_x != DPC_ELEM_F64 &&
         !few_rows(p);
}

// Whether every workgroup codes its rows itself, up to 16,384 elements of them (in
// steps of 256), which costs less than a launch.  Of experts the host knows the
// average alone: a tile is taken to have twice as many rows.  Device times, us, one
// kernel and two: 1 row of 1,600 float32 to 240 channels 3.7 and 5.9, 8 rows 4.8 and
// 6.1, 16 rows 6.4 and 6.3; 1 bfloat16 row of 4,096 to 4,096 4.2 and 6.5, 4 rows 5.4 and
// 6.8, 16 rows 10.2 and 6.9.
inline bool coded_inside(const Product& p) {
  const int most = p.m < 16 ? p.m : 16, likely = (2 * p.m + p.ngroup - 1) / p.ngroup;
  const int rows = p.offsets && likely < most ? likely : most;
  return few_rows(p) && rows * p.steps <= 64 && few_bytes(p) <= 65536;
}

int product_args(dpc_elem elem_y, int ntok, int topk, int n, int k, int ngroup) {
  if (!elem_ok(elem_y) || ntok < 0 || topk < 1 || n < 1 || k < 1 || ngroup < 1) return DPC_EINVAL;
  if (topk > DPC_MAX_TOPK || k > DPC_MAX_MX4_COLS || ngroup > DPC_MAX_EXPERTS || n > kMaxChannels ||
      (int64_t)ntok * topk > kMaxProduct)
    return DPC_ENOTSUP;
  return DPC_OK;
}

bool product_ptrs(dpc_elem elem_y, int topk, int n, int ngroup, const int* rows, const int* offsets, const uint8_t* qw,
                  const uint8_t* sw, const float* bias, const void* y, int64_t ldy) {
  if ((!rows && topk != 1) || (!offsets && ngroup != 1)) return false;
  return qw && sw && y && ldy >= n && elem_aligned(qw, 16) && elem_aligned(sw, 8) && elem_aligned(bias, 4) &&
         elem_aligned(rows, 4) && elem_aligned(offsets, 4) && elem_aligned(y, elem_size(elem_y));
}

int rows_args(dpc_elem elem, int ngroup, int nrows, int ncols) {
  if (!elem_ok(elem) || ngroup < 0 || nrows < 0 || ncols < 1) return DPC_EINVAL;
  if (ncols > DPC_MAX_MX4_COLS || (int64_t)ngroup * nrows > kMaxRows) return DPC_ENOTSUP;
  return DPC_OK;
}
bool rows_ptrs(dpc_elem elem, int ncols, const void* x, int64_t ldx, const uint8_t* q, const uint8_t* scale) {
  return x && q && scale && ldx >= ncols && elem_aligned(x, elem_size(elem)) && elem_aligned(q, 16) && elem_aligned(scale, 8);
}

}  // namespace

extern "C" int dpc_quant_mx4(void* stream, dpc_elem elem, int ngroup, int nrows, int ncols, const void* x, int64_t ldx,
                             uint8_t* q, uint8_t* scale) {
  const int st = rows_args(elem, ngroup, nrows, ncols);
  if (st != DPC_OK) return st;
  if (ngroup == 0 || nrows == 0) return DPC_OK;
  if (!rows_ptrs(elem, ncols, x, ldx, q, scale)) return DPC_EINVAL;
  return quant(static_cast<hipStream_t>(stream), elem, ngroup, nrows, ncols, x, ldx, q, scale);
}

extern "C" int dpc_values_mx4(void* stream, dpc_elem elem, int ngroup, int nrows, int ncols, const uint8_t* q,
                              const uint8_t* scale, void* y, int64_t ldy) {
  const int st = rows_args(elem, ngroup, nrows, ncols);
  if (st != DPC_OK) return st;
  if (ngroup == 0 || nrows == 0) return DPC_OK;
  if (!rows_ptrs(elem, ncols, y, ldy, q, scale)) return DPC_EINVAL;
  const int64_t rows = (int64_t)ngroup * nrows;
  const int es = (int)elem_size(elem), VE = 16 / es, nch = (ncols + VE - 1) / VE;
  int l = 0;
  while (l < 6 && (1 << l) * kChunks < nch) ++l;
  const int64_t blocks = (rows + (kBlock >> l) - 1) / (kBlock >> l), wide = blocks < kWide ? blocks : kWide;
  const dim3 grid((unsigned)wide, (unsigned)((nch + (kChunks << l) - 1) / (kChunks << l)), (unsigned)((blocks + wide - 1) / wide));
  const bool once = rows * ncols * es >= kOnceBytes && (int64_t)ncols * es % 16 == 0 && ldy * es % 16 == 0 && elem_aligned(y, 16);
  return by_elem(elem, [&](auto t) {
    typedef decltype(t) T;
    hipLaunchKernelGGL((once ? values_kernel<T, true> : values_kernel<T, false>), grid, dim3(kBlock), 0,
                       static_cast<hipStream_t>(stream), rows, nrows, ncols, l, q, scale, (T*)y, ldy);
  });
}

extern "C" int dpc_matmul_mx4(void* stream, dpc_elem elem_y, int ntok, int topk, int n, int k, int ngroup, const uint8_t* qx,
                              const uint8_t* sx, const int* rows, const int* offsets, const uint8_t* qw, const uint8_t* sw,
                              const float* bias, void* y, int64_t ldy) {
  const int st = product_args(elem_y, ntok, topk, n, k, ngroup);
  if (st != DPC_OK) return st;
  if (ntok == 0) return DPC_OK;
  if (!qx || !sx || !elem_aligned(qx, 16) || !elem_aligned(sx, 8) ||
      !product_ptrs(elem_y, topk, n, ngroup, rows, offsets, qw, sw, bias, y, ldy))
    return DPC_EINVAL;
  const Product p{ntok, topk, ntok * topk, n, k, DPC_MX4_LD(k) / 256, ngroup, qx, sx, rows, offsets, qw, sw, bias};
  return product(static_cast<hipStream_t>(stream), elem_y, p, y, ldy);
}

extern "C" size_t dpc_linear_mx4_workspace_bytes(int ntok, int k) {
  if (ntok < 0 || ntok > kMaxRows || k < 1 || k > DPC_MAX_MX4_COLS) return 0;
  return ((size_t)ntok * (DPC_MX4_LD(k) / 256) * 136 + 255) / 256 * 256 + 256;
}

extern "C" int dpc_linear_mx4(void* stream, dpc_elem elem_x, dpc_elem elem_y, int ntok, int topk, int n, int k, int ngroup,
                              const void* x, int64_t ldx, const int* rows, const int* offsets, const uint8_t* qw,
                              const uint8_t* sw, const float* bias, void* workspace, size_t workspace_bytes, void* y,
                              int64_t ldy) {
  const int st = product_args(elem_y, ntok, topk, n, k, ngroup);
  if (st != DPC_OK) return st;
  if (!elem_ok(elem_x)) return DPC_EINVAL;
  if (ntok == 0) return DPC_OK;
  if (!x || ldx < k || !elem_aligned(x, elem_size(elem_x)) || !workspace || !elem_aligned(workspace, 16) ||
      workspace_bytes < dpc_linear_mx4_workspace_bytes(ntok, k) ||
      !product_ptrs(elem_y, topk, n, ngroup, rows, offsets, qw, sw, bias, y, ldy))
    return DPC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int steps = DPC_MX4_LD(k) / 256;
  uint8_t* q = static_cast<uint8_t*>(workspace);
  uint8_t* scale = q + (size_t)ntok * steps * 128;
  const Product p{ntok, topk, ntok * topk, n, k, steps, ngroup, q, scale, rows, offsets, qw, sw, bias};
  if (coded_inside(p)) {
    return by_elem(elem_x, [&](auto tx) {
      by_elem(elem_y, [&](auto ty) { launch_few(s, p, (const decltype(tx)*)x, ldx, (decltype(ty)*)y, ldy); });
    });
  }
  if (one_kernel(p, elem_x)) {
    return by_elem(elem_x, [&](auto tx) {
      typedef std::conditional_t<sizeof(tx) == 8, float, decltype(tx)> TX;  // never float64
      hipLaunchKernelGGL(coded_product_kernel<TX>, dim3((unsigned)most_tiles(p, kCodedRows)), dim3(64 * kCodedWaves), 0, s, p,
                         elem_y, (const TX*)x, ldx, y, ldy);
    });
  }
  const int qs = quant(s, elem_x, 1, ntok, k, x, ldx, q, scale);
  if (qs != DPC_OK) return qs;
  return product(s, elem_y, p, y, ldy);
}
