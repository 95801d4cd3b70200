// Layers in 8-bit integers (dpc_quant_rows, dpc_matmul_i8, dpc_linear_i8).
//
// Codes: one read of a row into registers, the largest magnitude across its
// lanes, then the codes.  Bound by HBM bandwidth (16,384 bfloat16 rows of 4,096:
// 201 MB read and written in 47 us), or by the latency of one load and two
// reductions for a few rows (16 rows of 8,192: 5.2 us).
//
// Product: y[r][c] = (sum_i qx[t][i] qw[g][c][i]) sx[t] sw[g][c] + bias[g][c].
// The sum over i is exact in 32-bit integers, so its order is free.  On the
// matrix cores W's rows are the rows and x's rows the columns of a tile: a
// lane of a result holds four channels of one row of y.  Which rows of W make
// a tile is free, so larger tiles are dealt rows that end as runs of 16 bytes
// of y in a lane (channel_of).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "dpc.h"
#include "dpc_elem.h"
#include "dpc_i8_tiles.h"
#include "dpc_internal.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30;      // rows of codes
constexpr int64_t kMaxProduct = (int64_t)1 << 27;   // rows of a product (a launch has under 2^32 threads)
constexpr int kMaxChannels = 1 << 24;

// ---------------------------------------------------------------------------
// codes
// ---------------------------------------------------------------------------
constexpr int kHeld = 8;  // chunks of a row that a lane holds

// Codes of one chunk: the product is rounded on its own, and adding 1.5 * 2^23
// rounds it to the nearest integer (ties to even), whose low byte is the code.
template <int VE>
__device__ __forceinline__ void codes_of(const float* v, float u, int8_t* q) {
#pragma clang fp contract(off)
  unsigned char b[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) {
    const float p = v[i] * u;
    b[i] = (unsigned char)__float_as_uint(p + 12582912.0f);
  }
  __builtin_memcpy(__builtin_assume_aligned(q, VE), b, VE);
}

// The largest magnitude of floats, as bits: as whole numbers magnitudes keep
// their order, with NaN the largest.  Of the bits with their signs, the largest
// signed number is the largest positive value, the largest unsigned one the
// largest negative value (or a positive one, if there is no negative).
struct Largest {
  int pos = 0;
  unsigned neg = 0;
  __device__ __forceinline__ void take(float v) {
    pos = max(pos, __float_as_int(v));
    neg = max(neg, __float_as_uint(v));
  }
  __device__ __forceinline__ unsigned bits() const { return max((unsigned)pos, neg & 0x7fffffffu); }
};

// The largest of a wavefront's values, for all of them.
__device__ __forceinline__ unsigned wave_max(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));  // row_shr:1
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));  // row_bcast:15
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));  // row_bcast:31
  return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}

// Scale and inverse of a row whose largest magnitude has the bits `top`.
__device__ __forceinline__ void scale_of(unsigned top, float* scale, float* inverse) {
  const float a = __uint_as_float(top);
  const bool finite = top < 0x7f800000u, live = finite && a >= 0x1p-100f;
  *inverse = live ? 127.0f / a : 0.0f;
  *scale = live ? a / 127.0f : finite ? 0.0f : __builtin_nanf("");
}

// LANES lanes of a row (up to 64: several rows in a wavefront; 256: a whole
// workgroup).  HELD: the row has a chunk and fits the lanes' registers, and is
// read once.  Up to 64 lanes, chunks that reach past its end take its last
// elements instead (no branch: one around each load would make it wait for the
// load before), which changes no maximum, and get the code 0 or are read again.
// A workgroup has few loads a lane and would make up to a lane's worth of them for
// nothing, so there a branch skips them.  Both, us, with and without branches:
// 131,072 bfloat16 rows of 512 (64 lanes) 73 and 49, 262,144 of 1,600 321 and 296,
// 262,144 float32 rows of 240 118 and 102; a workgroup: 262,144 float64 rows of
// 1,600 708 and 926, 32,768 float32 rows of 4,096 124 and 135, 32,768 bfloat16
// rows of 8,192 154 and 161.
// Rows longer than a workgroup holds (8,192 of float32) are read element by
// element, twice: 16,384 float32 rows of 16,384 467 us (2.9 TB/s), 16,384 float64
// rows of 8,192 361 (3.4), 16,384 bfloat16 rows of 32,768 1,007 (1.6).
template <typename T, int LANES, bool HELD>
__global__ __launch_bounds__(256) void quant_kernel(int nrows, int ncols, const T* __restrict__ x, int64_t ldx,
                                                    int8_t* __restrict__ q, float* __restrict__ scale) {
  constexpr int VE = Chunk<T>::kElems;
  constexpr bool kSkip = LANES > 64;  // chunks past the row's end are not loaded
  const int lane = threadIdx.x & (LANES - 1);
  const int ld = DPC_I8_LD(ncols), nch = ld / VE;
  const int64_t groups = (int64_t)gridDim.x * (256 / LANES);
  const int64_t rounds = (nrows + groups - 1) / groups;
  int64_t r = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  for (int64_t i = 0; i < rounds; ++i, r += groups) {
    const bool in = r < nrows;
    int row = in ? (int)r : 0;
    if (LANES >= 64) row = __builtin_amdgcn_readfirstlane(row);
    const T* px = x + (int64_t)row * ldx;
    auto single = [&](int c, float* v) __attribute__((always_inline)) {  // an element at a time
#pragma unroll
      for (int k = 0; k < VE; ++k) v[k] = c * VE + k < ncols ? (float)px[c * VE + k] : 0.0f;
    };
    Chunk<T> held[HELD ? kHeld : 1];
    Largest most;
    if (HELD) {
#pragma unroll
      for (int h = 0; h < kHeld; ++h) {
        const int c = lane + h * LANES;
        if (!kSkip) {
          if (h * LANES < nch) held[h].load(px + (unsigned)min(c * VE, ncols - VE));
        } else if (c * VE + VE <= ncols) {
          held[h].load(px + c * VE);
        } else if (c < nch) {
#pragma unroll
          for (int k = 0; k < VE; ++k) held[h].v[k] = c * VE + k < ncols ? px[c * VE + k] : (T)0;
        }
      }
#pragma unroll
      for (int h = 0; h < kHeld; ++h)
        if ((kSkip ? lane : 0) + h * LANES < nch)
#pragma unroll
          for (int k = 0; k < VE; ++k) most.take((float)held[h].v[k]);
    } else {
      for (int c = lane; c < nch; c += LANES) {
        float v[VE];
        single(c, v);
#pragma unroll
        for (int k = 0; k < VE; ++k) most.take(v[k]);
      }
    }
    unsigned top = most.bits();
    if (LANES < 64) {
#pragma unroll
      for (int m = LANES >> 1; m; m >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, m));
    } else {
      top = wave_max(top);
    }
    if (LANES > 64) {
      __shared__ unsigned tops[4];
      __syncthreads();  // the row before has been read
      if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
      __syncthreads();
      top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    if (!in) continue;
    const bool finite = top < 0x7f800000u;
    float row_scale, u;
    scale_of(top, &row_scale, &u);
    if (lane == 0) scale[r] = row_scale;
    int8_t* pq = q + r * ld;
    auto put = [&](int c, const float* v, float u) __attribute__((always_inline)) {
      float w[VE];
#pragma unroll
      for (int k = 0; k < VE; ++k) w[k] = finite ? v[k] : 0.0f;
      codes_of<VE>(w, u, pq + c * VE);
    };
    if (HELD) {
#pragma unroll
      for (int h = 0; h < kHeld; ++h) {
        const int c = lane + h * LANES;
        if (c >= nch) continue;
        float v[VE];
#pragma unroll
        for (int k = 0; k < VE; ++k) v[k] = (float)held[h].v[k];
        put(c, v, kSkip || c * VE + VE <= ncols ? u : 0.0f);
      }
      if (!kSkip && ncols % VE && lane == ncols / VE % LANES) {  // the lane that wrote zeros there
        float v[VE];
        single(ncols / VE, v);
        put(ncols / VE, v, u);
      }
    } else {
      for (int c = lane; c < nch; c += LANES) {
        float v[VE];
        single(c, v);
        put(c, v, u);
      }
    }
  }
}

template <typename T>
void launch_quant(hipStream_t s, int nrows, int ncols, const T* x, int64_t ldx, int8_t* q, float* scale) {
  const int nch = DPC_I8_LD(ncols) / Chunk<T>::kElems;
  auto go = [&](auto kernel, int lanes) {
    const int64_t per = 256 / lanes, blocks = (nrows + per - 1) / per, most = 1 << 20;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s, nrows, ncols, x, ldx, q,
                       scale);
  };
  // the fewest lanes that hold a row, at most two chunks each in short rows
  if (ncols < Chunk<T>::kElems) go(quant_kernel<T, 16, false>, 16);
  else if (nch <= 16 * 2) go(quant_kernel<T, 16, true>, 16);
  else if (nch <= 64 * kHeld) go(quant_kernel<T, 64, true>, 64);
  else if (nch <= 256 * kHeld) go(quant_kernel<T, 256, true>, 256);
  else go(quant_kernel<T, 256, false>, 256);
}

int quant(hipStream_t s, dpc_elem elem, int nrows, int ncols, const void* x, int64_t ldx, int8_t* q, float* scale) {
  (void)hipGetLastError();  // report only what this launch raises
  switch (elem) {
    case DPC_ELEM_F64: launch_quant(s, nrows, ncols, (const double*)x, ldx, q, scale); break;
    case DPC_ELEM_F32: launch_quant(s, nrows, ncols, (const float*)x, ldx, q, scale); break;
    case DPC_ELEM_F16: launch_quant(s, nrows, ncols, (const _Float16*)x, ldx, q, scale); break;
    default: launch_quant(s, nrows, ncols, (const __bf16*)x, ldx, q, scale); break;
  }
  return dpc_internal_launch_status();
}

// ---------------------------------------------------------------------------
// product
// ---------------------------------------------------------------------------
typedef int v4i __attribute__((ext_vector_type(4)));

struct Product {
  int ntok, topk, m, n, k, ld, ngroup;
  const int8_t* qx;
  const float* sx;
  const int* rows;
  const int* offsets;
  const int8_t* qw;
  const float* sw;
  const float* bias;
};

// Rows [row0, end) of one tile of a group, or of the empty rows (group < 0);
// end = row0 if the tile does not exist.
struct Tile {
  int group, row0, end;
};

// The tile-th tile of `size` rows: the tiles of group 0, of group 1, ... and of
// the rows past the last group.  Whole wavefronts call this.
__device__ __forceinline__ Tile find_tile(const Product& p, int size, int tile) {
  if (!p.offsets) {
    const int row0 = tile * size;
    return Tile{0, row0 < p.m ? row0 : p.m, row0 + size < p.m ? row0 + size : p.m};
  }
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int g0 = 0; g0 <= p.ngroup; g0 += 64) {
    const int g = g0 + lane;
    int first = p.m, last = p.m;
    if (g <= p.ngroup) first = min(max(p.offsets[g], 0), p.m);
    if (g < p.ngroup) last = max(min(max(p.offsets[g + 1], 0), p.m), first);
    const int tiles = (last - first + size - 1) / size;
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    const unsigned long long past = __ballot(before + sum > tile);
    if (past) {
      const int at = __ffsll(past) - 1;
      const int lo = __shfl(first, at), hi = __shfl(last, at);
      const int row0 = lo + (tile - before - __shfl(sum - tiles, at)) * size;
      return Tile{g0 + at < p.ngroup ? g0 + at : -1, row0, min(row0 + size, hi)};
    }
    before += __shfl(sum, 63);
  }
  return Tile{-1, p.m, p.m};
}

// Tiles of `size` rows that exist, on the device.
__device__ __forceinline__ int count_tiles(const Product& p, int size) {
  if (!p.offsets) return (p.m + size - 1) / size;
  const int lane = threadIdx.x & 63;
  int sum = 0;
  for (int g = lane; g <= p.ngroup; g += 64) {
    const int first = min(max(p.offsets[g], 0), p.m);
    const int last = g < p.ngroup ? max(min(max(p.offsets[g + 1], 0), p.m), first) : p.m;
    sum += (last - first + size - 1) / size;
  }
#pragma unroll
  for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
  return __builtin_amdgcn_readfirstlane(sum);
}

// Tiles of `size` rows that find_tile can be asked for.
inline int64_t most_tiles(const Product& p, int size) {
  return i8_most_tiles(p.m, p.ngroup, p.offsets != nullptr, size);
}

inline bool few_rows(const Product& p) { return i8_few_rows(p.m, p.n, p.ngroup, p.offsets != nullptr); }

// token of row r, or -1
__device__ __forceinline__ int token_of(const Product& p, int r) {
  if (!p.rows) return r;
  const int s = p.rows[r];
  return (unsigned)s < (unsigned)p.m ? (int)((unsigned)s / (unsigned)p.topk) : -1;
}

// One result from its sum: in float64, where neither scale nor their product
// leaves the range, rounded to float32 and from there to 16 bits.
template <typename TY>
__device__ __forceinline__ TY scaled(int acc, double sx, float sw, float bias) {
  const double v = fma((double)acc, sx * (double)sw, (double)bias);
  if constexpr (sizeof(TY) == 8) return v;
  float f = (float)v;
  if constexpr (sizeof(TY) == 2) asm("" : "+v"(f));  // two roundings: one from float64 takes eight instructions
  return (TY)f;
}

// 16 rows of 64 bytes, loaded with the 4 chunks of a row in neighbouring lanes,
// to the lanes of a product's operand: row l % 16, chunk l / 16.  (Loaded in
// those lanes at once, every lane of a load meets another cache line than its
// neighbours, and the cache's tags take four times as long.)
__device__ __forceinline__ v4i to_rows(v4i w) {
  const int lane = threadIdx.x & 63, from = ((lane & 15) * 4 + (lane >> 4)) * 4;
  v4i r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_ds_bpermute(from, w[i]);
  return r;
}

// Few rows: 16 rows times 16 channels of y for each `share` wavefronts of a
// workgroup of 8, which take the steps of K in turn and whose sums are added in
// LDS.  W is read once for each 16 rows of an expert, 8 KiB of it under way in
// every wavefront: bound by that read, or for short rows by latency.  TX is the type of rows that the workgroup
// codes itself (into LDS), or int8_t for rows that are codes already.
constexpr int kFewWaves = 8, kFewAhead = 4;

template <typename TX, typename TY>
__global__ __launch_bounds__(64 * kFewWaves) void few_product_kernel(Product p, int share, const TX* __restrict__ x,
                                                                     int64_t ldx, TY* __restrict__ y, int64_t ldy) {
  constexpr bool kCoded = sizeof(TX) == 1;
  extern __shared__ __attribute__((aligned(16))) int8_t codes[];  // 16 rows of codes, if they are made here
  __shared__ int sums[kFewWaves][256];
  __shared__ float scales[16];
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile t = find_tile(p, 16, blockIdx.y + gridDim.y * blockIdx.z);
  if (t.row0 >= t.end) return;
  const int tiles = kFewWaves / share;  // channel tiles of the workgroup
  const int c0 = (blockIdx.x * tiles + wave / share) * 16, part = wave % share;
  const int steps = p.ld / 128, group = max(t.group, 0);
  const int8_t* pw = p.qw + ((int64_t)group * p.n + min(c0 + (lane >> 2), p.n - 1)) * p.ld + (lane & 3) * 16;
  const int mine = t.group < 0 ? -1 : token_of(p, min(t.row0 + (lane >> 2), t.end - 1));
  const int8_t* pq = kCoded ? (const int8_t*)x + (int64_t)max(mine, 0) * p.ld + (lane & 3) * 16 : nullptr;
  v4i w[kFewAhead][2], q[kFewAhead][2];
  auto fetch = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int s = min(s0 + u * share, steps - 1);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        w[u][k] = *reinterpret_cast<const v4i*>(pw + s * 128 + k * 64);
        if (kCoded) q[u][k] = *reinterpret_cast<const v4i*>(pq + s * 128 + k * 64);
      }
    }
  };
  fetch(part);
  if constexpr (!kCoded) {
    constexpr int VE = Chunk<TX>::kElems;
    for (int row = wave; row < 16; row += kFewWaves) {
      if (t.row0 + row >= t.end) break;
      const int tok = __builtin_amdgcn_readfirstlane(t.group < 0 ? -1 : token_of(p, t.row0 + row));
      const TX* px = x + (int64_t)max(tok, 0) * ldx;
      auto element = [&](int i) { return i < p.k ? (float)px[i] : 0.0f; };
      Largest most;
      for (int c = lane * VE; c < p.k; c += 64 * VE) {
        if (c + VE <= p.k) {
          Chunk<TX> ch;
          ch.load(px + c);
#pragma unroll
          for (int e = 0; e < VE; ++e) most.take((float)ch.v[e]);
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) most.take(element(c + e));
        }
      }
      const unsigned top = wave_max(most.bits());
      const bool finite = top < 0x7f800000u;
      float scale, u;
      scale_of(top, &scale, &u);
      if (lane == 0) scales[row] = scale;
      for (int c = lane * VE; c < p.ld; c += 64 * VE) {
        float v[VE];
        if (c + VE <= p.k) {
          Chunk<TX> ch;
          ch.load(px + c);
#pragma unroll
          for (int e = 0; e < VE; ++e) v[e] = finite ? (float)ch.v[e] : 0.0f;
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) v[e] = finite ? element(c + e) : 0.0f;
        }
        codes_of<VE>(v, u, codes + row * p.ld + (c ^ ((row & 7) << 4)));
      }
    }
    __syncthreads();
  }
  const int high = min(t.end - t.row0, 16) - 1;  // rows of the tile past its end repeat its last one
  v4i acc = {0, 0, 0, 0};
  for (int s0 = part; s0 < steps; s0 += share * kFewAhead) {
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int s = s0 + u * share;
      if (s >= steps) break;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        v4i b;
        if constexpr (kCoded) {
          b = to_rows(q[u][k]);
        } else {
          const int row = min(l16, high);
          b = *reinterpret_cast<const v4i*>(codes + row * p.ld + s * 128 + (((k * 4 + quad) ^ (row & 7)) << 4));
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(to_rows(w[u][k]), b, acc, 0, 0, 0);
      }
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
    int sum = 0;
    for (int v = 0; v < share; ++v) sum += sums[tile * share + v][e & 255];
    const int tok = t.group < 0 ? -1 : token_of(p, r);
    TY out = (TY)0;
    if (tok >= 0) {
      const int64_t gc = (int64_t)group * p.n + c;
      out = scaled<TY>(sum, (double)(kCoded ? p.sx[tok] : scales[row]), p.sw[gc], p.bias ? p.bias[gc] : 0.0f);
    }
    y[(int64_t)r * ldy + c] = out;
  }
}

template <typename TX, typename TY>
void launch_few(hipStream_t s, const Product& p, const TX* x, int64_t ldx, TY* y, int64_t ldy) {
  const int64_t tiles = most_tiles(p, 16);
  const unsigned gy = (unsigned)(tiles < 32768 ? tiles : 32768);
  // wavefronts that share a tile: about 16 in all for each of 256 CUs (16 rows
  // of 2,048 for 16 of 64 experts with 2,048 channels: 15.8 us with 2, 24.7 with
  // 8; 16 rows through 8,192 x 8,192: 14.3 with 8, 19.2 with 2)
  const int64_t wide = (p.n + 15) / 16;
  int share = kFewWaves;
  while (share > 1 && wide * tiles * share > 4096) share /= 2;
  hipLaunchKernelGGL((few_product_kernel<TX, TY>),
                     dim3((unsigned)((wide * share + kFewWaves - 1) / kFewWaves), gy, (unsigned)((tiles + gy - 1) / gy)),
                     dim3(64 * kFewWaves), sizeof(TX) == 1 ? 0 : (size_t)(p.m < 16 ? p.m : 16) * p.ld, s, p, share, x,
                     ldx, y, ldy);
}

// Which channel stands in row r of channel tile j.  A lane of the products ends
// with rows 4 quad .. 4 quad + 3 of every tile; W's rows are dealt to the tiles so
// that these are runs of VE channels (16 bytes of results), and the four lanes
// that share a row of x store 64 bytes in a piece: result 4 j + q of a lane is
// channel (4 j + q) / VE * 4 VE + quad VE + (4 j + q) % VE.  (262,144 rows of 256
// to 1,024 channels, us, bf16, float32, float64: 211, 273, 461; with 4 channels
// a lane for each type and a branch around each store 237, 343, 571, and these
// past the caches 418, 305, 616.)
template <int VE>
__device__ __forceinline__ constexpr int channel_of(int j, int r) {
  const int at = 4 * j + r % 4;
  return at / VE * 4 * VE + r / 4 * VE + at % VE;
}

// r & 7 of the row r that a channel stands in: moves its chunks in LDS, so that
// 8 lanes that read one chunk of 8 rows meet all banks.
template <int VE>
__device__ __forceinline__ int turn_of(int channel) {
  return VE == 8   ? (channel & 3) | (channel >> 1 & 4)
         : VE == 4 ? channel & 7
                   : (channel & 1) | (channel >> 2 & 2) | (channel << 1 & 4);
}

// A run of results, of which `left` exist.
template <typename TY>
__device__ __forceinline__ void put_run(TY* p, const TY* v, int left) {
  constexpr int VE = 16 / sizeof(TY);
  typedef int Run __attribute__((ext_vector_type(4), aligned(2)));  // any address that an element may have
  if (left >= VE) {
    Run t;
    __builtin_memcpy(&t, v, 16);
    *reinterpret_cast<Run*>(p) = t;
    return;
  }
#pragma unroll
  for (int q = 0; q < VE; ++q)
    if (q < left) p[q] = v[q];
}

// Tiles of BM rows times BN channels, K in steps of 128 bytes: both operands
// go from memory to LDS without passing registers, the next step's while the
// matrix cores work on this one's.  A row of a step is 8 chunks of 16 bytes;
// chunk c of row r lies in slot c ^ (r & 7), so that the lanes of one LDS read
// (16 rows, the same chunk) meet all banks.  WM x WN wavefronts.
//
// 8192 x 8192 x 8192 in 440 to 510 us (2.2 to 2.5e15 operations a second, the
// more the cooler the card), 32,768 rows for 16 experts' 4096 x 4096 in 540 to
// 600.  In the largest tile a step's LDS reads and writes (1,536 + 512 clocks)
// take as long as its products (2,048): the matrix cores are 56% busy, at 1.8 to
// 2.1 GHz.  Tried without gain: 32 x 32 products (610 us), four wavefronts of
// 128 x 128 (600), wavefronts of 64 x 128 (466, with spills), priorities, halves
// of the wavefronts that take turns at LDS and the matrix cores (463 for 446).
typedef const __attribute__((address_space(1))) void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;

template <typename TY, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void product_tiled_kernel(Product p, int col_tiles,
                                                                     TY* __restrict__ y, int64_t ldy) {
  constexpr int VE = 16 / sizeof(TY);
  constexpr int kWaves = WM * WN, TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
  constexpr int kStep = 128, kRows = BM + BN;
  constexpr int kLoads = kRows / 8 / kWaves;  // 8 rows each
  static_assert(kLoads * kWaves * 8 == kRows, "every load takes 8 rows");
  __shared__ __attribute__((aligned(16))) int8_t lds[2][kRows * kStep];
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

  v4i acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = v4i{0, 0, 0, 0};

  // this lane's rows of the loads: x rows first, then rows of W
  const int8_t* src[kLoads];
  int dst[kLoads];
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int r8 = (wave * kLoads + l) * 8, r = r8 + (lane >> 3);
    const int chunk = (lane & 7) ^ (r < BM ? r & 7 : turn_of<VE>(r));
    const int8_t* row;
    if (r < BM) {
      const int tok = token_of(p, min(t.row0 + r, t.end - 1));
      row = p.qx + (int64_t)(tok < 0 ? 0 : tok) * p.ld;
    } else {
      row = p.qw + ((int64_t)t.group * p.n + min(c0 + r - BM, p.n - 1)) * p.ld;
    }
    src[l] = row + chunk * 16;
    dst[l] = r8 * kStep;
  }
  auto fetch = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      __builtin_amdgcn_global_load_lds((GlobalPtr)src[l], (LdsPtr)(&lds[buf][dst[l]]), 16, 0, 0);
      src[l] += kStep;
    }
  };
  const int steps = p.ld / kStep;
  fetch(0);
  for (int s = 0; s < steps; ++s) {
    // vmcnt(0), lgkmcnt(0): this step's rows are in LDS, the step before has
    // been read; the barrier says so for every wavefront
    __builtin_amdgcn_s_waitcnt(0x0070);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + 1 < steps) fetch((s + 1) & 1);
    const int8_t* xs = &lds[s & 1][wm * TM * kStep];
    const int8_t* ws = &lds[s & 1][(BM + wn * TN) * kStep];
    v4i a[2][NI], b[2][MI];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int slot = ((k * 4 + quad) ^ (l16 & 7)) * 16;
#pragma unroll
      for (int j = 0; j < NI; ++j) a[k][j] = *reinterpret_cast<const v4i*>(ws + (channel_of<VE>(j, 0) + channel_of<VE>(0, l16)) * kStep + slot);
#pragma unroll
      for (int i = 0; i < MI; ++i) b[k][i] = *reinterpret_cast<const v4i*>(xs + (i * 16 + l16) * kStep + slot);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[k][j], b[k][i], acc[i][j], 0, 0, 0);
    // LDS reads of the second half between the products of the first: one after
    // every other product (left alone, the reads come in clumps with a wait
    // behind each; 8192 x 8192 x 8192: 530 -> 513 us)
    constexpr int kReads = NI + MI, kSpaced = 2 * kReads <= MI * NI ? 2 : 1;
    __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
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
  float sw[kRuns][VE], bias[kRuns][VE];
  const float* psw = p.sw + (int64_t)t.group * p.n;
  const float* pbias = p.bias ? p.bias + (int64_t)t.group * p.n : psw;
  if (whole) {
#pragma unroll
    for (int g = 0; g < kRuns; ++g) {
      __builtin_memcpy(sw[g], psw + first + g * 4 * VE, 4 * VE);
      __builtin_memcpy(bias[g], pbias + first + g * 4 * VE, 4 * VE);
    }
  } else {
#pragma unroll
    for (int g = 0; g < kRuns; ++g)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int c = min(first + g * 4 * VE + e, p.n - 1);
        sw[g][e] = psw[c];
        bias[g][e] = pbias[c];
      }
  }
  if (!p.bias) {
#pragma unroll
    for (int g = 0; g < kRuns; ++g)
#pragma unroll
      for (int e = 0; e < VE; ++e) bias[g][e] = 0.0f;
  }
  int tok[MI];
  float sx[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) tok[i] = token_of(p, min(t.row0 + wm * TM + i * 16 + l16, t.end - 1));
#pragma unroll
  for (int i = 0; i < MI; ++i) sx[i] = p.sx[max(tok[i], 0)];
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = t.row0 + wm * TM + i * 16 + l16;
    TY* py = y + (int64_t)r * ldy + first;
#pragma unroll
    for (int g = 0; g < kRuns; ++g) {
      TY out[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        out[e] = scaled<TY>(acc[i][(g * VE + e) / 4][(g * VE + e) % 4], (double)sx[i], sw[g][e], bias[g][e]);
        if (tok[i] < 0) out[e] = (TY)0;  // a row of the group that no slot owns
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
  switch (i8_tile(p.m, p.n, p.ld, p.ngroup, p.offsets != nullptr)) {
    case 0: return launch_tiled<TY, 256, 256, 2, 4>(s, p, y, ldy);
    case 1: return launch_tiled<TY, 128, 128, 2, 2>(s, p, y, ldy);
    case 2: return launch_tiled<TY, 128, 64, 2, 2>(s, p, y, ldy);
    default: return launch_tiled<TY, 64, 64, 2, 2>(s, p, y, ldy);
  }
}

int product(hipStream_t s, dpc_elem elem_y, const Product& p, void* y, int64_t ldy) {
  (void)hipGetLastError();  // report only what this launch raises
  switch (elem_y) {
    case DPC_ELEM_F64: launch_product(s, p, (double*)y, ldy); break;
    case DPC_ELEM_F32: launch_product(s, p, (float*)y, ldy); break;
    case DPC_ELEM_F16: launch_product(s, p, (_Float16*)y, ldy); break;
    default: launch_product(s, p, (__bf16*)y, ldy); break;
  }
  return dpc_internal_launch_status();
}

// A lane's 8 results of a row in the type of y, runs at c, c + 4 VE, ... of n.
template <typename TY>
__device__ __forceinline__ void put_row(TY* y, int c, int n, const v4i (&acc)[2], double sx, const float* sw,
                                        const float* bias, bool exists, bool owned) {
  constexpr int VE = 16 / sizeof(TY);
#pragma unroll
  for (int g = 0; g < 8 / VE; ++g) {
    TY out[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int at = g * VE + e;
      out[e] = owned ? scaled<TY>(acc[at / 4][at % 4], sx, sw[at], bias[at]) : (TY)0;
    }
    put_run(y + c + g * 4 * VE, out, exists ? n - c - g * 4 * VE : 0);
  }
}

// Codes and product in one, for layers of few channels: the codes of 32 rows
// stay in LDS and never see memory.  Each of 8 wavefronts codes 4 rows, the next
// one on its way while it codes one; a lane holds TURNS chunks of a row.  Then
// wavefront w makes channels 32 w .. 32 w + 31 of each 256, with W's rows
// straight from L2 (each of them meets all 32 rows of the workgroup at once).
// Chunks of codes lie as in the tiles above.
//
// Bound by the read of x: 1,048,576 float32 rows of 1,600 to 240 channels (7.7
// GB) in 1.83 to 1.87 ms, 1.67 without the products, which two workgroups of a
// CU do not hide entirely; 32,000 rows in 64 us.  float64 rows of 1,025 to 2,048
// take 16 turns, two rows of which do not fit (128 registers, 27 in scratch memory):
// 1,048,576 of 1,600 in 3.49 ms (15.4 GB: 4.4 TB/s).  Reading x past the caches
// leaves L2 to W (1.90 -> 1.87 ms).  Tried without gain: 16 wavefronts (2.7 ms,
// spills), three workgroups (3.2 ms, spills), W asked for before the codes are
// done, swizzled lanes for to_rows (its bank conflicts cost nothing).
constexpr int kCodedRows = 32, kCodedLd = kI8OneKernelLd;

template <typename TX, int TURNS>
__global__ __launch_bounds__(512, 4) void coded_product_kernel(Product p, dpc_elem elem_y, const TX* __restrict__ x,
                                                               int64_t ldx, void* __restrict__ y, int64_t ldy) {
  constexpr int VE = Chunk<TX>::kElems, kTurn = 64 * VE, kPitch = TURNS * kTurn;
  __shared__ __attribute__((aligned(16))) int8_t codes[kCodedRows * kPitch];
  __shared__ float scales[kCodedRows];
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile t = find_tile(p, kCodedRows, blockIdx.x);
  if (t.row0 >= t.end) return;

  // elements of this lane's chunks; those that reach past the end take the row's
  // last ones instead (no branch: one around each load would make it wait for
  // the load before), which changes no maximum and gets the code 0 below
  int at[TURNS];
#pragma unroll
  for (int h = 0; h < TURNS; ++h) at[h] = min(lane * VE + h * kTurn, p.k - VE);
  auto row_of = [&](int a) __attribute__((always_inline)) {
    const int tok = t.group < 0 ? -1 : token_of(p, min(t.row0 + wave * 4 + a, t.end - 1));
    return x + (int64_t)max(__builtin_amdgcn_readfirstlane(tok), 0) * ldx;
  };
  auto take = [&](const TX* px, Chunk<TX> (&held)[TURNS]) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < TURNS; ++h) held[h].load_once(px + (unsigned)at[h]);
  };
  auto code = [&](int a, const TX* px, const Chunk<TX> (&held)[TURNS]) __attribute__((always_inline)) {
    Largest most;
#pragma unroll
    for (int h = 0; h < TURNS; ++h)
#pragma unroll
      for (int e = 0; e < VE; ++e) most.take((float)held[h].v[e]);
    const unsigned top = wave_max(most.bits());
    const int row = wave * 4 + a, turn = (row & 7) << 4;
    float scale, u;
    scale_of(top, &scale, &u);
    if (lane == 0) scales[row] = scale;
    // byte b of the row, its 16-byte chunk moved among the 8 of its step
    int8_t* to = codes + row * kPitch;
    const bool finite = top < 0x7f800000u;
#pragma unroll
    for (int h = 0; h < TURNS; ++h) {
      const float uc = lane * VE + h * kTurn + VE <= p.k ? u : 0.0f;  // whole chunks
      float v[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = finite ? (float)held[h].v[e] : 0.0f;
      codes_of<VE>(v, uc, to + ((lane * VE) ^ turn) + h * kTurn);
    }
    const int rest = p.k % VE;  // elements behind the last whole chunk: over the zeros written there
    if (rest && lane < rest) {
      const int last = p.k - rest + lane;
      const float v = finite ? (float)px[last] : 0.0f;
      codes_of<1>(&v, u, to + (last ^ turn));
    }
  };
  {
    Chunk<TX> held[2][TURNS];
    const TX *px0 = row_of(0), *px1;
    take(px0, held[0]);
    px1 = row_of(1);
    take(px1, held[1]);
    code(0, px0, held[0]);
    px0 = row_of(2);
    take(px0, held[0]);
    code(1, px1, held[1]);
    px1 = row_of(3);
    take(px1, held[1]);
    code(2, px0, held[0]);
    code(3, px1, held[1]);
  }
  __syncthreads();

  const int group = max(t.group, 0), steps = p.ld / 128;
  const int ve = elem_y == DPC_ELEM_F64 ? 2 : elem_y == DPC_ELEM_F32 ? 4 : 8;
  auto channel = [&](int j, int r) __attribute__((always_inline)) {
    return ve == 2 ? channel_of<2>(j, r) : ve == 4 ? channel_of<4>(j, r) : channel_of<8>(j, r);
  };
  for (int c0 = wave * 32; c0 < p.n; c0 += 256) {
    const int8_t* pw[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      pw[j] = p.qw + ((int64_t)group * p.n + min(c0 + channel(j, lane >> 2), p.n - 1)) * p.ld + (lane & 3) * 16;
    v4i acc[2][2], a0[2][2], a1[2][2];  // a0, a1: W of two steps, on their way
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = v4i{0, 0, 0, 0};
    auto fetch = [&](int s, v4i (&w)[2][2]) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) w[k][j] = *reinterpret_cast<const v4i*>(pw[j] + min(s, steps - 1) * 128 + k * 64);
    };
    // step s with w, which then takes step s + 2
    auto step = [&](int s, v4i (&w)[2][2]) __attribute__((always_inline)) {
      v4i a[2][2], b[2][2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          a[k][i] = to_rows(w[k][i]);
          b[k][i] = *reinterpret_cast<const v4i*>(codes + (i * 16 + l16) * kPitch + s * 128 + (((k * 4 + quad) ^ (l16 & 7)) << 4));
        }
      fetch(s + 2, w);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[k][j], b[k][i], acc[i][j], 0, 0, 0);
    };
    fetch(0, a0);
    fetch(1, a1);
    int s = 0;
    for (; s + 1 < steps; s += 2) {
      step(s, a0);
      step(s + 1, a1);
    }
    if (s < steps) step(s, a0);
    const float* psw = p.sw + (int64_t)group * p.n;
    const float* pbias = p.bias ? p.bias + (int64_t)group * p.n : psw;
    float sw[8], bias[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int c = min(c0 + channel(q / 4, quad * 4 + q % 4), p.n - 1);
      sw[q] = psw[c];
      bias[q] = pbias[c];
      if (!p.bias) bias[q] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = t.row0 + i * 16 + l16, c = c0 + quad * ve;
      const bool exists = r < t.end, owned = exists && t.group >= 0 && token_of(p, r) >= 0;
      const double sx = (double)scales[i * 16 + l16];
      auto put = [&](auto* py) __attribute__((always_inline)) {
        put_row(py + (int64_t)r * ldy, c, p.n, acc[i], sx, sw, bias, exists, owned);
      };
      switch (elem_y) {
        case DPC_ELEM_F64: put((double*)y); break;
        case DPC_ELEM_F32: put((float*)y); break;
        case DPC_ELEM_F16: put((_Float16*)y); break;
        default: put((__bf16*)y); break;
      }
    }
  }
}

template <typename TX, int TURNS = 1>
void launch_coded(hipStream_t s, const Product& p, dpc_elem elem_y, const TX* x, int64_t ldx, void* y, int64_t ldy) {
  constexpr int kTurn = 64 * Chunk<TX>::kElems;
  if constexpr (TURNS * kTurn < kCodedLd) {
    // float64: 1, 2, 4, 8, 16 turns; others every number
    if (p.ld > TURNS * kTurn)
      return launch_coded<TX, sizeof(TX) == 8 ? 2 * TURNS : TURNS + 1>(s, p, elem_y, x, ldx, y, ldy);
  }
  hipLaunchKernelGGL((coded_product_kernel<TX, TURNS>), dim3((unsigned)most_tiles(p, kCodedRows)), dim3(512), 0, s, p,
                     elem_y, x, ldx, y, ldy);
}

template <typename TX>
void few_by_type(hipStream_t s, const Product& p, dpc_elem elem_y, const TX* x, int64_t ldx, void* y, int64_t ldy) {
  switch (elem_y) {
    case DPC_ELEM_F64: launch_few(s, p, x, ldx, (double*)y, ldy); break;
    case DPC_ELEM_F32: launch_few(s, p, x, ldx, (float*)y, ldy); break;
    case DPC_ELEM_F16: launch_few(s, p, x, ldx, (_Float16*)y, ldy); break;
    default: launch_few(s, p, x, ldx, (__bf16*)y, ldy); break;
  }
}

// The layer in one kernel, if it is one for that: true and its status.
bool coded_product(hipStream_t s, dpc_elem elem_x, dpc_elem elem_y, const Product& p, const void* x, int64_t ldx, void* y,
                   int64_t ldy, int* status) {
  // Up to 256 channels, which a workgroup makes in one turn (i8_one_kernel has both
  // sides' times).  With 320 and 512 channels of float32 rows of 1,600 this kernel
  // takes 16.6 and 20.8 us where two take 15.5 and 16.0 at 2,048 rows, 73 and 91
  // where they take 90 and 97 at 32,000; with 320 of bfloat16 rows of 240 161 where
  // they take 129 at 262,144.  Rows that go to several experts would be
  // coded once for each.
  // Few rows in all, short ones: every workgroup codes them again, one row in
  // each wavefront, which costs less than a launch (device times: one float32 row
  // of 1,600 to 240 channels 5.6 us and 6.9 in two kernels, 8 rows 6.6 and 7.5; but
  // 16 rows 9.8 and 7.7, one bfloat16 row of 4,096 to 4,096 channels 9.2 and 9.0, 8
  // rows 12.9 and 11.0).  Coding float64 rows takes longer than a launch of its own
  // on the device (one row 7.7 and 6.5, 8 rows 9.2 and 6.8) but not with the
  // host's part of it (9.6 and 12.3).
  const bool few = p.m <= kFewWaves && p.ld <= 2048;
  if (!few && (p.topk != 1 || p.n > 256 || few_rows(p))) return false;
  (void)hipGetLastError();  // report only what this launch raises
  const auto go = [&](auto* px) {
    if (few) {
      few_by_type(s, p, elem_y, px, ldx, y, ldy);
    } else {
      if (!i8_one_kernel(p.m, p.k, p.ld, Chunk<std::remove_const_t<std::remove_pointer_t<decltype(px)>>>::kElems))
        return false;
      launch_coded(s, p, elem_y, px, ldx, y, ldy);
    }
    *status = dpc_internal_launch_status();
    return true;
  };
  switch (elem_x) {
    case DPC_ELEM_F64: return go((const double*)x);
    case DPC_ELEM_F32: return go((const float*)x);
    case DPC_ELEM_F16: return go((const _Float16*)x);
    default: return go((const __bf16*)x);
  }
}

int product_args(dpc_elem elem_y, int ntok, int topk, int n, int k, int ngroup) {
  if (!elem_ok(elem_y) || ntok < 0 || topk < 1 || n < 1 || k < 1 || ngroup < 1) return DPC_EINVAL;
  if (topk > DPC_MAX_TOPK || k > DPC_MAX_I8_COLS || ngroup > DPC_MAX_EXPERTS || n > kMaxChannels ||
      (int64_t)ntok * topk > kMaxProduct)
    return DPC_ENOTSUP;
  return DPC_OK;
}

bool product_ptrs(dpc_elem elem_y, int topk, int n, int ngroup, const int* rows, const int* offsets, const int8_t* qw,
                  const float* sw, const float* bias, const void* y, int64_t ldy) {
  if ((!rows && topk != 1) || (!offsets && ngroup != 1)) return false;
  return qw && sw && y && ldy >= n && elem_aligned(qw, 16) && elem_aligned(sw, 4) && elem_aligned(bias, 4) &&
         elem_aligned(rows, 4) && elem_aligned(offsets, 4) && elem_aligned(y, elem_size(elem_y));
}

}  // namespace

extern "C" int dpc_quant_rows(void* stream, dpc_elem elem, int nrows, int ncols, const void* x, int64_t ldx, int8_t* q,
                              float* scale) {
  if (!elem_ok(elem) || nrows < 0 || ncols < 1) return DPC_EINVAL;
  if (ncols > DPC_MAX_I8_COLS || nrows > kMaxRows) return DPC_ENOTSUP;
  if (nrows == 0) return DPC_OK;
  if (!x || !q || !scale || ldx < ncols || !elem_aligned(x, elem_size(elem)) || !elem_aligned(q, 16) ||
      !elem_aligned(scale, 4))
    return DPC_EINVAL;
  return quant(static_cast<hipStream_t>(stream), elem, nrows, ncols, x, ldx, q, scale);
}

extern "C" int dpc_matmul_i8(void* stream, dpc_elem elem_y, int ntok, int topk, int n, int k, int ngroup,
                             const int8_t* qx, const float* sx, const int* rows, const int* offsets, const int8_t* qw,
                             const float* sw, const float* bias, void* y, int64_t ldy) {
  const int st = product_args(elem_y, ntok, topk, n, k, ngroup);
  if (st != DPC_OK) return st;
  if (ntok == 0) return DPC_OK;
  if (!qx || !sx || !elem_aligned(qx, 16) || !elem_aligned(sx, 4) ||
      !product_ptrs(elem_y, topk, n, ngroup, rows, offsets, qw, sw, bias, y, ldy))
    return DPC_EINVAL;
  const Product p{ntok, topk, ntok * topk, n, k, DPC_I8_LD(k), ngroup, qx, sx, rows, offsets, qw, sw, bias};
  return product(static_cast<hipStream_t>(stream), elem_y, p, y, ldy);
}

extern "C" size_t dpc_linear_i8_workspace_bytes(int ntok, int k) {
  if (ntok < 0 || ntok > kMaxRows || k < 1 || k > DPC_MAX_I8_COLS) return 0;
  return ((size_t)ntok * DPC_I8_LD(k) + (size_t)ntok * sizeof(float) + 255) / 256 * 256 + 256;
}

extern "C" int dpc_linear_i8(void* stream, dpc_elem elem_x, dpc_elem elem_y, int ntok, int topk, int n, int k,
                             int ngroup, const void* x, int64_t ldx, const int* rows, const int* offsets,
                             const int8_t* qw, const float* sw, const float* bias, void* workspace,
                             size_t workspace_bytes, void* y, int64_t ldy) {
  const int st = product_args(elem_y, ntok, topk, n, k, ngroup);
  if (st != DPC_OK) return st;
  if (!elem_ok(elem_x)) return DPC_EINVAL;
  if (ntok == 0) return DPC_OK;
  if (!x || ldx < k || !elem_aligned(x, elem_size(elem_x)) || !workspace || !elem_aligned(workspace, 16) ||
      workspace_bytes < dpc_linear_i8_workspace_bytes(ntok, k) ||
      !product_ptrs(elem_y, topk, n, ngroup, rows, offsets, qw, sw, bias, y, ldy))
    return DPC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  int8_t* q = static_cast<int8_t*>(workspace);
  float* scale = reinterpret_cast<float*>(q + (size_t)ntok * DPC_I8_LD(k));
  Product p{ntok, topk, ntok * topk, n, k, DPC_I8_LD(k), ngroup, q, scale, rows, offsets, qw, sw, bias};
  int coded;
  if (coded_product(s, elem_x, elem_y, p, x, ldx, y, ldy, &coded)) return coded;
  const int qs = quant(s, elem_x, ntok, k, x, ldx, q, scale);
  if (qs != DPC_OK) return qs;
  return product(s, elem_y, p, y, ldy);
}
