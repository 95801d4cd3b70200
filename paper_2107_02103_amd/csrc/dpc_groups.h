// Rows in groups (one for each expert) and the tiles of a product over them, for
// the products of codes.
//
// A product P has m rows of results, topk of them for each token; rows[r], if
// given, is the slot of row r (its token times topk and more), offsets[g], if
// given, the first row of group g < ngroup.
#ifndef DPC_GROUPS_H
#define DPC_GROUPS_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// Rows [row0, end) of one tile of a group, or of the empty rows (group < 0);
// end = row0 if the tile does not exist.
struct Tile {
  int group, row0, end;
};

// The tile-th tile of `size` rows: the tiles of group 0, of group 1, ... and of
// the rows past the last group.  Whole wavefronts call this.
template <typename P>
__device__ __forceinline__ Tile find_tile(const P& p, int size, int tile) {
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
template <typename P>
__device__ __forceinline__ int count_tiles(const P& p, int size) {
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

// token of row r, or -1
template <typename P>
__device__ __forceinline__ int token_of(const P& p, int r) {
  if (!p.rows) return r;
  const int s = p.rows[r];
  return (unsigned)s < (unsigned)p.m ? (int)((unsigned)s / (unsigned)p.topk) : -1;
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

typedef const __attribute__((address_space(1))) void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;

}  // namespace

#endif  // DPC_GROUPS_H
