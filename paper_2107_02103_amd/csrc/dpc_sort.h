// Stable counting sort of numbers below a limit, for jobs that say what is
// sorted and where it goes.
//
// With h[e][c] the count of key e in part c of the slots (parts in order), the
// row of a slot is
//   sum_{e' < e, c} h[e'][c] + sum_{c' < c} h[e][c'] + (slots of e before it in c).
// A part is what one wavefront walks, 64 slots at a time: lanes with the same
// key find each other by one ballot per bit of the key, and their rank is the
// number of such lanes below.  No atomics: the order is the same on every call.
// Bound by latency: 3 us for a few slots, 11 us for 331,776 of 2 keys in two
// launches, 15 us for 16,384 of 256 keys.
//
// A job has
//   kPart                            slots of a workgroup, at least (constexpr int)
//   int key(int64_t s)               key of slot s; none of [0, nkey): dropped
//   int64_t size(int64_t n)          slots that exist, at most n
//   void put(int64_t s, int e, int row)   slot s goes to row (-1: dropped)
//   void first(int e, int row)       first row of key e (once for each)
//   void total(int kept)             rows in all (once)
//   void empty(int64_t r)            row r < n stays empty
#ifndef DPC_SORT_H
#define DPC_SORT_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

// Up to here one workgroup sorts.  With 64 keys, us: 4,096 slots 9.4 so and
// 13.6 in three launches, 8,192 14.4 and 14.1, 16,384 24.3 and 14.1 (2 keys
// 6.9, 10.5; 9.5, 10.6; 14.8, 10.9).
constexpr int kOneBlockSlots = 8192;
constexpr int kMaxBlocks = 1024;
// Counts (one for each key and workgroup) up to which every workgroup of the last launch
// adds them up for itself, which saves a launch and costs reads by the square of the
// workgroups.  Plans, us, so and with the launch between:
//   262,144 slots of 32 keys 13.1 14.3, of 64 15.6 15.1;  524,288 of 16 13.1 14.8, of 32 15.3 15.7, of 64 20.8 16.9
//   1,048,576 of 2 12.0 15.8, of 8 15.1 17.8, of 16 18.1 18.4, of 32 24.5 19.8;  16,777,216 of 16 133 135
constexpr int kSelfCounts = 16384;
constexpr int kPlanWaves = 4;          // wavefronts of a workgroup of the three launches

// Beyond, a workgroup takes a job's kPart slots at least.
inline int plan_blocks(int64_t nslot, int part) {
  const int64_t b = (nslot + part - 1) / part;
  return (int)(b < kMaxBlocks ? b : kMaxBlocks);
}
// slots of a workgroup: every wavefront gets whole groups of 64
inline int64_t plan_part(int64_t nslot, int blocks) {
  const int64_t unit = 64 * kPlanWaves;
  return ((nslot + blocks - 1) / blocks + unit - 1) / unit * unit;
}

// Walks slots [lo, hi) of one wavefront, 64 at a time in order, calling
// f(slot, in range, key, kept, lanes of the same key).
template <typename Job, typename F>
__device__ __forceinline__ void walk(const Job& job, int64_t lo, int64_t hi, int nkey, F f) {
  const int lane = threadIdx.x & 63;
  const int bits = nkey > 1 ? 32 - __clz(nkey - 1) : 0;
  for (int64_t s0 = lo; s0 < hi; s0 += 64) {
    const int64_t s = s0 + lane;
    const int e = s < hi ? job.key(s) : -1;
    const bool kept = (unsigned)e < (unsigned)nkey;
    unsigned long long same = __ballot(kept);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((e >> b) & 1);
      same &= (e >> b) & 1 ? set : ~set;
    }
    f(s, s < hi, e, kept, same);
  }
}

// Counts of the keys among the slots [lo, hi) of one wavefront, in LDS.
template <typename Job>
__device__ __forceinline__ void count(const Job& job, int64_t lo, int64_t hi, int nkey, int* cnt) {
  const int lane = threadIdx.x & 63;
  walk(job, lo, hi, nkey, [&](int64_t, bool, int e, bool kept, unsigned long long same) {
    // the lowest lane of each key adds for all of them: one lane per address
    if (kept && (same & ((1ull << lane) - 1)) == 0) cnt[e] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  });
}

// Rows of the slots [lo, hi) of one wavefront; next[e]: its next row of key e.
template <typename Job>
__device__ __forceinline__ void place(const Job& job, int64_t lo, int64_t hi, int nkey, int* next) {
  const int lane = threadIdx.x & 63;
  walk(job, lo, hi, nkey, [&](int64_t s, bool in, int e, bool kept, unsigned long long same) {
    const int before = __popcll(same & ((1ull << lane) - 1));
    const int first = kept ? next[e] : 0;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (kept && before == 0) next[e] = first + __popcll(same);
    if (in) job.put(s, e, kept ? first + before : -1);
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

// Few slots: one workgroup.  LDS: counts [waves][nkey], totals [nkey], one int
// per wavefront.
template <typename Job>
__global__ __launch_bounds__(1024) void plan_one_kernel(int nslot, int nkey, Job job) {
  extern __shared__ int plan_lds[];
  const int waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int* cnt = plan_lds;
  int* tot = cnt + waves * nkey;
  int* tmp = tot + nkey;
  const int n = (int)job.size(nslot);
  const int part = ((nslot + waves - 1) / waves + 63) & ~63;
  const int lo = wave * part < n ? wave * part : n;
  const int hi = lo + part < n ? lo + part : n;
  for (int i = threadIdx.x; i < waves * nkey; i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  count(job, lo, hi, nkey, cnt + wave * nkey);
  __syncthreads();
  for (int e = threadIdx.x; e < nkey; e += blockDim.x) {
    int run = 0;
    for (int w = 0; w < waves; ++w) {
      const int c = cnt[w * nkey + e];
      cnt[w * nkey + e] = run;
      run += c;
    }
    tot[e] = run;
  }
  __syncthreads();
  const int kept = block_scan(tot, nkey, tmp);
  for (int e = threadIdx.x; e < nkey; e += blockDim.x) {
    const int first = tot[e];
    job.first(e, first);
    for (int w = 0; w < waves; ++w) cnt[w * nkey + e] += first;
  }
  if (threadIdx.x == 0) job.total(kept);
  for (int r = kept + threadIdx.x; r < nslot; r += blockDim.x) job.empty(r);
  __syncthreads();
  place(job, lo, hi, nkey, cnt + wave * nkey);
}

// Many slots, first launch: hist[e][block] = slots of key e in the block's part.
template <typename Job>
__global__ __launch_bounds__(64 * kPlanWaves) void plan_count_kernel(int64_t nslot, int64_t part, int nkey, Job job,
                                                                     int* __restrict__ hist) {
  extern __shared__ int plan_lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n = job.size(nslot);
  for (int i = threadIdx.x; i < kPlanWaves * nkey; i += blockDim.x) plan_lds[i] = 0;
  __syncthreads();
  const int64_t first = blockIdx.x * part + wave * (part / kPlanWaves);
  const int64_t lo = first < n ? first : n;
  const int64_t hi = lo + part / kPlanWaves < n ? lo + part / kPlanWaves : n;
  count(job, lo, hi, nkey, plan_lds + wave * nkey);
  __syncthreads();
  for (int e = threadIdx.x; e < nkey; e += blockDim.x) {
    int sum = 0;
    for (int w = 0; w < kPlanWaves; ++w) sum += plan_lds[w * nkey + e];
    hist[(int64_t)e * gridDim.x + blockIdx.x] = sum;
  }
}

// Second launch, one workgroup per key: hist[e] to its exclusive prefix sums
// over the blocks, total[e] to their sum.
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

// Third launch: rows of the block's part.  SELF: there was no second one, the
// counts are read as they are; each workgroup adds them up for itself.
template <typename Job, bool SELF>
__global__ __launch_bounds__(64 * kPlanWaves) void plan_place_kernel(int64_t nslot, int64_t part, int nkey, Job job,
                                                                     const int* __restrict__ hist,
                                                                     const int* __restrict__ total) {
  extern __shared__ int plan_lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int* cnt = plan_lds;
  int* off = cnt + kPlanWaves * nkey;
  int* tmp = off + nkey;
  int* prior = tmp + kPlanWaves;  // SELF: slots of each key in the blocks before
  const int64_t n = job.size(nslot);
  for (int i = threadIdx.x; i < kPlanWaves * nkey; i += blockDim.x) cnt[i] = 0;
  if (SELF) {
    int lanes = 1;  // of a key
    while (lanes < 64 && lanes * 2 * nkey <= 64 * kPlanWaves) lanes *= 2;
    const int lane = threadIdx.x & (lanes - 1), blocks = gridDim.x;
    for (int e0 = 0; e0 < nkey; e0 += 64 * kPlanWaves / lanes) {  // whole wavefronts stay: sums across lanes
      const int e = e0 + threadIdx.x / lanes;
      int all = 0, before = 0;
      if (e < nkey) {
        for (int b0 = lane; b0 < blocks; b0 += 8 * lanes) {
          int h[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) h[u] = hist[(int64_t)e * blocks + min(b0 + u * lanes, blocks - 1)];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int b = b0 + u * lanes;
            all += b < blocks ? h[u] : 0;
            before += b < (int)blockIdx.x ? h[u] : 0;  // one of the blocks
          }
        }
      }
      for (int m = lanes >> 1; m; m >>= 1) {
        all += __shfl_xor(all, m);
        before += __shfl_xor(before, m);
      }
      if (e < nkey && lane == 0) {
        off[e] = all;
        prior[e] = before;
      }
    }
  } else {
    for (int e = threadIdx.x; e < nkey; e += blockDim.x) off[e] = total[e];
  }
  __syncthreads();
  const int kept = block_scan(off, nkey, tmp);
  const int64_t first = blockIdx.x * part + wave * (part / kPlanWaves);
  const int64_t lo = first < n ? first : n;
  const int64_t hi = lo + part / kPlanWaves < n ? lo + part / kPlanWaves : n;
  count(job, lo, hi, nkey, cnt + wave * nkey);
  __syncthreads();
  for (int e = threadIdx.x; e < nkey; e += blockDim.x) {
    int run = off[e] + (SELF ? prior[e] : hist[(int64_t)e * gridDim.x + blockIdx.x]);
    for (int w = 0; w < kPlanWaves; ++w) {
      const int c = cnt[w * nkey + e];
      cnt[w * nkey + e] = run;
      run += c;
    }
    if (blockIdx.x == 0) job.first(e, off[e]);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) job.total(kept);
  for (int64_t r = kept + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; r < nslot; r += (int64_t)gridDim.x * blockDim.x)
    job.empty(r);
  __syncthreads();
  place(job, lo, hi, nkey, cnt + wave * nkey);
}

// Bytes of workspace that a sort of nslot slots needs.
template <typename Job>
size_t sort_workspace_bytes(int64_t nslot, int nkey) {
  const size_t blocks = nslot <= kOneBlockSlots ? 0 : plan_blocks(nslot, Job::kPart);
  return ((blocks + 1) * nkey * sizeof(int) + 255) / 256 * 256;
}

// Enqueues the sort of nslot slots with keys below nkey <= 1024.
template <typename Job>
void launch_sort(hipStream_t s, int64_t nslot, int nkey, const Job& job, void* workspace) {
  if (nslot <= kOneBlockSlots) {
    const int waves = nslot <= 256 ? 4 : 16;
    const size_t lds = ((size_t)(waves + 1) * nkey + waves) * sizeof(int);
    hipLaunchKernelGGL(plan_one_kernel<Job>, dim3(1), dim3(64 * waves), lds, s, (int)nslot, nkey, job);
    return;
  }
  const int blocks = plan_blocks(nslot, Job::kPart);
  const int64_t part = plan_part(nslot, blocks);
  int* hist = static_cast<int*>(workspace);
  int* total = hist + (size_t)blocks * nkey;
  const dim3 block(64 * kPlanWaves);
  hipLaunchKernelGGL(plan_count_kernel<Job>, dim3(blocks), block, (size_t)kPlanWaves * nkey * sizeof(int), s, nslot, part,
                     nkey, job, hist);
  const size_t lds = ((size_t)(kPlanWaves + 1) * nkey + kPlanWaves) * sizeof(int);
  // Few counts: every workgroup adds them up, which takes less than a launch.
  if ((int64_t)blocks * nkey <= kSelfCounts) {
    hipLaunchKernelGGL((plan_place_kernel<Job, true>), dim3(blocks), block, lds + nkey * sizeof(int), s, nslot, part, nkey,
                       job, hist, total);
    return;
  }
  hipLaunchKernelGGL(plan_scan_kernel, dim3(nkey), dim3(256), 0, s, blocks, hist, total);
  hipLaunchKernelGGL((plan_place_kernel<Job, false>), dim3(blocks), block, lds, s, nslot, part, nkey, job, hist, total);
}

}  // namespace

#endif  // DPC_SORT_H
