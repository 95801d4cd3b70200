// Element types of rows: storage type, type of sums, 16-byte chunks.
#ifndef DPC_ELEM_H
#define DPC_ELEM_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dpc.h"

template <typename T>
struct ElemAcc {
  typedef float type;
};
template <>
struct ElemAcc<double> {
  typedef double type;
};

// A 16-byte chunk of a row.  Rows are aligned to their elements alone, so the
// chunk is too: the hardware takes 16-byte loads and stores at any address.
template <typename T>
struct Chunk {
  static constexpr int kElems = 16 / sizeof(T);
  T v[kElems];
  __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(v, p, 16); }
  __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, v, 16); }
  // past the caches, for what is not used again before they would have lost it
  __device__ __forceinline__ void load_once(const T* p) {
    const u4 w = __builtin_nontemporal_load(reinterpret_cast<const u4*>(p));
    __builtin_memcpy(v, &w, 16);
  }
  __device__ __forceinline__ void store_once(T* p) const {
    u4 w;
    __builtin_memcpy(&w, v, 16);
    __builtin_nontemporal_store(w, reinterpret_cast<u4*>(p));
  }

 private:
  typedef unsigned u4 __attribute__((ext_vector_type(4), aligned(2)));  // of its elements, at least
};

// weight times an element: a product in the type of sums, rounded to it before it
// is rounded to the element's type (one fused multiply would round once, and
// differ from what a caller gets from the two operations)
template <typename T>
__device__ __forceinline__ T times(typename ElemAcc<T>::type w, T v) {
  typename ElemAcc<T>::type p = w * (typename ElemAcc<T>::type)v;
  if constexpr (sizeof(T) == 2) asm("" : "+v"(p));  // the product is a value of its own
  return (T)p;
}

inline size_t elem_size(dpc_elem e) { return e == DPC_ELEM_F64 ? 8 : e == DPC_ELEM_F32 ? 4 : 2; }
inline bool elem_ok(dpc_elem e) {
  return e == DPC_ELEM_F64 || e == DPC_ELEM_F32 || e == DPC_ELEM_F16 || e == DPC_ELEM_BF16;
}
inline bool elem_aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

#endif  // DPC_ELEM_H
