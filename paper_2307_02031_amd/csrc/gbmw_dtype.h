// Internal: element types of the layer operators, 16-byte pieces of rows, sums over
// a wave or a workgroup.  Not part of the ABI.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace gbmw {

using f16 = _Float16;
using bf16 = __bf16;

// As many elements as 16 bytes hold.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

template <typename T>
struct alignas(sizeof(T)) Pack {   // no more aligned than one element: rows may start anywhere
  T v[kVec<T>];
};

// n (clipped to 0..kVec) elements at p, zeros behind them.  Whole pieces are one load; the
// hardware takes global addresses of any alignment.
template <typename T>
__device__ __forceinline__ Pack<T> load_pack(const T* p, int n) {
  Pack<T> r;
  if (n >= kVec<T>) {
    __builtin_memcpy(&r, p, 16);
  } else {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) r.v[i] = i < n ? p[i] : (T)0.0f;
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void store_pack(T* p, const Pack<T>& r, int n) {
  if (n >= kVec<T>) {
    __builtin_memcpy(p, &r, 16);
  } else {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
      if (i < n) p[i] = r.v[i];
  }
}

template <typename V>
__device__ __forceinline__ V wave_sum(V x) {   // the same bits in every lane
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

}  // namespace gbmw
