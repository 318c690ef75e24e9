// Internal: element types of the layer operators, 16-byte pieces of rows, sums over
// a wave or a workgroup, divisions.  Not part of the ABI.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace gbmw {

using f16 = _Float16;
using bf16 = __bf16;

// Division of 0 <= n < 2^31 by a number the host knows, without the dozens of instructions that a
// division is.
struct Divisor {
  int d;
  unsigned magic;   // 2^32 / d, rounded up (0 for 1)
  __device__ __forceinline__ int of(int n) const {
    if (d == 1) return n;
    const unsigned x = __umulhi((unsigned)n, magic);   // at most one too large
    return (int)(x * (unsigned)d > (unsigned)n ? x - 1 : x);
  }
};
inline Divisor divisor(int64_t d) { return {(int)d, (unsigned)(((1ull << 32) + d - 1) / d)}; }

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

__device__ __forceinline__ double wave_sum(double x) {   // the same bits in every lane
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// x of this lane and of the lane across: halves of 32 (or 16 of each 32) exchanged between two copies
__device__ __forceinline__ float sum_across32(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float sum_across16(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
template <int CTRL>
__device__ __forceinline__ float sum_dpp(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true);
  return x + __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float wave_sum(float x) {   // the same bits in every lane
  x = sum_dpp<0xB1>(x);    // lane ^ 1
  x = sum_dpp<0x4E>(x);    // lane ^ 2
  x = sum_dpp<0x141>(x);   // the other half of eight
  x = sum_dpp<0x140>(x);   // the other half of sixteen
  return sum_across32(sum_across16(x));
}

}  // namespace gbmw
