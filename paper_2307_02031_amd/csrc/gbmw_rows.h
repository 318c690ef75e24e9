// Internal: what the norms share (rows held in registers, sums over them, shares of column sums), scales of values in 8
// bits, and the host's checks of the layer operators' arrays.  Not part of the ABI.
#pragma once
#include <algorithm>
#include <climits>
#include <cmath>

#include "gbmw_ctx.h"
#include "gbmw_dtype.h"

namespace gbmw {
namespace {

// Floats from one share of dweight or dbias to the next: each starts at 16 bytes.
__host__ __device__ constexpr int share_stride(int cols) { return (cols + 3) / 4 * 4; }

// Sums of N values over the NT threads of a row.  `scratch`: N * (NT / 64) floats of the
// row's own, others than at the last call.  Every thread of the workgroup calls it.
template <int NT, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float* scratch) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
  if constexpr (NT > 64) {
    const int t = threadIdx.x % NT;
    if (t % 64 == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) scratch[i * (NT / 64) + t / 64] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < NT / 64; ++w) s[i] += scratch[i * (NT / 64) + w];
    }
  }
}

// V elements of a row from column c on, of which those before column `from` are another piece's.
// Rows of fewer than V columns (TINY: there may be such) have one piece, of n columns.
template <int V, bool WHOLE, bool TINY>
struct Span {
  static constexpr bool kTiny = TINY;
  int c, from, n, row;
  Span() = default;
  __device__ __forceinline__ Span(int piece, int cols) : row(cols) {
    from = piece * V;
    const bool there = from < cols;
    c = there ? (WHOLE ? from : max(0, min(from, cols - V))) : 0;
    n = there ? (TINY ? min(V, cols) : V) : 0;
  }
  __device__ __forceinline__ bool has(int i) const { return WHOLE ? n > 0 : c + i >= from && i < n; }
  template <typename W>
  __device__ __forceinline__ void load(float (&x)[V], const W* row) const {   // what it does not have may be anything
    if (!TINY || this->row >= V) {
      Pack<W> r[V / kVec<W>];
      __builtin_memcpy(r, row + c, V * sizeof(W));
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = (float)r[i / kVec<W>].v[i % kVec<W>];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = i < n ? (float)row[i] : 0.0f;
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (&y)[V]) const {
    Pack<T> r;
    static_assert(V == kVec<T>, "");
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = (T)y[i];
    if (!TINY || n == V) __builtin_memcpy(row + c, &r, 16);   // shared columns are written twice, the same
    else store_pack(row, r, n);
  }
};

// The raw bytes of a thread's pieces: loaded early, looked at late.
template <typename T, int NJ, bool TINY>
struct Held {
  Pack<T> p[NJ];
  template <typename S>
  __device__ __forceinline__ void load(const S (&span)[NJ], const T* row, int cols) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if (!TINY || cols >= kVec<T>) __builtin_memcpy(&p[j], row + span[j].c, 16);
      else p[j] = load_pack(row, span[j].n);
    }
  }
};

// Of a thread's NJ pieces the first so many are whole and there, whatever the row's length
// (1024 threads have kernels of 1, 2, 4 and 8 pieces, so more than half are).
template <int NT, int NJ>
constexpr int kSure = NT < 1024 || NJ <= 2 ? NJ - 1 : NJ / 2;

template <int NT, int NJ>
constexpr bool kRunsAhead = NT < 1024 || NJ == 1;

// Sums of `parts` shares of gridDim.y arrays (dw, and db if there are two): 32 columns a workgroup,
// four of every 128th share a thread (8 threads read a line of the cache).  256 shares of 4574 columns: 4.8 us, 1.9 TB/s from the cache
// (one column a thread and half a line at a time: 7.4); 146 of 9714: 7.
template <typename W>
__global__ __launch_bounds__(1024) void k_norm_join(const float* partial, int parts, int cols, W* dw, W* db) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  __shared__ f32x4 sums[16][8];
  const int quad = threadIdx.x % 8, c = blockIdx.x * 32 + quad * 4, stride = share_stride(cols);
  W* out = blockIdx.y ? db : dw;
  if (!out) return;
  f32x4 s = {};
  if (c < cols)
#pragma unroll 4
    for (int k = threadIdx.x / 8; k < parts; k += 128)
      s += *(const f32x4*)(partial + ((int64_t)k * gridDim.y + blockIdx.y) * stride + c);
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = sum_across32(sum_across16(sum_dpp<0x128>(s[e])));   // lanes 8, 16 and 32 apart
  if (threadIdx.x % 64 < 8) sums[threadIdx.x / 64][quad] = s;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const int col = blockIdx.x * 32 + (int)threadIdx.x;
  float total = 0.0f;
#pragma unroll
  for (int w = 0; w < 16; ++w) total += sums[w][threadIdx.x / 4][threadIdx.x % 4];
  if (col < cols) out[col] = (W)total;
}

// Values in 8 bits share a scale: the largest of them over the largest code, by that one's reciprocal.  Never 0 or subnormal; a
// NaN stays.
__device__ __forceinline__ float scale_of(float most, float per_top) {
  const float s = most * per_top;
  return s < 0x1p-126f ? 0x1p-126f : s;
}

// x / scale, rounded once: the product with the rounded reciprocal is off by a unit of its last place, and what it leaves of
// x, which a fused operation has exactly, puts that right.  What is left of x is no number of 32 bits where x is below
// 2^-103: small scales are taken times 2^64, and else such an x has code 0 either way.  By a factor where registers are
// short (AdamW; a branch costs it 11), or by a branch where operations are (RMS norm, 8192 x 5120: 55 us, by a factor 59, with
// the quotient left a last place off 53).  A scale that is infinite or NaN has no reciprocal: x / inf is 0.
template <bool BRANCH, int N>
__device__ __forceinline__ void divide(float (&x)[N], float scale) {
  const bool small = scale < 0x1p-60f;
  const float up = small ? 0x1p64f : 1.0f;
  scale *= up;
  if (!BRANCH || small)
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] *= up;
  const float by = 1.0f / scale, taken = by > 0.0f ? scale : 0.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float q = x[e] * by;
    x[e] = __builtin_fmaf(-__builtin_fmaf(q, taken, -x[e]), by, q);   // with these signs -0 stays -0
  }
}

inline int element_size(int dtype) { return dtype == GBMW_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == GBMW_F32 || dtype == GBMW_F16 || dtype == GBMW_BF16; }

// Threads of a row and 16-byte pieces of each: few threads for short rows, so that the sums
// stay inside a wave, and few pieces a thread, so that they stay in registers (three of 16-bit
// values in the backward pass take 208; with four it spills).
struct Shape {
  int nt, nj;
};
inline Shape shape_of(int dtype, int cols) {
  const int vec = 16 / element_size(dtype), n = (cols + vec - 1) / vec;
  if (n <= 3 * 64) return {64, (n + 63) / 64};
  if (n <= 3 * 256) return {256, (n + 255) / 256};
  const int nj = (n + 1023) / 1024;
  return {1024, nj <= 2 ? nj : nj <= 4 ? 4 : 8};
}

inline gbmw_status check_array(const char* name, const void* ptr, int size, int64_t stride, int64_t least) {
  if (!ptr) return gbmw_detail::fail(GBMW_ERR_INVALID_ARG, "%s is null", name);
  if ((uintptr_t)ptr % (unsigned)size) return gbmw_detail::fail(GBMW_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
  if (stride < least || stride > (INT64_MAX >> 34))
    return gbmw_detail::fail(GBMW_ERR_INVALID_ARG, "%s: row stride %lld", name, (long long)stride);
  return GBMW_OK;
}

}  // namespace
}  // namespace gbmw

#define CHECK(expr)                            \
  do {                                         \
    const gbmw_status st_ = (expr);            \
    if (st_ != GBMW_OK) return st_;            \
  } while (0)
