// Layer norm (forward and backward) and gradient clipping: the memory-bound operators
// of a transformer layer's training.  Contracts: include/gbmw.h.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <vector>

#include "gbmw_rows.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

// ---- layer norm -------------------------------------------------------------------------
//
// NT threads share a row and keep it in registers, thread t the 16-byte pieces t, t + NT,
// ... (NJ of them), so the row is read once: the mean first, then the sum of the squared
// distances from it, which does not cancel where the mean is large.
//
// Where the row is no whole number of pieces, its last piece starts early enough to be whole:
// it shares its first columns with the piece before it, which count there (Span::from).
// Every load is then one unconditional instruction, and all of a row's are in flight at once.
//
// Bound by HBM; one pass over x (and dy) is its floor.  16384 x 5120 bf16: forward 57 us, 5.8 TB/s;
// backward 103 us, 4.9 TB/s, and 5 us to join the weights' shares (a large copy runs at 4.7 TB/s,
// reads and writes together).  6304 x 1283 fp32: 12 and 20 us.  512 x 1280 bf16: 3.6 us, two sums
// after one load, bound by latency.

struct NormArgs {
  int64_t rows;
  int cols;
  float eps;
  const void *x, *dy, *w, *b;
  bool wide;       // weight and bias are fp32, whatever x is
  void *y, *dx;
  int64_t xs, ys, dys, dxs;
  float *mean, *rstd;
  float* partial;  // [gridDim.x][2][share_stride(cols)]
};

constexpr int kNormFwdThreads = 256, kNormBwdThreads = 512;

// Workgroups of G rows at a time, rows blockIdx.x * G + g, then gridDim.x * G further on: a thread
// reads its columns of weight and bias once, and the next row is on its way while one is worked on
// (not with several pieces for each of 1024 threads, which have half the registers).
template <typename T, int NT, int NJ, bool WHOLE>
__global__ __launch_bounds__(NT < kNormFwdThreads ? kNormFwdThreads : NT) void k_norm_fwd(NormArgs a) {
  constexpr int V = kVec<T>, G = (NT < kNormFwdThreads ? kNormFwdThreads : NT) / NT;
  constexpr bool kAhead = kRunsAhead<NT, NJ>;
  __shared__ float scratch[2][G][NT / 64];
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  constexpr bool kTiny = !WHOLE && NT * NJ == 64;
  Span<V, WHOLE, kTiny> span[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) span[j] = Span<V, WHOLE, kTiny>(t + j * NT, a.cols);
  Held<T, NJ, kTiny> x, next;
  auto fetch = [&](int64_t row) { next.load(span, (const T*)a.x + (row < a.rows ? row : 0) * a.xs, a.cols); };
  const int64_t step = (int64_t)gridDim.x * G;
  fetch((int64_t)blockIdx.x * G + g);
  float w[NJ][V], b[NJ][V];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[j][i] = 1.0f, b[j][i] = 0.0f;
    if (a.w) a.wide ? span[j].load(w[j], (const float*)a.w) : span[j].load(w[j], (const T*)a.w);
    if (a.b) a.wide ? span[j].load(b[j], (const float*)a.b) : span[j].load(b[j], (const T*)a.b);
  }
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.rows; first += step) {
    const int64_t row = first + g;
    x = next;
    if constexpr (kAhead) fetch(row + step);
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += j < kSure<NT, NJ> || span[j].has(i) ? (float)x.p[j].v[i] : 0.0f;
    row_sum<NT>(s, scratch[0][g]);
    const float mean = s[0] / (float)a.cols;
    s[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = j < kSure<NT, NJ> || span[j].has(i) ? (float)x.p[j].v[i] - mean : 0.0f;
        s[0] = __builtin_fmaf(d, d, s[0]);
      }
    row_sum<NT>(s, scratch[1][g]);
    const float rstd = 1.0f / __builtin_sqrtf(s[0] / (float)a.cols + a.eps);
    if (row < a.rows) {
      if (t == 0) a.mean[row] = mean, a.rstd[row] = rstd;
      T* y = (T*)a.y + row * a.ys;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (span[j].n == 0) continue;
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = __builtin_fmaf(((float)x.p[j].v[i] - mean) * rstd, w[j][i], b[j][i]);
        span[j].store(y, out);
      }
    }
    if constexpr (!kAhead) fetch(row + step);
  }
}

// Whether one workgroup of k_norm_bwd has a compute unit to itself.
template <typename T, int NT, int NJ>
constexpr bool kOne = NT == 1024 || (sizeof(T) == 2 && NJ == 3);

// The same walk over the rows.  A thread keeps its columns' share of dweight and dbias in
// registers over all its rows; the workgroup's shares go to `partial` and k_norm_join adds them
// up in a fixed order, so the result does not depend on which workgroup ends first.  weight waits
// in LDS (the registers are taken) by pieces, four columns of each after the other, so that a wave
// reads 16 bytes a lane one after the other.  13673 x 4574 bf16, whose last piece starts early:
// 75 us; with weight read by columns, every column masked and rows shorter than a piece allowed
// for where there are none, 176.
//
// Rows that are not there are masked (kOne) or branched around.  A mask lets the compiler keep all
// converted values from the sums to dx, in 200 registers: better where only one workgroup fits
// anyway (16384 x 5120 bf16: 103 us, with a branch 108), worse where it makes one of two (20000 x
// 768 in 32 bits: 38 us, with a branch 34).
template <typename T, int NT, int NJ, bool WHOLE>
__global__ __launch_bounds__(NT < kNormBwdThreads ? kNormBwdThreads : NT) void k_norm_bwd(NormArgs a) {
  constexpr int V = kVec<T>, G = (NT < kNormBwdThreads ? kNormBwdThreads : NT) / NT;
  constexpr bool kAhead = kRunsAhead<NT, NJ>;
  __shared__ float scratch[2][G][2 * (NT / 64)];
  extern __shared__ __attribute__((aligned(16))) float columns[];   // [V/4][pieces][4] weight, then [cols] shares
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  constexpr bool kTiny = !WHOLE && NT * NJ == 64;
  Span<V, WHOLE, kTiny> span[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) span[j] = Span<V, WHOLE, kTiny>(t + j * NT, a.cols);
  Held<T, NJ, kTiny> x, dy, next_x, next_dy;
  float mean, rstd, next_mean, next_rstd;
  auto fetch = [&](int64_t row) {
    const int64_t at = row < a.rows ? row : 0;
    next_x.load(span, (const T*)a.x + at * a.xs, a.cols);
    next_dy.load(span, (const T*)a.dy + at * a.dys, a.cols);
    next_mean = a.mean[at], next_rstd = a.rstd[at];
  };
  const int64_t step = (int64_t)gridDim.x * G;
  fetch((int64_t)blockIdx.x * G + g);
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const int pieces = (a.cols + V - 1) / V;
  f32x4* weight = (f32x4*)columns;
  for (int k = threadIdx.x; k < pieces; k += blockDim.x) {
    const Span<V, WHOLE, kTiny> s(k, a.cols);
    float w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = 1.0f;
    if (a.w) a.wide ? s.load(w, (const float*)a.w) : s.load(w, (const T*)a.w);
#pragma unroll
    for (int q = 0; q < V / 4; ++q) weight[q * pieces + k] = f32x4{w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]};
  }
  __syncthreads();
  auto weight_of = [&](int j, float (&w)[V]) {
    const int k = span[j].from / V;
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const f32x4 r = weight[q * pieces + (j < kSure<NT, NJ> || k < pieces ? k : 0)];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * q + i] = r[i];
    }
  };
  float dw[NJ][V] = {}, db[NJ][V] = {};
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.rows; first += step, turn ^= 1) {
    const int64_t row = first + g;
    const bool live = row < a.rows;
    x = next_x, dy = next_dy, mean = next_mean, rstd = next_rstd;
    if constexpr (kAhead) fetch(row + step);
    float s[2] = {0.0f, 0.0f};
    if (kOne<T, NT, NJ> || live) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float w[V];
        weight_of(j, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const bool has = (live || !kOne<T, NT, NJ>) && (j < kSure<NT, NJ> || span[j].has(i));
          const float xhat = has ? ((float)x.p[j].v[i] - mean) * rstd : 0.0f, d = has ? (float)dy.p[j].v[i] : 0.0f;
          dw[j][i] = __builtin_fmaf(d, xhat, dw[j][i]);
          db[j][i] += d;
          s[0] = __builtin_fmaf(d, w[i], s[0]);
          s[1] = __builtin_fmaf(d * w[i], xhat, s[1]);
        }
      }
    }
    row_sum<NT>(s, scratch[turn][g]);
    const float c1 = s[0] / (float)a.cols, c2 = s[1] / (float)a.cols;
    if (live) {
      T* dx = (T*)a.dx + row * a.dxs;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (span[j].n == 0) continue;
        float w[V], out[V];
        weight_of(j, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float xhat = ((float)x.p[j].v[i] - mean) * rstd;
          out[i] = __builtin_fmaf(-xhat, c2, __builtin_fmaf((float)dy.p[j].v[i], w[i], -c1)) * rstd;
        }
        span[j].store(dx, out);
      }
    }
    if constexpr (!kAhead) fetch(row + step);
  }
  if (!a.partial) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    for (int k = 0; k < G; ++k) {   // one row's threads after the other add their share
      __syncthreads();
      if (g == k)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int c = span[j].c + i;
            const float v = which ? db[j][i] : dw[j][i];
            if (span[j].has(i)) columns[c] = k ? columns[c] + v : v;
          }
    }
    __syncthreads();
    float* out = a.partial + ((int64_t)blockIdx.x * 2 + which) * share_stride(a.cols);
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) out[c] = columns[c];
  }
}

// ---- gradient norm and clipping -----------------------------------------------------------
//
// Two launches, bound by HBM: one reads every gradient for the norm, one reads and writes them
// all, because no value can be written before the last has been read.  236M bf16 gradients into
// fp32: together 342 us (387 with ordinary stores), 1.9 GB at 5.5 TB/s; 20M fp32 ones: 39 us (49).
// Squares are added in fp64, at a few per cent of its rate: nothing overflows, and the norm is
// right to the last bit of fp32.
//
// A factor below fp32's normal numbers (gradients near the largest ones, whose norm fp32 may not
// hold) would lose its digits, so it is taken with an exponent of its own.
struct Factor {
  float value;   // times 2^exponent
  int exponent = 0;
  __device__ __forceinline__ explicit Factor(double factor) : value((float)factor) {
    if (factor < 0x1p-126 && (double)value != factor) value = (float)frexp(factor, &exponent);
  }
  __device__ __forceinline__ bool is_one() const { return value == 1.0f && exponent == 0; }
  __device__ __forceinline__ float of(float x) const { return __builtin_ldexpf(x * value, exponent); }
};

struct Piece {   // a run of at most kPiece elements of one tensor
  const void* in;
  void* out;
  int32_t n, in_dtype, out_dtype, unused;
};
constexpr int64_t kPiece = 32768;
constexpr int kNormGroups = 2048;   // at most so many partial sums
constexpr int kUnroll = 4;          // loads in flight of a thread

// Sum over the 256 threads of a workgroup, the same bits in each of them.
__device__ __forceinline__ double group_sum(double s, double (&sums)[4]) {
  s = wave_sum(s);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
  __syncthreads();
  return (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

template <typename T>
__device__ __forceinline__ void add_squares(const Piece& pc, double (&part)[8]) {
  constexpr int V = kVec<T>, U = kUnroll;
  const T* in = (const T*)pc.in;
  auto add = [&](const Pack<T>& x) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const double d = (double)(float)x.v[e];
      part[e] = __builtin_fma(d, d, part[e]);
    }
  };
  int i = threadIdx.x * V;
  for (; i + ((U - 1) * 256 + 1) * V <= pc.n; i += U * 256 * V) {
    Pack<T> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(&x[u], in + i + u * 256 * V, 16);
#pragma unroll
    for (int u = 0; u < U; ++u) add(x[u]);
  }
  for (; i < pc.n; i += 256 * V) add(load_pack(in + i, pc.n - i));
}

// Tensors of several types may be in one list: which, is the same for a whole workgroup.
__global__ __launch_bounds__(256) void k_clip_norm(const Piece* pieces, int count, double* partial) {
  __shared__ double sums[4];
  double part[8] = {};
  for (int k = blockIdx.x; k < count; k += gridDim.x) {
    const Piece pc = pieces[k];
    if (pc.in_dtype == GBMW_F32) add_squares<float>(pc, part);
    else if (pc.in_dtype == GBMW_F16) add_squares<f16>(pc, part);
    else add_squares<bf16>(pc, part);
  }
  double s = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += part[e];
  s = group_sum(s, sums);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// STREAM: the stores pass the cache by (a wave's are whole lines of it), so that what is still to
// be read stays there.
template <typename T, typename O, bool STREAM>
__device__ __forceinline__ void scale_piece(const Piece& pc, Factor factor) {
  constexpr int V = kVec<O>, U = kUnroll;   // as many elements as a store of 16 bytes takes
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const T* in = (const T*)pc.in;
  O* out = (O*)pc.out;
  int i = threadIdx.x * V;
  for (; i + ((U - 1) * 256 + 1) * V <= pc.n; i += U * 256 * V) {
    T x[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(&x[u], in + i + u * 256 * V, V * sizeof(T));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Pack<O> y;
#pragma unroll
      for (int e = 0; e < V; ++e) y.v[e] = (O)factor.of((float)x[u][e]);
      if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(f32x4, y), (f32x4*)(out + i + u * 256 * V));
      else __builtin_memcpy(out + i + u * 256 * V, &y, 16);
    }
  }
  for (; i < pc.n; i += 256 * V)
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (i + e < pc.n) out[i + e] = (O)factor.of((float)in[i + e]);
}

template <typename T, typename O>
__device__ __forceinline__ void scale_piece(const Piece& pc, Factor factor) {
  if ((uintptr_t)pc.out % 128 == 0) scale_piece<T, O, true>(pc, factor);
  else scale_piece<T, O, false>(pc, factor);
}

// Every workgroup adds the `parts` partial sums itself, in one order: 16 KB from the cache at
// most, and no workgroup has to wait for another or to make its sum visible to others before its
// kernel ends (which costs each of them a pass over its die's cache).
// The pieces last read by the norm come first: they may still be in the cache.
__global__ __launch_bounds__(256) void k_clip_scale(const Piece* pieces, int count, const double* partial, int parts,
                                                    double max_norm, double scale, float* norm_out) {
  __shared__ double sums[4];
  double s = 0.0;
#pragma unroll 8
  for (int k = threadIdx.x; k < parts; k += 256) s += partial[k];
  const double norm = __builtin_sqrt(group_sum(s, sums)) * scale;
  const bool clips = norm > max_norm && norm < __builtin_inf();
  const Factor factor(clips ? scale * (max_norm / norm) : scale);
  if (blockIdx.x == 0 && threadIdx.x == 0 && norm_out) *norm_out = (float)norm;
  for (int k = count - 1 - (int)blockIdx.x; k >= 0; k -= gridDim.x) {
    const Piece pc = pieces[k];
    if (factor.is_one() && pc.in == pc.out) continue;   // the values are there
    if (pc.in_dtype == GBMW_F32) scale_piece<float, float>(pc, factor);
    else if (pc.in_dtype == GBMW_F16 && pc.out_dtype == GBMW_F16) scale_piece<f16, f16>(pc, factor);
    else if (pc.in_dtype == GBMW_F16) scale_piece<f16, float>(pc, factor);
    else if (pc.out_dtype == GBMW_BF16) scale_piece<bf16, bf16>(pc, factor);
    else scale_piece<bf16, float>(pc, factor);
  }
}

// ---- host ---------------------------------------------------------------------------------

gbmw_status check_norm(const gbmw_layer_norm_problem* p) {
  if (!p) return fail(GBMW_ERR_INVALID_ARG, "null problem");
  if (!known_dtype(p->dtype)) return fail(GBMW_ERR_INVALID_ARG, "dtype=%d", p->dtype);
  if (p->wdtype != p->dtype && p->wdtype != GBMW_F32)
    return fail(GBMW_ERR_INVALID_ARG, "wdtype=%d is neither dtype nor GBMW_F32", p->wdtype);
  if (p->rows < 0 || p->rows > INT32_MAX) return fail(GBMW_ERR_INVALID_ARG, "rows=%lld", (long long)p->rows);
  if (p->cols < 1 || p->cols > 32768) return fail(GBMW_ERR_INVALID_ARG, "cols=%d not in 1..32768", p->cols);
  return GBMW_OK;
}

// Workgroups: as many as the chip holds at a time, each with several rows where there are many, and
// no more than it takes for the most that one of them has.  Forward, two of 1024 threads with a
// piece each fit (4000 x 8192 bf16: 25 us, with one 30), of more pieces one does.  Backward, every one more costs a row of
// shares to write and read: with 16-bit values and three pieces a thread, or with 1024 threads, only
// one fits a compute unit's registers (16384 x 5120: 103 us and 5 to join them); else two do (6304 x
// 1283 in 32 bits: 20 us, with half as many 34).
int norm_groups(const gbmw_layer_norm_problem* p, bool backward) {
  const Shape s = shape_of(p->dtype, p->cols);
  const int per = std::max(1, (backward ? kNormBwdThreads : kNormFwdThreads) / s.nt);
  const bool one = s.nt == 1024 || (s.nj == 3 && p->dtype != GBMW_F32);   // kOne
  const int64_t most = !backward ? s.nt < 1024 ? 2048 : s.nj == 1 ? 512 : 256 : one ? 256 : 512, all = (p->rows + per - 1) / per;
  if (all <= most) return (int)all;
  const int64_t turns = (all + most - 1) / most;   // of the one that has most rows: no more workgroups than that takes
  return (int)((all + turns - 1) / turns);
}

template <typename T, int NT, int NJ, bool WHOLE>
gbmw_status launch_norm(const NormArgs& a, bool backward, int groups, hipStream_t st) {
  if (!backward) {
    hipLaunchKernelGGL((k_norm_fwd<T, NT, NJ, WHOLE>), dim3(groups), dim3(std::max(NT, kNormFwdThreads)), 0, st, a);
  } else {
    const size_t lds = 16 * (size_t)((a.cols + kVec<T> - 1) / kVec<T>) * (kVec<T> / 4);
    if (lds > 60 * 1024) {
      const hipError_t e = hipFuncSetAttribute((const void*)&k_norm_bwd<T, NT, NJ, WHOLE>,
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(GBMW_ERR_DEVICE, "%zu bytes of shared memory: %s", lds, hipGetErrorString(e));
      }
    }
    hipLaunchKernelGGL((k_norm_bwd<T, NT, NJ, WHOLE>), dim3(groups), dim3(std::max(NT, kNormBwdThreads)), lds, st, a);
  }
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

template <typename T, int NT, int NJ>
gbmw_status launch_norm(const NormArgs& a, bool backward, int groups, hipStream_t st) {
  return a.cols % kVec<T> ? launch_norm<T, NT, NJ, false>(a, backward, groups, st)
                          : launch_norm<T, NT, NJ, true>(a, backward, groups, st);
}

template <typename T>
gbmw_status launch_norm(const NormArgs& a, Shape s, bool backward, int groups, hipStream_t st) {
  if (s.nt == 64) switch (s.nj) {
    case 1: return launch_norm<T, 64, 1>(a, backward, groups, st);
    case 2: return launch_norm<T, 64, 2>(a, backward, groups, st);
    default: return launch_norm<T, 64, 3>(a, backward, groups, st);
  }
  if (s.nt == 256) switch (s.nj) {
    case 1: return launch_norm<T, 256, 1>(a, backward, groups, st);
    case 2: return launch_norm<T, 256, 2>(a, backward, groups, st);
    default: return launch_norm<T, 256, 3>(a, backward, groups, st);
  }
  if (s.nj == 1) return launch_norm<T, 1024, 1>(a, backward, groups, st);
  if (s.nj == 2) return launch_norm<T, 1024, 2>(a, backward, groups, st);
  if (s.nj == 4) return launch_norm<T, 1024, 4>(a, backward, groups, st);
  if constexpr (sizeof(T) == 4) return launch_norm<T, 1024, 8>(a, backward, groups, st);
  return fail(GBMW_ERR_UNSUPPORTED, "no kernel for %d columns", a.cols);
}

gbmw_status launch_norm(const gbmw_layer_norm_problem* p, const NormArgs& a, bool backward, int groups) {
  const Shape s = shape_of(p->dtype, p->cols);
  hipStream_t st = (hipStream_t)p->stream;
  if (p->dtype == GBMW_F32) return launch_norm<float>(a, s, backward, groups, st);
  if (p->dtype == GBMW_F16) return launch_norm<f16>(a, s, backward, groups, st);
  return launch_norm<bf16>(a, s, backward, groups, st);
}

}  // namespace
}  // namespace gbmw

using namespace gbmw;

extern "C" int64_t gbmw_layer_norm_workspace(const gbmw_layer_norm_problem* p) {
  gbmw_detail::clear_error();
  if (check_norm(p) != GBMW_OK) return -1;
  return (int64_t)norm_groups(p, true) * 2 * share_stride(p->cols) * 4;
}

extern "C" gbmw_status gbmw_layer_norm_forward(const gbmw_layer_norm_problem* p) {
  gbmw_detail::clear_error();
  CHECK(check_norm(p));
  if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return fail(GBMW_ERR_INVALID_ARG, "eps=%g", (double)p->eps);
  if (p->rows == 0) return GBMW_OK;
  const int size = element_size(p->dtype), wsize = element_size(p->wdtype);
  CHECK(check_array("x", p->x, size, p->x_stride, 0));
  CHECK(check_array("y", p->y, size, p->y_stride, p->cols));
  CHECK(check_array("mean", p->mean, 4, 1, 0));
  CHECK(check_array("rstd", p->rstd, 4, 1, 0));
  if (p->weight) CHECK(check_array("weight", p->weight, wsize, 1, 0));
  if (p->bias) CHECK(check_array("bias", p->bias, wsize, 1, 0));
  if (p->x == p->y && p->x_stride != p->y_stride)
    return fail(GBMW_ERR_INVALID_ARG, "y is x, with another row stride");
  NormArgs a{};
  a.rows = p->rows, a.cols = p->cols, a.eps = p->eps;
  a.x = p->x, a.w = p->weight, a.b = p->bias, a.y = p->y, a.wide = p->wdtype == GBMW_F32;
  a.xs = p->x_stride, a.ys = p->y_stride, a.mean = p->mean, a.rstd = p->rstd;
  return launch_norm(p, a, false, norm_groups(p, false));
}

extern "C" gbmw_status gbmw_layer_norm_backward(const gbmw_layer_norm_problem* p) {
  gbmw_detail::clear_error();
  CHECK(check_norm(p));
  const int size = element_size(p->dtype), wsize = element_size(p->wdtype);
  const bool wanted = p->dweight || p->dbias;
  if (p->dweight) CHECK(check_array("dweight", p->dweight, wsize, 1, 0));
  if (p->dbias) CHECK(check_array("dbias", p->dbias, wsize, 1, 0));
  if (p->rows > 0) {
    CHECK(check_array("x", p->x, size, p->x_stride, 0));
    CHECK(check_array("dy", p->dy, size, p->dy_stride, 0));
    CHECK(check_array("dx", p->dx, size, p->dx_stride, p->cols));
    CHECK(check_array("mean", p->mean, 4, 1, 0));
    CHECK(check_array("rstd", p->rstd, 4, 1, 0));
    if (p->weight) CHECK(check_array("weight", p->weight, wsize, 1, 0));
    if (p->dx == p->dy && p->dx_stride != p->dy_stride)
      return fail(GBMW_ERR_INVALID_ARG, "dx is dy, with another row stride");
  }
  const int groups = norm_groups(p, true);
  if (wanted && p->rows > 0) {
    const int64_t need = (int64_t)groups * 2 * share_stride(p->cols) * 4;
    if (!p->workspace || p->workspace_bytes < need || (uintptr_t)p->workspace % 16)
      return fail(GBMW_ERR_INVALID_ARG, "workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
  }
  if (p->rows > 0) {
    NormArgs a{};
    a.rows = p->rows, a.cols = p->cols;
    a.x = p->x, a.dy = p->dy, a.w = p->weight, a.dx = p->dx, a.wide = p->wdtype == GBMW_F32;
    a.xs = p->x_stride, a.dys = p->dy_stride, a.dxs = p->dx_stride, a.mean = p->mean, a.rstd = p->rstd;
    a.partial = wanted ? (float*)p->workspace : nullptr;
    CHECK(launch_norm(p, a, true, groups));
  }
  if (wanted) {   // without rows: zeros
    const dim3 grid((p->cols + 31) / 32, 2);
    hipStream_t st = (hipStream_t)p->stream;
    const float* part = (const float*)p->workspace;
    if (p->wdtype == GBMW_F32)
      hipLaunchKernelGGL(k_norm_join<float>, grid, dim3(1024), 0, st, part, groups, p->cols, (float*)p->dweight,
                         (float*)p->dbias);
    else if (p->wdtype == GBMW_F16)
      hipLaunchKernelGGL(k_norm_join<f16>, grid, dim3(1024), 0, st, part, groups, p->cols, (f16*)p->dweight,
                         (f16*)p->dbias);
    else
      hipLaunchKernelGGL(k_norm_join<bf16>, grid, dim3(1024), 0, st, part, groups, p->cols, (bf16*)p->dweight,
                         (bf16*)p->dbias);
    HIP_TRY(hipGetLastError());
  }
  return GBMW_OK;
}

struct gbmw_gradient_list {
  gbmw_detail::DevBuf buf;   // partial sums | pieces
  int count = 0, device = 0;
  bool writes = true;        // else it is for the norm alone
  double* partial() const { return (double*)buf.p; }
  Piece* pieces() const { return (Piece*)((char*)buf.p + 8 * kNormGroups); }
};

extern "C" gbmw_status gbmw_gradient_list_create(int32_t n, const void* const* in, void* const* out,
                                                 const int64_t* numel, const int32_t* in_dtype,
                                                 const int32_t* out_dtype, gbmw_gradient_list** list) {
  gbmw_detail::clear_error();
  if (!list) return fail(GBMW_ERR_INVALID_ARG, "null list");
  *list = nullptr;
  if (n < 0 || (n > 0 && (!in || !numel || !in_dtype || (out && !out_dtype))))
    return fail(GBMW_ERR_INVALID_ARG, "n=%d, or a null array", n);
  const bool writes = out;
  if (!writes) out = const_cast<void* const*>(in), out_dtype = in_dtype;
  int64_t count = 0;
  for (int i = 0; i < n; ++i) {
    if (!known_dtype(in_dtype[i])) return fail(GBMW_ERR_INVALID_ARG, "in_dtype[%d]=%d", i, in_dtype[i]);
    if (out_dtype[i] != in_dtype[i] && out_dtype[i] != GBMW_F32)
      return fail(GBMW_ERR_INVALID_ARG, "out_dtype[%d]=%d is neither the gradient's nor GBMW_F32", i, out_dtype[i]);
    const int isize = element_size(in_dtype[i]), osize = element_size(out_dtype[i]);
    if (numel[i] < 0 || numel[i] > (1ll << 41)) return fail(GBMW_ERR_INVALID_ARG, "numel[%d]=%lld", i, (long long)numel[i]);
    if (numel[i] == 0) continue;
    if (!in[i] || !out[i]) return fail(GBMW_ERR_INVALID_ARG, "tensor %d is null", i);
    if ((uintptr_t)in[i] % (unsigned)isize || (uintptr_t)out[i] % (unsigned)osize)
      return fail(GBMW_ERR_INVALID_ARG, "tensor %d is not aligned to its elements", i);
    if (in[i] == out[i] && isize != osize) return fail(GBMW_ERR_INVALID_ARG, "tensor %d: in place, with another type", i);
    count += (numel[i] + kPiece - 1) / kPiece;
  }
  if (count > (1 << 26)) return fail(GBMW_ERR_INVALID_ARG, "more than 2^41 elements");
  try {
    std::vector<Piece> pieces;
    pieces.reserve((size_t)count);
    for (int i = 0; i < n; ++i)
      for (int64_t at = 0; at < numel[i]; at += kPiece)
        pieces.push_back({(const char*)in[i] + at * element_size(in_dtype[i]), (char*)out[i] + at * element_size(out_dtype[i]),
                          (int32_t)std::min(kPiece, numel[i] - at), in_dtype[i], out_dtype[i], 0});
    gbmw_gradient_list* l = new gbmw_gradient_list;
    l->count = (int)count, l->writes = writes;
    const size_t head = 8 * kNormGroups;
    gbmw_status st = l->buf.reserve(head + sizeof(Piece) * (size_t)count);
    if (st == GBMW_OK) {
      hipError_t e = hipGetDevice(&l->device);
      if (e == hipSuccess && count)
        e = hipMemcpy(l->pieces(), pieces.data(), sizeof(Piece) * (size_t)count, hipMemcpyHostToDevice);
      if (e != hipSuccess) {
        (void)hipGetLastError();
        st = fail(GBMW_ERR_DEVICE, "gradient list: %s", hipGetErrorString(e));
      }
    }
    if (st != GBMW_OK) {
      l->buf.release();
      delete l;
      return st;
    }
    *list = l;
    return GBMW_OK;
  } catch (const std::bad_alloc&) {
    return fail(GBMW_ERR_OOM, "host memory for %lld pieces", (long long)count);
  }
}

extern "C" gbmw_status gbmw_clip_gradients(gbmw_gradient_list* l, float max_norm, float scale, float* norm,
                                           void* stream) {
  gbmw_detail::clear_error();
  if (!l) return fail(GBMW_ERR_INVALID_ARG, "null list");
  if (!(max_norm > 0.0f)) return fail(GBMW_ERR_INVALID_ARG, "max_norm=%g is not positive", (double)max_norm);
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(GBMW_ERR_INVALID_ARG, "scale=%g", (double)scale);
  if ((uintptr_t)norm % 4) return fail(GBMW_ERR_INVALID_ARG, "norm is not aligned to a float");
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != l->device) return fail(GBMW_ERR_INVALID_ARG, "the list is on device %d, device %d is current", l->device, dev);
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid(std::max(1, std::min(l->count, kNormGroups))), block(256);
  hipLaunchKernelGGL(k_clip_norm, grid, block, 0, st, l->pieces(), l->count, l->partial());
  // without outputs one workgroup writes the norm
  hipLaunchKernelGGL(k_clip_scale, l->writes ? grid : dim3(1), block, 0, st, l->pieces(), l->writes ? l->count : 0, l->partial(),
                     (int)grid.x, (double)max_norm, (double)scale, norm);
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

extern "C" void gbmw_gradient_list_destroy(gbmw_gradient_list* l) {
  if (!l) return;
  int current = l->device;
  (void)hipGetDevice(&current);
  if (current != l->device) (void)hipSetDevice(l->device);
  (void)hipDeviceSynchronize();
  l->buf.release();
  if (current != l->device) (void)hipSetDevice(current);
  delete l;
}
