// RMS norm after a residual's addition, to the arrays' type or to 8 bits with scales, and its
// backward pass.  Contract: include/gbmw.h.
#include "gbmw_rows.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

// NT threads hold a row in registers, as in layer norm, a wave four rows where a quarter of it holds one: one pass
// over x and the residual, one sum, and for 8 bits the largest of a group's threads.
//
// Bound by HBM.  16384 x 5120 bf16 with a residual: forward 113 us, 5.9 TB/s; backward 125, 5.4 TB/s, of
// which 5 to join the shares of dweight.  8192 x 5120 to 8 bits, a scale for each 128 columns: 54 us, 5.4 TB/s (int8 56).  4 x 5120:
// 4.4 us, latency of a load, a sum and a store.  Rows at odd addresses (16-bit values, an odd number a row) cost up to
// 1.4 times as much (4096 x 10001 102 us, 4096 x 10002 72); rows beyond 16384 columns spill in the backward pass
// (2048 x 20000 bf16: 139 us, forward 62; 512 x 30000 100, 1024 x 32768 fp32 265: 2 to 4 times what their bytes take).
struct RmsArgs {
  int64_t rows;
  int cols;
  float eps;
  const void *x, *res, *w, *dy, *dres;
  bool wide;       // weight is fp32, whatever x is
  void *h, *y, *dx;
  uint8_t* q;
  int64_t xs, rs, hs, ys, qs, dys, drs, dxs;
  bool whole_numbers;   // q is GBMW_I8
  int group, groups;    // columns of a scale, or 0; scales of a row
  float *scale, *rstd;
  float* partial;  // [gridDim.x][share_stride(cols)], with more than one workgroup
  void* dw;        // dweight
  bool stream;     // past the cache
};

constexpr int kRmsFwdThreads = 256, kRmsBwdThreads = 512;
// Rows that a workgroup has at a time.
template <int NT, bool BACKWARD>
constexpr int kRows = NT < (BACKWARD ? kRmsBwdThreads : kRmsFwdThreads) ? (BACKWARD ? kRmsBwdThreads : kRmsFwdThreads) / NT : 1;

template <int WORDS>
using Words = uint32_t __attribute__((ext_vector_type(WORDS), aligned(1)));

// A thread's pieces of a row, as they are.  STREAM: past the cache.
template <bool STREAM, typename T, int NJ, typename S>
__device__ __forceinline__ void load_row(Pack<T> (&p)[NJ], const S (&span)[NJ], const T* row) {
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (!S::kTiny || span[j].row >= kVec<T>) {
      if constexpr (STREAM) {
        const auto w = __builtin_nontemporal_load((const Words<4>*)(row + span[j].c));
        __builtin_memcpy(&p[j], &w, 16);
      } else {
        __builtin_memcpy(&p[j], row + span[j].c, 16);
      }
    } else {
      p[j] = load_pack(row, span[j].n);
    }
  }
}
template <bool STREAM, typename T, typename S, int V>
__device__ __forceinline__ void store_row(const S& span, T* row, const float (&y)[V]) {
  if constexpr (STREAM) {
    if (!S::kTiny || span.n == V) {
      Pack<T> r;
#pragma unroll
      for (int i = 0; i < V; ++i) r.v[i] = (T)y[i];
      Words<4> w;
      __builtin_memcpy(&w, &r, 16);
      __builtin_nontemporal_store(w, (Words<4>*)(row + span.c));
      return;
    }
  }
  span.store(row, y);
}

// Sum over the NT threads of a row, of which a wave may have four.  `scratch`: NT / 64 floats of the row's own.
template <int NT>
__device__ __forceinline__ float sum_of_row(float x, float* scratch) {
  if constexpr (NT == 16) {
    return sum_dpp<0x140>(sum_dpp<0x141>(sum_dpp<0x4E>(sum_dpp<0xB1>(x))));
  } else {
    float s[1] = {x};
    row_sum<NT>(s, scratch);
    return s[0];
  }
}

template <int NT>
constexpr int kWaves = NT < 64 ? 1 : NT / 64;   // of a row

// Largest of |x| as bits: a NaN is larger than any number, and stays.
__device__ __forceinline__ unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }

template <int CTRL>
__device__ __forceinline__ unsigned max_dpp(unsigned x) {
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}
// Over the aligned lanes of which this is one (4, 8, 16, 32 or 64): the same in each of them.
__device__ __forceinline__ unsigned lanes_max(unsigned x, int lanes) {
  x = max_dpp<0xB1>(x);                      // lane ^ 1
  x = max_dpp<0x4E>(x);                      // lane ^ 2
  if (lanes > 4) x = max_dpp<0x141>(x);      // the other half of eight
  if (lanes > 8) x = max_dpp<0x140>(x);      // the other half of sixteen
  if (lanes > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((unsigned)r[0], (unsigned)r[1]);
  }
  if (lanes > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = max((unsigned)r[0], (unsigned)r[1]);
  }
  return x;
}

// V values over their scale in 8 bits, four in a word.
template <int V>
__device__ __forceinline__ void to_codes(const float (&x)[V], bool whole_numbers, unsigned (&code)[V / 4]) {
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    if (whole_numbers) {
      code[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = (int)__builtin_fminf(__builtin_fmaxf(__builtin_rintf(x[4 * i + e]), -127.0f), 127.0f);
        code[i] |= (unsigned)(n & 255) << (8 * e);
      }
    } else {
      int word = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
      code[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], word, true);
    }
  }
}

template <typename T, int NT, int NJ, bool WHOLE, bool STREAM>
__global__ __launch_bounds__((NT * kRows<NT, false>)) void k_rms_fwd(RmsArgs a) {
  constexpr int V = kVec<T>, G = kRows<NT, false>;
  __shared__ float scratch[2][G][kWaves<NT>];
  __shared__ unsigned most_of[G][kWaves<NT>];
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  Span<V, WHOLE, !WHOLE && NT * NJ == 16> span[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) span[j] = {t + j * NT, a.cols};
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.rows; first += (int64_t)gridDim.x * G, turn ^= 1) {
    const int64_t row = first + g, at = row < a.rows ? row : 0;
    Pack<T> h[NJ], r[NJ];
    load_row<STREAM>(h, span, (const T*)a.x + at * a.xs);
    if (a.res) load_row<STREAM>(r, span, (const T*)a.res + at * a.rs);
    // weight's loads go out with the row's, but where the row fills the registers (1024 x 32768 fp32: 99 us, else 142)
    constexpr bool kLate = NT == 1024 && NJ > 2;
    float w[kLate ? 1 : NJ][V];
    auto weight_of = [&](int j, float (&w)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = 1.0f;
      if (a.w) a.wide ? span[j].load(w, (const float*)a.w) : span[j].load(w, (const T*)a.w);
    };
    if constexpr (!kLate)
#pragma unroll
      for (int j = 0; j < NJ; ++j) weight_of(j, w[j]);
    if (a.res) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) h[j].v[i] = (T)((float)h[j].v[i] + (float)r[j].v[i]);
    }
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = j < kSure<NT, NJ> || span[j].has(i) ? (float)h[j].v[i] : 0.0f;
        s = __builtin_fmaf(d, d, s);
      }
    // stores come after the sum, which has every thread's values of the row: it may be written in place
    s = sum_of_row<NT>(s, scratch[turn][g]);
    const float rstd = 1.0f / __builtin_sqrtf(s / (float)a.cols + a.eps);
    const bool live = row < a.rows;
    auto normed = [&](int j, float (&y)[V]) {
      if constexpr (kLate) weight_of(j, w[0]);
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = (float)h[j].v[i] * rstd * w[kLate ? 0 : j][i];
    };
    if (live) {
      if (t == 0 && a.rstd) a.rstd[row] = rstd;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (span[j].n == 0) continue;
        float y[V];
        if (a.h) {
#pragma unroll
          for (int i = 0; i < V; ++i) y[i] = (float)h[j].v[i];
          store_row<STREAM>(span[j], (T*)a.h + row * a.hs, y);
        }
        if (a.y) {
          normed(j, y);
          store_row<STREAM>(span[j], (T*)a.y + row * a.ys, y);
        }
      }
    }
    if (!a.q) continue;
    const float per_top = a.whole_numbers ? 1.0f / 127.0f : 1.0f / 448.0f;
    unsigned most[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      float y[V];
      normed(j, y);
      most[j] = 0;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (j < kSure<NT, NJ> || span[j].has(i)) most[j] = max(most[j], magnitude(y[i]));
    }
    if (a.group) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) most[j] = lanes_max(most[j], min(a.group / V, NT));
    } else {
      unsigned all = most[0];
#pragma unroll
      for (int j = 1; j < NJ; ++j) all = max(all, most[j]);
      all = lanes_max(all, NT < 64 ? NT : 64);
      if constexpr (NT > 64) {
        if (t % 64 == 0) most_of[g][t / 64] = all;
        __syncthreads();
        all = 0;
#pragma unroll
        for (int k = 0; k < NT / 64; ++k) all = max(all, most_of[g][k]);
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) most[j] = all;
    }
    if (!live) continue;
    uint8_t* out = a.q + row * a.qs;
    float* scales = a.scale + row * a.groups;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if (span[j].n == 0) continue;
      const float scale = scale_of(__builtin_bit_cast(float, most[j]), per_top);
      if (a.group ? span[j].from % a.group == 0 : t == 0 && j == 0) scales[a.group ? span[j].from / a.group : 0] = scale;
      float y[V];
      normed(j, y);
      divide<true>(y, scale);
      unsigned code[V / 4];
      to_codes(y, a.whole_numbers, code);
      // a piece that starts early has columns of another group: those are the piece's before it
      if (WHOLE || (span[j].n == V && span[j].c == span[j].from)) {
        __builtin_memcpy(out + span[j].c, code, V);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (span[j].has(i)) out[span[j].c + i] = (uint8_t)(code[i / 4] >> (8 * (i % 4)));
      }
    }
  }
}

// The same walk; a thread keeps its columns' share of dweight over all its rows, as layer norm's does.
template <typename T, int NT, int NJ, bool WHOLE, bool STREAM>
__global__ __launch_bounds__((NT * kRows<NT, true>)) void k_rms_bwd(RmsArgs a) {
  constexpr int V = kVec<T>, G = kRows<NT, true>;
  constexpr bool kAhead = kRunsAhead<NT, NJ>;
  __shared__ float scratch[2][G][kWaves<NT>];
  extern __shared__ __attribute__((aligned(16))) float columns[];   // [V/4][pieces][4] weight, then [cols] shares
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  using Piece = Span<V, WHOLE, !WHOLE && NT * NJ == 16>;
  Piece span[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) span[j] = Piece(t + j * NT, a.cols);
  Pack<T> x[NJ], dy[NJ], dres[NJ], next_x[NJ], next_dy[NJ], next_dres[NJ];
  float rstd, next_rstd;
  auto fetch = [&](int64_t row) {
    const int64_t at = row < a.rows ? row : 0;
    load_row<STREAM>(next_x, span, (const T*)a.x + at * a.xs);
    load_row<STREAM>(next_dy, span, (const T*)a.dy + at * a.dys);
    if (a.dres) load_row<STREAM>(next_dres, span, (const T*)a.dres + at * a.drs);
    next_rstd = a.rstd[at];
  };
  const int64_t step = (int64_t)gridDim.x * G, begin = (int64_t)blockIdx.x * G, end = a.rows;
  fetch(begin + g);
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const int pieces = (a.cols + V - 1) / V;
  f32x4* weight = (f32x4*)columns;
  for (int k = threadIdx.x; k < pieces; k += blockDim.x) {
    const Piece s(k, a.cols);
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
  float dw[NJ][V] = {};
  int turn = 0;
  for (int64_t first = begin; first < end; first += step, turn ^= 1) {
    const int64_t row = first + g;
    const bool live = row < end;
    rstd = next_rstd;
#pragma unroll
    for (int j = 0; j < NJ; ++j) x[j] = next_x[j], dy[j] = next_dy[j], dres[j] = next_dres[j];
    if constexpr (kAhead) fetch(row + step);
    float s = 0.0f;
    if (live) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float w[V];
        weight_of(j, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const bool has = j < kSure<NT, NJ> || span[j].has(i);
          const float xhat = has ? (float)x[j].v[i] * rstd : 0.0f, d = has ? (float)dy[j].v[i] : 0.0f;
          dw[j][i] = __builtin_fmaf(d, xhat, dw[j][i]);
          s = __builtin_fmaf(d * w[i], xhat, s);
        }
      }
    }
    if constexpr (!WHOLE) {   // two threads load the columns that two pieces share: both have, before dx may go there
      typedef int i32x4 __attribute__((ext_vector_type(4)));
      if (a.dres)
#pragma unroll
        for (int j = 0; j < NJ; ++j) asm volatile("" ::"v"(__builtin_bit_cast(i32x4, dres[j])));
    }
    const float c = sum_of_row<NT>(s, scratch[turn][g]) / (float)a.cols;
    if (live) {
      T* dx = (T*)a.dx + row * a.dxs;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (span[j].n == 0) continue;
        float w[V], out[V];
        weight_of(j, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float xhat = (float)x[j].v[i] * rstd;
          out[i] = __builtin_fmaf(-xhat, c, (float)dy[j].v[i] * w[i]) * rstd;
          if (a.dres) out[i] += (float)dres[j].v[i];
        }
        store_row<STREAM>(span[j], dx, out);
      }
    }
    if constexpr (!kAhead) fetch(row + step);
  }
  if (!a.dw) return;
  // the shares of the G rows' threads side by side, then added in order
  __syncthreads();
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (span[j].has(i)) columns[g * a.cols + span[j].c + i] = dw[j][i];
  __syncthreads();
  float* out = a.partial + (int64_t)blockIdx.x * share_stride(a.cols);
  for (int col = threadIdx.x; col < a.cols; col += blockDim.x) {
    float sum = columns[col];
#pragma unroll
    for (int k = 1; k < G; ++k) sum += columns[k * a.cols + col];
    if (gridDim.x > 1) out[col] = sum;
    else if (a.wide) ((float*)a.dw)[col] = sum;
    else ((T*)a.dw)[col] = (T)sum;
  }
}

// ---- host ---------------------------------------------------------------------------------

gbmw_status check_rms(const gbmw_rms_norm_problem* p) {
  if (!p) return fail(GBMW_ERR_INVALID_ARG, "null problem");
  if (!known_dtype(p->dtype)) return fail(GBMW_ERR_INVALID_ARG, "dtype=%d", p->dtype);
  if (p->wdtype != p->dtype && p->wdtype != GBMW_F32)
    return fail(GBMW_ERR_INVALID_ARG, "wdtype=%d is neither dtype nor GBMW_F32", p->wdtype);
  if (p->rows < 0 || p->rows > INT32_MAX) return fail(GBMW_ERR_INVALID_ARG, "rows=%lld", (long long)p->rows);
  if (p->cols < 1 || p->cols > 32768) return fail(GBMW_ERR_INVALID_ARG, "cols=%d not in 1..32768", p->cols);
  return GBMW_OK;
}

// As layer norm's, and: 16 threads where a row of up to 48 pieces fits them (not where a scale has columns of
// more threads than these), 128 where 256 would leave many without a piece, 512 between the rows of 256 and those of 1024.
// Backward 320 for 4097 to 5120 16-bit values, where they beat three pieces of 256 threads: up to 512 rows, which have a workgroup
// each (512 x 4608 12.9 us for 14.2, 4609 14.2 for 14.8, 5120 the same), and from 2048 rows on of whole pieces (16384
// x 4104 110 for 117, 4608 111 for 114, 5120 119 for 124; 2048 x 5120 25.9 for 26.8).  Not in between (1500 x 5120 24.9 for
// 22.7), nor where rows share pieces (16384 x 4609 153 for 140, 2048 x 5119 30.9 for 28.2); forward 117 for 112, 8192 x 2560
// in 32 bits 62 for 60.
Shape rms_shape(const gbmw_rms_norm_problem* p, bool backward) {
  const int vec = 16 / element_size(p->dtype), n = (p->cols + vec - 1) / vec;
  if (n <= 16 || (n <= 3 * 16 && (backward || !p->q || p->group <= 16 * vec))) return {16, (n + 15) / 16};
  if (n <= 3 * 64) return {64, (n + 63) / 64};
  if (n > 2 * 128 && n <= 3 * 128) return {128, 3};
  const bool few = p->rows <= 512, many_whole = p->rows >= 2048 && p->cols % vec == 0;
  if (backward && vec == 8 && n > 2 * 256 && n <= 2 * 320 && (few || many_whole)) return {320, 2};
  if (n <= 3 * 256) return {256, (n + 255) / 256};
  if (n <= 3 * 512) return {512, (n + 511) / 512};
  const int nj = (n + 1023) / 1024;
  return {1024, nj <= 4 ? nj : 8};
}

// Workgroups: forward one for every so many rows (many short ones keep memory busier than some that stay: 16384 x 5120
// 117 us, with 2048 that walk 129); backward so few that their shares of dweight cost little, one or two for a compute
// unit.  Two where rows are short enough that one leaves memory idle (16384 x 2560 76 us, with one 91; 65536 x 128 19 and
// 21) and there are rows for it (8192 x 1280, two turns of two or four of one: 27 and 24).
int rms_groups(const gbmw_rms_norm_problem* p, bool backward) {
  const Shape s = rms_shape(p, backward);
  const int64_t per = std::max(1, (backward ? kRmsBwdThreads : kRmsFwdThreads) / s.nt), all = (p->rows + per - 1) / per;
  if (!backward) return (int)std::min<int64_t>(all, 1 << 21);
  if (all <= 4) return all > 0;   // four turns take less than joining does (4 us and a launch)
  const int64_t most = s.nt == 1024 || s.nj == 3 || all < 4 * 512 ? 256 : 512;
  if (all <= most) return (int)all;
  const int64_t turns = (all + most - 1) / most;   // of the one that has most rows: no more workgroups than that takes
  return (int)((all + turns - 1) / turns);
}

// For the workgroups' shares of dweight; one writes it itself.
int64_t rms_workspace(const gbmw_rms_norm_problem* p, int groups) {
  return groups > 1 ? (int64_t)groups * share_stride(p->cols) * 4 : 0;
}

template <typename T, int NT, int NJ, bool WHOLE, bool STREAM>
gbmw_status launch_rms(const RmsArgs& a, bool backward, int groups, hipStream_t st) {
  if (!backward) {
    if constexpr (NT != 320)
      hipLaunchKernelGGL((k_rms_fwd<T, NT, NJ, WHOLE, STREAM>), dim3(groups), dim3(NT * kRows<NT, false>), 0, st, a);
  } else {
    const size_t weight = 16 * (size_t)((a.cols + kVec<T> - 1) / kVec<T>) * (kVec<T> / 4);
    const size_t lds = std::max(weight, 4 * (size_t)a.cols * kRows<NT, true>);
    if (lds > 60 * 1024) {
      const hipError_t e = hipFuncSetAttribute((const void*)&k_rms_bwd<T, NT, NJ, WHOLE, STREAM>,
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(GBMW_ERR_DEVICE, "%zu bytes of shared memory: %s", lds, hipGetErrorString(e));
      }
    }
    hipLaunchKernelGGL((k_rms_bwd<T, NT, NJ, WHOLE, STREAM>), dim3(groups), dim3(NT * kRows<NT, true>), lds, st, a);
  }
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

template <typename T, int NT, int NJ>
gbmw_status launch_rms(const RmsArgs& a, bool backward, int groups, hipStream_t st) {
  if (a.cols % kVec<T>) return launch_rms<T, NT, NJ, false, false>(a, backward, groups, st);
  return a.stream ? launch_rms<T, NT, NJ, true, true>(a, backward, groups, st) : launch_rms<T, NT, NJ, true, false>(a, backward, groups, st);
}

template <typename T>
gbmw_status launch_rms(const RmsArgs& a, Shape s, bool backward, int groups, hipStream_t st) {
  switch (s.nt * 10 + s.nj) {
    case 161: return launch_rms<T, 16, 1>(a, backward, groups, st);
    case 162: return launch_rms<T, 16, 2>(a, backward, groups, st);
    case 163: return launch_rms<T, 16, 3>(a, backward, groups, st);
    case 641: return launch_rms<T, 64, 1>(a, backward, groups, st);
    case 642: return launch_rms<T, 64, 2>(a, backward, groups, st);
    case 643: return launch_rms<T, 64, 3>(a, backward, groups, st);
    case 1283: return launch_rms<T, 128, 3>(a, backward, groups, st);
    case 2561: return launch_rms<T, 256, 1>(a, backward, groups, st);
    case 2562: return launch_rms<T, 256, 2>(a, backward, groups, st);
    case 2563: return launch_rms<T, 256, 3>(a, backward, groups, st);
    case 3202:
      if constexpr (sizeof(T) == 2) return launch_rms<T, 320, 2>(a, backward, groups, st);
      break;
    case 5122: return launch_rms<T, 512, 2>(a, backward, groups, st);
    case 5123: return launch_rms<T, 512, 3>(a, backward, groups, st);
    case 10242: return launch_rms<T, 1024, 2>(a, backward, groups, st);
    case 10243: return launch_rms<T, 1024, 3>(a, backward, groups, st);
    case 10244: return launch_rms<T, 1024, 4>(a, backward, groups, st);
    default: break;
  }
  if constexpr (sizeof(T) == 4) return launch_rms<T, 1024, 8>(a, backward, groups, st);
  return fail(GBMW_ERR_UNSUPPORTED, "no kernel for %d columns", a.cols);
}

gbmw_status launch_rms(const gbmw_rms_norm_problem* p, const RmsArgs& a, bool backward, int groups) {
  const Shape s = rms_shape(p, backward);
  hipStream_t st = (hipStream_t)p->stream;
  if (p->dtype == GBMW_F32) return launch_rms<float>(a, s, backward, groups, st);
  if (p->dtype == GBMW_F16) return launch_rms<f16>(a, s, backward, groups, st);
  return launch_rms<bf16>(a, s, backward, groups, st);
}

// Whether a call that moves `bytes` passes the cache by: where it would not hold the results for who reads them next.
// With a matrix product that reads them, 4096 x 5120 (168 MB) through the cache and past it: 116 and 120 us, 6144 (252 MB)
// 167 and 162, 16384 (671 MB) 421 and 413; backward 114 and 119, 166 and 158, 406 and 395.
bool past_cache(int64_t bytes) { return bytes >= 200000000; }

// An output that is one of its inputs has to have its rows at the same places.
gbmw_status check_place(const char* out, const void* o, int64_t os, const char* in, const void* i, int64_t is) {
  if (o && o == i && os != is) return fail(GBMW_ERR_INVALID_ARG, "%s is %s, with another row stride", out, in);
  return GBMW_OK;
}

}  // namespace
}  // namespace gbmw

using namespace gbmw;

extern "C" int64_t gbmw_rms_norm_workspace(const gbmw_rms_norm_problem* p) {
  gbmw_detail::clear_error();
  if (check_rms(p) != GBMW_OK) return -1;
  return rms_workspace(p, rms_groups(p, true));
}

extern "C" gbmw_status gbmw_rms_norm_forward(const gbmw_rms_norm_problem* p) {
  gbmw_detail::clear_error();
  CHECK(check_rms(p));
  if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return fail(GBMW_ERR_INVALID_ARG, "eps=%g", (double)p->eps);
  if (p->q) {
    if (p->qtype != GBMW_E4M3 && p->qtype != GBMW_I8) return fail(GBMW_ERR_INVALID_ARG, "qtype=%d", p->qtype);
    if (p->group != 0 && p->group != 32 && p->group != 64 && p->group != 128)
      return fail(GBMW_ERR_INVALID_ARG, "group=%d is none of 0, 32, 64, 128", p->group);
  }
  if (p->rows == 0) return GBMW_OK;
  const int size = element_size(p->dtype);
  CHECK(check_array("x", p->x, size, p->x_stride, 0));
  if (p->weight) CHECK(check_array("weight", p->weight, element_size(p->wdtype), 1, 0));
  if (p->rstd) CHECK(check_array("rstd", p->rstd, 4, 1, 0));
  if (p->residual) CHECK(check_array("residual", p->residual, size, p->residual_stride, 0));
  void* h = p->residual ? p->h : nullptr;
  if (h) CHECK(check_array("h", h, size, p->h_stride, p->cols));
  if (!p->y && !p->q) return fail(GBMW_ERR_INVALID_ARG, "neither y nor q is wanted");
  if (p->y) CHECK(check_array("y", p->y, size, p->y_stride, p->cols));
  if (p->q) {
    CHECK(check_array("q", p->q, 1, p->q_stride, p->cols));
    CHECK(check_array("scale", p->scale, 4, 1, 0));
  }
  CHECK(check_place("y", p->y, p->y_stride, "x", p->x, p->x_stride));
  CHECK(check_place("h", h, p->h_stride, "x", p->x, p->x_stride));
  if (p->residual) {
    CHECK(check_place("y", p->y, p->y_stride, "residual", p->residual, p->residual_stride));
    CHECK(check_place("h", h, p->h_stride, "residual", p->residual, p->residual_stride));
  }
  if (h && h == p->y) return fail(GBMW_ERR_INVALID_ARG, "h and y are one array");
  RmsArgs a{};
  a.rows = p->rows, a.cols = p->cols, a.eps = p->eps;
  a.x = p->x, a.res = p->residual, a.w = p->weight, a.wide = p->wdtype == GBMW_F32;
  a.h = h, a.y = p->y, a.q = (uint8_t*)p->q, a.rstd = p->rstd, a.scale = p->scale;
  a.xs = p->x_stride, a.rs = p->residual_stride, a.hs = p->h_stride, a.ys = p->y_stride, a.qs = p->q_stride;
  a.whole_numbers = p->qtype == GBMW_I8, a.group = p->q ? p->group : 0;
  a.groups = a.group ? (p->cols + a.group - 1) / a.group : 1;
  const int64_t n = p->rows * p->cols;
  a.stream = past_cache(n * size * (1 + (p->residual != nullptr) + (h != nullptr) + (p->y != nullptr)) + (p->q ? n : 0));
  return launch_rms(p, a, false, rms_groups(p, false));
}

extern "C" gbmw_status gbmw_rms_norm_backward(const gbmw_rms_norm_problem* p) {
  gbmw_detail::clear_error();
  CHECK(check_rms(p));
  const int size = element_size(p->dtype), wsize = element_size(p->wdtype);
  if (p->dweight) CHECK(check_array("dweight", p->dweight, wsize, 1, 0));
  const int groups = rms_groups(p, true);
  if (p->rows > 0) {
    CHECK(check_array("x", p->x, size, p->x_stride, 0));
    CHECK(check_array("dy", p->dy, size, p->dy_stride, 0));
    CHECK(check_array("dx", p->dx, size, p->dx_stride, p->cols));
    CHECK(check_array("rstd", p->rstd, 4, 1, 0));
    if (p->dres) CHECK(check_array("dres", p->dres, size, p->dres_stride, 0));
    if (p->weight) CHECK(check_array("weight", p->weight, wsize, 1, 0));
    CHECK(check_place("dx", p->dx, p->dx_stride, "dy", p->dy, p->dy_stride));
    CHECK(check_place("dx", p->dx, p->dx_stride, "dres", p->dres, p->dres_stride));
    const int64_t need = rms_workspace(p, groups);
    if (p->dweight && need && (!p->workspace || p->workspace_bytes < need || (uintptr_t)p->workspace % 16))
      return fail(GBMW_ERR_INVALID_ARG, "workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
    RmsArgs a{};
    a.rows = p->rows, a.cols = p->cols;
    a.x = p->x, a.dy = p->dy, a.dres = p->dres, a.w = p->weight, a.dx = p->dx, a.wide = p->wdtype == GBMW_F32;
    a.xs = p->x_stride, a.dys = p->dy_stride, a.drs = p->dres_stride, a.dxs = p->dx_stride, a.rstd = p->rstd;
    a.partial = (float*)p->workspace, a.dw = p->dweight;
    a.stream = past_cache(p->rows * p->cols * size * (p->dres ? 4 : 3));
    CHECK(launch_rms(p, a, true, groups));
  }
  if (p->dweight && groups != 1) {   // without rows: zeros
    const dim3 grid((p->cols + 31) / 32, 1);
    hipStream_t st = (hipStream_t)p->stream;
    const float* part = (const float*)p->workspace;
    if (p->wdtype == GBMW_F32)
      hipLaunchKernelGGL(k_norm_join<float>, grid, dim3(1024), 0, st, part, groups, p->cols, (float*)p->dweight,
                         (float*)nullptr);
    else if (p->wdtype == GBMW_F16)
      hipLaunchKernelGGL(k_norm_join<f16>, grid, dim3(1024), 0, st, part, groups, p->cols, (f16*)p->dweight, (f16*)nullptr);
    else
      hipLaunchKernelGGL(k_norm_join<bf16>, grid, dim3(1024), 0, st, part, groups, p->cols, (bf16*)p->dweight,
                         (bf16*)nullptr);
    HIP_TRY(hipGetLastError());
  }
  return GBMW_OK;
}
