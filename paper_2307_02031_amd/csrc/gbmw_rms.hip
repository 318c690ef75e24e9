// RMS norm after a residual's addition, to the arrays' type or to 8 bits with scales, and its
// backward pass.  Contract: include/gbmw.h.
#include "gbmw_rows.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

// NT threads hold a row in registers, as in layer norm: one pass over x and the residual, and one sum.
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
  float* partial;  // [gridDim.x][share_stride(cols)]
};

constexpr int kRmsFwdThreads = 256, kRmsBwdThreads = 512;

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

// V values in 8 bits, four in a word.
template <int V>
__device__ __forceinline__ void to_codes(const float (&x)[V], float by, bool whole_numbers, unsigned (&code)[V / 4]) {
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    if (whole_numbers) {
      code[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = (int)__builtin_fminf(__builtin_fmaxf(__builtin_rintf(x[4 * i + e] * by), -127.0f), 127.0f);
        code[i] |= (unsigned)(n & 255) << (8 * e);
      }
    } else {
      int word = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * by, x[4 * i + 1] * by, 0, false);
      code[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * by, x[4 * i + 3] * by, word, true);
    }
  }
}

template <typename T, int NT, int NJ, bool WHOLE>
__global__ __launch_bounds__(NT < kRmsFwdThreads ? kRmsFwdThreads : NT) void k_rms_fwd(RmsArgs a) {
  constexpr int V = kVec<T>, G = (NT < kRmsFwdThreads ? kRmsFwdThreads : NT) / NT;
  constexpr bool kAhead = kRunsAhead<NT, NJ>;
  __shared__ float scratch[2][G][NT / 64];
  __shared__ unsigned most_of[G][NT / 64];
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  constexpr bool kTiny = !WHOLE && NT * NJ == 64;
  Span<V, WHOLE, kTiny> span[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) span[j] = Span<V, WHOLE, kTiny>(t + j * NT, a.cols);
  Held<T, NJ, kTiny> h, r, next, next_r;
  auto fetch = [&](int64_t row) {
    const int64_t at = row < a.rows ? row : 0;
    next.load(span, (const T*)a.x + at * a.xs, a.cols);
    if (a.res) next_r.load(span, (const T*)a.res + at * a.rs, a.cols);
  };
  const int64_t step = (int64_t)gridDim.x * G;
  fetch((int64_t)blockIdx.x * G + g);
  float w[NJ][V];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[j][i] = 1.0f;
    if (a.w) a.wide ? span[j].load(w[j], (const float*)a.w) : span[j].load(w[j], (const T*)a.w);
  }
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.rows; first += step, turn ^= 1) {
    const int64_t row = first + g;
    h = next;
    if (a.res) r = next_r;
    if constexpr (kAhead) fetch(row + step);
    if (a.res) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) h.p[j].v[i] = (T)((float)h.p[j].v[i] + (float)r.p[j].v[i]);
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = j < kSure<NT, NJ> || span[j].has(i) ? (float)h.p[j].v[i] : 0.0f;
        s[0] = __builtin_fmaf(d, d, s[0]);
      }
    // stores come after the sum, which has every thread's values of the row: it may be written in place
    row_sum<NT>(s, scratch[turn][g]);
    const float rstd = 1.0f / __builtin_sqrtf(s[0] / (float)a.cols + a.eps);
    const bool live = row < a.rows;
    auto normed = [&](int j, float (&y)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = (float)h.p[j].v[i] * rstd * w[j][i];
    };
    if (live) {
      if (t == 0 && a.rstd) a.rstd[row] = rstd;
      if (a.h) {
        T* out = (T*)a.h + row * a.hs;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (span[j].n == 0) continue;
          float v[V];
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = (float)h.p[j].v[i];
          span[j].store(out, v);
        }
      }
      if (a.y) {
        T* out = (T*)a.y + row * a.ys;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (span[j].n == 0) continue;
          float y[V];
          normed(j, y);
          span[j].store(out, y);
        }
      }
    }
    if (a.q) {
      const float top = a.whole_numbers ? 127.0f : 448.0f;
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
        for (int j = 0; j < NJ; ++j) most[j] = lanes_max(most[j], a.group / V);
      } else {
        unsigned all = most[0];
#pragma unroll
        for (int j = 1; j < NJ; ++j) all = max(all, most[j]);
        all = lanes_max(all, 64);
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
      if (live) {
        uint8_t* out = a.q + row * a.qs;
        float* scales = a.scale + row * a.groups;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (span[j].n == 0) continue;
          const float most_f = __builtin_bit_cast(float, most[j]) / top;
          const float scale = most_f < 0x1p-126f ? 0x1p-126f : most_f, by = 1.0f / scale;
          if (a.group ? span[j].from % a.group == 0 : t == 0 && j == 0)
            scales[a.group ? span[j].from / a.group : 0] = scale;
          float y[V];
          normed(j, y);
          unsigned code[V / 4];
          to_codes(y, by, a.whole_numbers, code);
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
    if constexpr (!kAhead) fetch(row + step);
  }
}

// The same walk; a thread keeps its columns' share of dweight over all its rows, as layer norm's does.
template <typename T, int NT, int NJ, bool WHOLE>
__global__ __launch_bounds__(NT < kRmsBwdThreads ? kRmsBwdThreads : NT) void k_rms_bwd(RmsArgs a) {
  constexpr int V = kVec<T>, G = (NT < kRmsBwdThreads ? kRmsBwdThreads : NT) / NT;
  constexpr bool kAhead = kRunsAhead<NT, NJ>;
  __shared__ float scratch[2][G][NT / 64];
  extern __shared__ __attribute__((aligned(16))) float columns[];   // [V/4][pieces][4] weight, then [cols] shares
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  constexpr bool kTiny = !WHOLE && NT * NJ == 64;
  Span<V, WHOLE, kTiny> span[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) span[j] = Span<V, WHOLE, kTiny>(t + j * NT, a.cols);
  Held<T, NJ, kTiny> x, dy, next_x, next_dy, dres, next_dres;
  float rstd, next_rstd;
  auto fetch = [&](int64_t row) {
    const int64_t at = row < a.rows ? row : 0;
    next_x.load(span, (const T*)a.x + at * a.xs, a.cols);
    next_dy.load(span, (const T*)a.dy + at * a.dys, a.cols);
    if (a.dres) next_dres.load(span, (const T*)a.dres + at * a.drs, a.cols);
    next_rstd = a.rstd[at];
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
  float dw[NJ][V] = {};
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.rows; first += step, turn ^= 1) {
    const int64_t row = first + g;
    const bool live = row < a.rows;
    x = next_x, dy = next_dy, rstd = next_rstd;
    if (a.dres) dres = next_dres;
    if constexpr (kAhead) fetch(row + step);
    float s[1] = {0.0f};
    if (live) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float w[V];
        weight_of(j, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const bool has = j < kSure<NT, NJ> || span[j].has(i);
          const float xhat = has ? (float)x.p[j].v[i] * rstd : 0.0f, d = has ? (float)dy.p[j].v[i] : 0.0f;
          dw[j][i] = __builtin_fmaf(d, xhat, dw[j][i]);
          s[0] = __builtin_fmaf(d * w[i], xhat, s[0]);
        }
      }
    }
    if constexpr (!WHOLE) {   // two threads load the columns that two pieces share: both have, before dx may go there
      typedef int i32x4 __attribute__((ext_vector_type(4)));
      if (a.dres)
#pragma unroll
        for (int j = 0; j < NJ; ++j) asm volatile("" ::"v"(__builtin_bit_cast(i32x4, dres.p[j])));
    }
    row_sum<NT>(s, scratch[turn][g]);
    const float c = s[0] / (float)a.cols;
    if (live) {
      T* dx = (T*)a.dx + row * a.dxs;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (span[j].n == 0) continue;
        float w[V], out[V];
        weight_of(j, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float xhat = (float)x.p[j].v[i] * rstd;
          out[i] = __builtin_fmaf(-xhat, c, (float)dy.p[j].v[i] * w[i]) * rstd;
          if (a.dres) out[i] += (float)dres.p[j].v[i];
        }
        span[j].store(dx, out);
      }
    }
    if constexpr (!kAhead) fetch(row + step);
  }
  if (!a.partial) return;
  for (int k = 0; k < G; ++k) {   // one row's threads after the other add their share
    __syncthreads();
    if (g == k)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int col = span[j].c + i;
          if (span[j].has(i)) columns[col] = k ? columns[col] + dw[j][i] : dw[j][i];
        }
  }
  __syncthreads();
  float* out = a.partial + (int64_t)blockIdx.x * share_stride(a.cols);
  for (int col = threadIdx.x; col < a.cols; col += blockDim.x) out[col] = columns[col];
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

int rms_groups(const gbmw_rms_norm_problem* p, bool backward) {
  const Shape s = shape_of(p->dtype, p->cols);
  const int per = std::max(1, (backward ? kRmsBwdThreads : kRmsFwdThreads) / s.nt);
  const int64_t most = !backward ? s.nt < 1024 ? 2048 : s.nj == 1 ? 512 : 256 : s.nt == 1024 ? 256 : 512;
  const int64_t all = (p->rows + per - 1) / per;
  if (all <= most) return (int)all;
  const int64_t turns = (all + most - 1) / most;
  return (int)((all + turns - 1) / turns);
}

template <typename T, int NT, int NJ, bool WHOLE>
gbmw_status launch_rms(const RmsArgs& a, bool backward, int groups, hipStream_t st) {
  if (!backward) {
    hipLaunchKernelGGL((k_rms_fwd<T, NT, NJ, WHOLE>), dim3(groups), dim3(std::max(NT, kRmsFwdThreads)), 0, st, a);
  } else {
    const size_t lds = 16 * (size_t)((a.cols + kVec<T> - 1) / kVec<T>) * (kVec<T> / 4);
    if (lds > 60 * 1024) {
      const hipError_t e = hipFuncSetAttribute((const void*)&k_rms_bwd<T, NT, NJ, WHOLE>,
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(GBMW_ERR_DEVICE, "%zu bytes of shared memory: %s", lds, hipGetErrorString(e));
      }
    }
    hipLaunchKernelGGL((k_rms_bwd<T, NT, NJ, WHOLE>), dim3(groups), dim3(std::max(NT, kRmsBwdThreads)), lds, st, a);
  }
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

template <typename T, int NT, int NJ>
gbmw_status launch_rms(const RmsArgs& a, bool backward, int groups, hipStream_t st) {
  return a.cols % kVec<T> ? launch_rms<T, NT, NJ, false>(a, backward, groups, st)
                          : launch_rms<T, NT, NJ, true>(a, backward, groups, st);
}

template <typename T>
gbmw_status launch_rms(const RmsArgs& a, Shape s, bool backward, int groups, hipStream_t st) {
  if (s.nt == 64) switch (s.nj) {
    case 1: return launch_rms<T, 64, 1>(a, backward, groups, st);
    case 2: return launch_rms<T, 64, 2>(a, backward, groups, st);
    default: return launch_rms<T, 64, 3>(a, backward, groups, st);
  }
  if (s.nt == 256) switch (s.nj) {
    case 1: return launch_rms<T, 256, 1>(a, backward, groups, st);
    case 2: return launch_rms<T, 256, 2>(a, backward, groups, st);
    default: return launch_rms<T, 256, 3>(a, backward, groups, st);
  }
  if (s.nj == 1) return launch_rms<T, 1024, 1>(a, backward, groups, st);
  if (s.nj == 2) return launch_rms<T, 1024, 2>(a, backward, groups, st);
  if (s.nj == 4) return launch_rms<T, 1024, 4>(a, backward, groups, st);
  if constexpr (sizeof(T) == 4) return launch_rms<T, 1024, 8>(a, backward, groups, st);
  return fail(GBMW_ERR_UNSUPPORTED, "no kernel for %d columns", a.cols);
}

gbmw_status launch_rms(const gbmw_rms_norm_problem* p, const RmsArgs& a, bool backward, int groups) {
  const Shape s = shape_of(p->dtype, p->cols);
  hipStream_t st = (hipStream_t)p->stream;
  if (p->dtype == GBMW_F32) return launch_rms<float>(a, s, backward, groups, st);
  if (p->dtype == GBMW_F16) return launch_rms<f16>(a, s, backward, groups, st);
  return launch_rms<bf16>(a, s, backward, groups, st);
}

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
  return (int64_t)rms_groups(p, true) * share_stride(p->cols) * 4;
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
    const int64_t need = (int64_t)groups * share_stride(p->cols) * 4;
    if (p->dweight && (!p->workspace || p->workspace_bytes < need || (uintptr_t)p->workspace % 16))
      return fail(GBMW_ERR_INVALID_ARG, "workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
    RmsArgs a{};
    a.rows = p->rows, a.cols = p->cols;
    a.x = p->x, a.dy = p->dy, a.dres = p->dres, a.w = p->weight, a.dx = p->dx, a.wide = p->wdtype == GBMW_F32;
    a.xs = p->x_stride, a.dys = p->dy_stride, a.drs = p->dres_stride, a.dxs = p->dx_stride, a.rstd = p->rstd;
    a.partial = p->dweight ? (float*)p->workspace : nullptr;
    CHECK(launch_rms(p, a, true, groups));
  }
  if (p->dweight) {   // without rows: zeros
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
