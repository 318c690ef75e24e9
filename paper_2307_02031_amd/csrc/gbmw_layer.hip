// Layer norm (forward and backward) and gradient clipping: the memory-bound operators
// of a transformer layer's training.  Contracts: include/gbmw.h.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <vector>

#include "gbmw_ctx.h"
#include "gbmw_dtype.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

// ---- layer norm -------------------------------------------------------------------------
//
// NT threads share a row and keep it in registers, thread t the 16-byte pieces t, t + NT,
// ... (NJ of them), so the row is read once: the mean first, then the sum of the squared
// distances from it, which does not cancel where the mean is large.
//
// Bound by HBM; one pass over x (and dy) is its floor.

struct NormArgs {
  int64_t rows;
  int cols;
  float eps;
  const void *x, *dy, *w, *b;
  void *y, *dx;
  int64_t xs, ys, dys, dxs;
  float *mean, *rstd;
  float* partial;  // [gridDim.x][2][cols]
};

// Sums of N values over the NT threads of a row.  `scratch`: N * (NT / 64) floats of the
// row's own.  Every thread of the workgroup calls it.
template <int NT, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float* scratch) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
  if constexpr (NT > 64) {
    const int t = threadIdx.x % NT;
    __syncthreads();   // the last call's values are read
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

template <typename T, typename W, int NT, int NJ>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_norm_fwd(NormArgs a) {
  constexpr int V = kVec<T>, G = (NT < 256 ? 256 : NT) / NT;
  __shared__ float scratch[G][NT / 64];
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  const int64_t row = (int64_t)blockIdx.x * G + g;
  const bool live = row < a.rows;
  const T* x = (const T*)a.x + (live ? row : 0) * a.xs;
  Pack<T> px[NJ];
  float s[1] = {0.0f};
#pragma unroll
  for (int j = 0; j < NJ; ++j) px[j] = load_pack(x + (t + j * NT) * V, live ? a.cols - (t + j * NT) * V : 0);
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) s[0] += (float)px[j].v[i];
  row_sum<NT>(s, scratch[g]);
  const float mean = s[0] / (float)a.cols;
  s[0] = 0.0f;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = (t + j * NT) * V + i < a.cols ? (float)px[j].v[i] - mean : 0.0f;
      s[0] = __builtin_fmaf(d, d, s[0]);
    }
  row_sum<NT>(s, scratch[g]);
  const float rstd = 1.0f / __builtin_sqrtf(s[0] / (float)a.cols + a.eps);
  if (!live) return;
  if (t == 0) a.mean[row] = mean, a.rstd[row] = rstd;
  T* y = (T*)a.y + row * a.ys;
  const W *w = (const W*)a.w, *b = (const W*)a.b;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int c = (t + j * NT) * V, n = a.cols - c;
    if (n <= 0) break;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float xhat = ((float)px[j].v[i] - mean) * rstd;
      const float wi = w && i < n ? (float)w[c + i] : 1.0f, bi = b && i < n ? (float)b[c + i] : 0.0f;
      px[j].v[i] = (T)__builtin_fmaf(xhat, wi, bi);
    }
    store_pack(y + c, px[j], n);
  }
}

constexpr int kNormBwdThreads = 512;

// G rows at a time per workgroup, rows blockIdx.x * G + g, then gridDim.x * G further on.  A
// thread keeps its columns' share of dweight and dbias in registers over all its rows; the
// workgroup's shares go to `partial` and k_norm_join adds them up in a fixed order, so the
// result does not depend on which workgroup ends first.
template <typename T, typename W, int NT, int NJ>
__global__ __launch_bounds__(NT < kNormBwdThreads ? kNormBwdThreads : NT) void k_norm_bwd(NormArgs a) {
  constexpr int V = kVec<T>, G = (NT < kNormBwdThreads ? kNormBwdThreads : NT) / NT;
  __shared__ float scratch[G][2 * (NT / 64)];
  extern __shared__ float joined[];   // [cols], where dweight or dbias is wanted
  const int t = threadIdx.x % NT, g = threadIdx.x / NT;
  const W* w = (const W*)a.w;
  float dw[NJ][V] = {}, db[NJ][V] = {};
  for (int64_t first = (int64_t)blockIdx.x * G; first < a.rows; first += (int64_t)gridDim.x * G) {
    const int64_t row = first + g;
    const bool live = row < a.rows;
    const T *x = (const T*)a.x + (live ? row : 0) * a.xs, *dy = (const T*)a.dy + (live ? row : 0) * a.dys;
    Pack<T> px[NJ], pg[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (t + j * NT) * V, n = live ? a.cols - c : 0;
      px[j] = load_pack(x + c, n);
      pg[j] = load_pack(dy + c, n);
    }
    const float mean = live ? a.mean[row] : 0.0f, rstd = live ? a.rstd[row] : 0.0f;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (t + j * NT) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool in = c + i < a.cols;   // beyond the row dy is 0, and xhat must not be large
        const float xhat = in ? ((float)px[j].v[i] - mean) * rstd : 0.0f, d = (float)pg[j].v[i];
        const float wi = w && in ? (float)w[c + i] : 1.0f;
        dw[j][i] = __builtin_fmaf(d, xhat, dw[j][i]);
        db[j][i] += d;
        s[0] = __builtin_fmaf(d, wi, s[0]);
        s[1] = __builtin_fmaf(d * wi, xhat, s[1]);
      }
    }
    row_sum<NT>(s, scratch[g]);
    const float c1 = s[0] / (float)a.cols, c2 = s[1] / (float)a.cols;
    T* dx = (T*)a.dx + row * a.dxs;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (t + j * NT) * V, n = live ? a.cols - c : 0;
      if (n <= 0) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float xhat = ((float)px[j].v[i] - mean) * rstd;
        const float wi = w && i < n ? (float)w[c + i] : 1.0f;
        pg[j].v[i] = (T)(__builtin_fmaf(-xhat, c2, __builtin_fmaf((float)pg[j].v[i], wi, -c1)) * rstd);
      }
      store_pack(dx + c, pg[j], n);
    }
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
            const int c = (t + j * NT) * V + i;
            const float v = which ? db[j][i] : dw[j][i];
            if (c < a.cols) joined[c] = k ? joined[c] + v : v;
          }
    }
    __syncthreads();
    float* out = a.partial + ((int64_t)blockIdx.x * 2 + which) * a.cols;
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) out[c] = joined[c];
  }
}

// dweight and dbias from `parts` shares: 64 columns a workgroup, its 16 waves every 16th share.
template <typename W>
__global__ __launch_bounds__(1024) void k_norm_join(const float* partial, int parts, int cols, W* dw, W* db) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int c = blockIdx.x * 64 + lane;
  W* out = blockIdx.y ? db : dw;
  if (!out) return;
  float s = 0.0f;
  if (c < cols)
    for (int k = wave; k < parts; k += 16) s += partial[((int64_t)k * 2 + blockIdx.y) * cols + c];
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) {
    for (int k = 1; k < 16; ++k) s += sums[k][lane];
    out[c] = (W)s;
  }
}

// ---- gradient norm and clipping -----------------------------------------------------------

struct Piece {   // a run of at most kPiece elements of one tensor
  const void* in;
  void* out;
  int64_t n;
};
constexpr int64_t kPiece = 32768;
constexpr int kNormGroups = 2048;   // at most so many partial sums

struct Clip {   // device memory of a list, in front of the partial sums
  float factor;
  unsigned arrived;
};

template <typename T>
__global__ __launch_bounds__(256) void k_clip_norm(const Piece* pieces, int count, double* partial, Clip* clip,
                                                   double max_norm, double scale, float* norm_out) {
  __shared__ double sums[4];
  __shared__ bool last;
  constexpr int V = kVec<T>;
  double s = 0.0;
  for (int k = blockIdx.x; k < count; k += gridDim.x) {
    const Piece pc = pieces[k];
    const T* in = (const T*)pc.in;
    for (int i = threadIdx.x * V; i < pc.n; i += 256 * V) {
      const Pack<T> x = load_pack(in + i, (int)pc.n - i);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const double d = (double)(float)x.v[e];
        s = __builtin_fma(d, d, s);
      }
    }
  }
  s = wave_sum(s);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    partial[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    // the sum is visible to whoever sees the count
    last = __hip_atomic_fetch_add(&clip->arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  // the workgroup that ends last adds the partial sums, in an order of their own
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  s = 0.0;
  for (int k = threadIdx.x; k < (int)gridDim.x; k += 256) s += partial[k];
  s = wave_sum(s);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    const double norm = __builtin_sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) * scale;
    const bool clips = norm > max_norm && norm < __builtin_inf();
    clip->factor = (float)(clips ? scale * (max_norm / norm) : scale);
    clip->arrived = 0;   // for the next call
    if (norm_out) *norm_out = (float)norm;
  }
}

template <typename T, typename O>
__global__ __launch_bounds__(256) void k_clip_scale(const Piece* pieces, int count, const Clip* clip) {
  constexpr int V = kVec<T>;
  const float factor = clip->factor;
  for (int k = blockIdx.x; k < count; k += gridDim.x) {
    const Piece pc = pieces[k];
    if (factor == 1.0f && pc.in == pc.out) continue;   // the values are there
    const T* in = (const T*)pc.in;
    O* out = (O*)pc.out;
    for (int i = threadIdx.x * V; i < pc.n; i += 256 * V) {
      const int n = (int)pc.n - i;
      const Pack<T> x = load_pack(in + i, n);
      Pack<O> y;
#pragma unroll
      for (int h = 0; h < V; h += kVec<O>) {
#pragma unroll
        for (int e = 0; e < kVec<O>; ++e) y.v[e] = (O)((float)x.v[h + e] * factor);
        store_pack(out + i + h, y, n - h);
      }
    }
  }
}

// ---- host ---------------------------------------------------------------------------------

int element_size(int dtype) { return dtype == GBMW_F32 ? 4 : 2; }
bool known_dtype(int dtype) { return dtype == GBMW_F32 || dtype == GBMW_F16 || dtype == GBMW_BF16; }

gbmw_status check_norm(const gbmw_layer_norm_problem* p) {
  if (!p) return fail(GBMW_ERR_INVALID_ARG, "null problem");
  if (!known_dtype(p->dtype)) return fail(GBMW_ERR_INVALID_ARG, "dtype=%d", p->dtype);
  if (p->wdtype != p->dtype && p->wdtype != GBMW_F32)
    return fail(GBMW_ERR_INVALID_ARG, "wdtype=%d is neither dtype nor GBMW_F32", p->wdtype);
  if (p->rows < 0 || p->rows > INT32_MAX) return fail(GBMW_ERR_INVALID_ARG, "rows=%lld", (long long)p->rows);
  if (p->cols < 1 || p->cols > 32768) return fail(GBMW_ERR_INVALID_ARG, "cols=%d not in 1..32768", p->cols);
  return GBMW_OK;
}

// Threads of a row and 16-byte pieces of each: few threads for short rows, so that the sums
// stay inside a wave, and at most four pieces a thread, so that they stay in registers.
struct Shape {
  int nt, nj;
};
Shape shape_of(const gbmw_layer_norm_problem* p) {
  const int vec = 16 / element_size(p->dtype), n = (p->cols + vec - 1) / vec;
  if (n <= 4 * 64) return {64, (n + 63) / 64};
  if (n <= 4 * 256) return {256, (n + 255) / 256};
  const int nj = (n + 1023) / 1024;
  return {1024, nj <= 2 ? 2 : nj <= 4 ? 4 : 8};
}

int norm_groups(const gbmw_layer_norm_problem* p) {   // workgroups of the backward pass
  const Shape s = shape_of(p);
  const int per = std::max(1, kNormBwdThreads / s.nt);
  return (int)std::min<int64_t>(512, (p->rows + per - 1) / per);
}

template <typename T, typename W, int NT, int NJ>
gbmw_status launch_norm(const NormArgs& a, bool backward, int groups, hipStream_t st) {
  if (!backward) {
    constexpr int threads = NT < 256 ? 256 : NT;
    const int64_t grid = (a.rows + threads / NT - 1) / (threads / NT);
    hipLaunchKernelGGL((k_norm_fwd<T, W, NT, NJ>), dim3((unsigned)grid), dim3(threads), 0, st, a);
  } else {
    constexpr int threads = NT < kNormBwdThreads ? kNormBwdThreads : NT;
    const size_t lds = a.partial ? 4 * (size_t)a.cols : 0;
    if (lds > 60 * 1024) {
      const hipError_t e = hipFuncSetAttribute((const void*)&k_norm_bwd<T, W, NT, NJ>,
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(GBMW_ERR_DEVICE, "%zu bytes of shared memory: %s", lds, hipGetErrorString(e));
      }
    }
    hipLaunchKernelGGL((k_norm_bwd<T, W, NT, NJ>), dim3(groups), dim3(threads), lds, st, a);
  }
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

template <typename T, typename W>
gbmw_status launch_norm(const NormArgs& a, Shape s, bool backward, int groups, hipStream_t st) {
  if (s.nt == 64) switch (s.nj) {
    case 1: return launch_norm<T, W, 64, 1>(a, backward, groups, st);
    case 2: return launch_norm<T, W, 64, 2>(a, backward, groups, st);
    case 3: return launch_norm<T, W, 64, 3>(a, backward, groups, st);
    default: return launch_norm<T, W, 64, 4>(a, backward, groups, st);
  }
  if (s.nt == 256) switch (s.nj) {
    case 2: return launch_norm<T, W, 256, 2>(a, backward, groups, st);
    case 3: return launch_norm<T, W, 256, 3>(a, backward, groups, st);
    default: return launch_norm<T, W, 256, 4>(a, backward, groups, st);
  }
  if (s.nj == 2) return launch_norm<T, W, 1024, 2>(a, backward, groups, st);
  if (s.nj == 4) return launch_norm<T, W, 1024, 4>(a, backward, groups, st);
  if constexpr (sizeof(T) == 4) return launch_norm<T, W, 1024, 8>(a, backward, groups, st);
  return fail(GBMW_ERR_UNSUPPORTED, "no kernel for %d columns", a.cols);
}

gbmw_status launch_norm(const gbmw_layer_norm_problem* p, const NormArgs& a, bool backward, int groups) {
  const Shape s = shape_of(p);
  hipStream_t st = (hipStream_t)p->stream;
  const bool same = p->wdtype == p->dtype;
  if (p->dtype == GBMW_F32) return launch_norm<float, float>(a, s, backward, groups, st);
  if (p->dtype == GBMW_F16)
    return same ? launch_norm<f16, f16>(a, s, backward, groups, st) : launch_norm<f16, float>(a, s, backward, groups, st);
  return same ? launch_norm<bf16, bf16>(a, s, backward, groups, st)
              : launch_norm<bf16, float>(a, s, backward, groups, st);
}

gbmw_status check_array(const char* name, const void* ptr, int size, int64_t stride, int64_t least) {
  if (!ptr) return fail(GBMW_ERR_INVALID_ARG, "%s is null", name);
  if ((uintptr_t)ptr % (unsigned)size) return fail(GBMW_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
  if (stride < least || stride > (INT64_MAX >> 34))
    return fail(GBMW_ERR_INVALID_ARG, "%s: row stride %lld", name, (long long)stride);
  return GBMW_OK;
}

}  // namespace
}  // namespace gbmw

using namespace gbmw;

#define CHECK(expr)                            \
  do {                                         \
    const gbmw_status st_ = (expr);            \
    if (st_ != GBMW_OK) return st_;            \
  } while (0)

extern "C" int64_t gbmw_layer_norm_workspace(const gbmw_layer_norm_problem* p) {
  gbmw_detail::clear_error();
  if (check_norm(p) != GBMW_OK) return -1;
  return (int64_t)norm_groups(p) * 2 * p->cols * 4;
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
  a.x = p->x, a.w = p->weight, a.b = p->bias, a.y = p->y;
  a.xs = p->x_stride, a.ys = p->y_stride, a.mean = p->mean, a.rstd = p->rstd;
  return launch_norm(p, a, false, 0);
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
  const int groups = norm_groups(p);
  if (wanted && p->rows > 0) {
    const int64_t need = (int64_t)groups * 2 * p->cols * 4;
    if (!p->workspace || p->workspace_bytes < need || (uintptr_t)p->workspace % 16)
      return fail(GBMW_ERR_INVALID_ARG, "workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
  }
  if (p->rows > 0) {
    NormArgs a{};
    a.rows = p->rows, a.cols = p->cols;
    a.x = p->x, a.dy = p->dy, a.w = p->weight, a.dx = p->dx;
    a.xs = p->x_stride, a.dys = p->dy_stride, a.dxs = p->dx_stride, a.mean = p->mean, a.rstd = p->rstd;
    a.partial = wanted ? (float*)p->workspace : nullptr;
    CHECK(launch_norm(p, a, true, groups));
  }
  if (wanted) {   // without rows: zeros
    const dim3 grid((p->cols + 63) / 64, 2);
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
  gbmw_detail::DevBuf buf;   // Clip (padded to 256 bytes) | partial sums | pieces
  int count = 0, in_dtype = 0, out_dtype = 0, device = 0;
  Clip* clip() const { return (Clip*)buf.p; }
  double* partial() const { return (double*)((char*)buf.p + 256); }
  Piece* pieces() const { return (Piece*)((char*)buf.p + 256 + 8 * kNormGroups); }
};

extern "C" gbmw_status gbmw_gradient_list_create(int32_t n, const void* const* in, void* const* out,
                                                 const int64_t* numel, int32_t in_dtype, int32_t out_dtype,
                                                 gbmw_gradient_list** list) {
  gbmw_detail::clear_error();
  if (!list) return fail(GBMW_ERR_INVALID_ARG, "null list");
  *list = nullptr;
  if (n < 0 || (n > 0 && (!in || !out || !numel))) return fail(GBMW_ERR_INVALID_ARG, "n=%d, or a null array", n);
  if (!known_dtype(in_dtype)) return fail(GBMW_ERR_INVALID_ARG, "in_dtype=%d", in_dtype);
  if (out_dtype != in_dtype && out_dtype != GBMW_F32)
    return fail(GBMW_ERR_INVALID_ARG, "out_dtype=%d is neither in_dtype nor GBMW_F32", out_dtype);
  const int isize = element_size(in_dtype), osize = element_size(out_dtype);
  int64_t count = 0;
  for (int i = 0; i < n; ++i) {
    if (numel[i] < 0 || numel[i] > (1ll << 44)) return fail(GBMW_ERR_INVALID_ARG, "numel[%d]=%lld", i, (long long)numel[i]);
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
        pieces.push_back({(const char*)in[i] + at * isize, (char*)out[i] + at * osize, std::min(kPiece, numel[i] - at)});
    gbmw_gradient_list* l = new gbmw_gradient_list;
    l->count = (int)count, l->in_dtype = in_dtype, l->out_dtype = out_dtype;
    const size_t head = 256 + 8 * kNormGroups;
    gbmw_status st = l->buf.reserve(head + sizeof(Piece) * (size_t)count);
    if (st == GBMW_OK) {
      hipError_t e = hipGetDevice(&l->device);
      const Clip zero{1.0f, 0u};
      if (e == hipSuccess) e = hipMemcpy(l->clip(), &zero, sizeof zero, hipMemcpyHostToDevice);
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
#define NORM(T) \
  hipLaunchKernelGGL(k_clip_norm<T>, grid, block, 0, st, l->pieces(), l->count, l->partial(), l->clip(), (double)max_norm, \
                     (double)scale, norm)
#define SCALE(T, O) hipLaunchKernelGGL((k_clip_scale<T, O>), grid, block, 0, st, l->pieces(), l->count, l->clip())
  if (l->in_dtype == GBMW_F32) NORM(float);
  else if (l->in_dtype == GBMW_F16) NORM(f16);
  else NORM(bf16);
  HIP_TRY(hipGetLastError());
  if (l->count) {
    if (l->in_dtype == GBMW_F32) SCALE(float, float);
    else if (l->in_dtype == GBMW_F16 && l->out_dtype == GBMW_F16) SCALE(f16, f16);
    else if (l->in_dtype == GBMW_F16) SCALE(f16, float);
    else if (l->out_dtype == GBMW_BF16) SCALE(bf16, bf16);
    else SCALE(bf16, float);
    HIP_TRY(hipGetLastError());
  }
#undef NORM
#undef SCALE
  return GBMW_OK;
}

extern "C" void gbmw_gradient_list_destroy(gbmw_gradient_list* l) {
  if (!l) return;
  (void)hipDeviceSynchronize();
  l->buf.release();
  delete l;
}
