// One AdamW step over many tensors, with states in 32 bits or in 8.  Contract: include/gbmw.h.
#include <new>
#include <vector>

#include "gbmw_rows.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

constexpr int kBlock = 256;        // elements that share a scale
constexpr int64_t kRun = 16384;    // at most so many elements of one tensor are a run
constexpr int kMostGroups = 2048;

struct Run {
  const void* grad;
  void *param, *copy, *m, *v;
  float *m_scale, *v_scale;
  int32_t n;
  uint32_t block;   // number of the run's first block in the list
  int32_t grad_dtype, dtype, copy_dtype;
  float decay;
};

struct AdamArgs {
  double lr, beta1, beta2, scale, max_norm;
  float eps;
  int64_t step;
  uint32_t seed;
  const float *norm, *lr_now;
  const int64_t* step_now;
};

// The numbers that all elements share: computed in fp64, rounded once.
struct Rates {
  float grad, b1, a1, b2, a2, eps, lr_c1, root_c2;
  double lr;
  uint32_t key;   // of the random numbers; 0: round to nearest
  bool skip;
};

__device__ __forceinline__ uint32_t hash(uint32_t x) {
  x *= 0x9E3779B1u;
  x = (x ^ (x >> 15)) * 0x85EBCA77u;
  return x ^ (x >> 13);
}

__device__ __forceinline__ Rates rates_of(const AdamArgs& a) {
  Rates r;
  double factor = a.scale;
  r.skip = false;
  if (a.norm) {
    const double norm = (double)*a.norm;
    r.skip = !(norm < __builtin_inf());   // a NaN too
    if (norm > a.max_norm) factor *= a.max_norm / norm;
  }
  r.lr = a.lr_now ? (double)*a.lr_now : a.lr;
  int64_t step = a.step_now ? *a.step_now : a.step;
  if (step < 1) step = 1;
  double p1 = 1.0, p2 = 1.0, q1 = a.beta1, q2 = a.beta2;   // beta^step by squares
  for (int64_t k = step; k; k >>= 1) {
    if (k & 1) p1 *= q1, p2 *= q2;
    q1 *= q1, q2 *= q2;
  }
  r.grad = (float)factor;
  r.b1 = (float)a.beta1, r.a1 = (float)(1.0 - a.beta1);
  r.b2 = (float)a.beta2, r.a2 = (float)(1.0 - a.beta2);
  r.eps = a.eps;
  r.lr_c1 = (float)(r.lr / (1.0 - p1));
  r.root_c2 = (float)(1.0 / __builtin_sqrt(1.0 - p2));
  r.key = a.seed ? hash(a.seed + (uint32_t)step * 0x9E3779B9u) : 0;
  return r;
}

// One element's step: m, the second moment before its root is taken, and the parameter.
__device__ __forceinline__ void step_of(const Rates& r, float keep, float g, float& m, float& v, float& root, float& p) {
  g *= r.grad;
  m = m * r.b1 + g * r.a1;
  v = v * r.b2 + g * g * r.a2;
  root = __builtin_sqrtf(v);
  p = p * keep - m / (root * r.root_c2 + r.eps) * r.lr_c1;
}

template <typename G, typename P>
__device__ __forceinline__ void copy_out(const Run& run, int i, int n, const float (&p)[4]) {
  if (!run.copy) return;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) {
      if (run.copy_dtype == GBMW_F16) ((f16*)run.copy)[i + e] = (f16)p[e];
      else ((bf16*)run.copy)[i + e] = (bf16)p[e];
    }
}

template <typename G, typename P>
__device__ __forceinline__ void run_of_32(const Run& run, const Rates& r) {
  const float keep = (float)(1.0 - r.lr * (double)run.decay);
  for (int i = threadIdx.x * 4; i < run.n; i += 256 * 4) {
    const int n = min(4, run.n - i);
    float p[4], m[4], v[4], g[4], root;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = i + min(e, n - 1);
      p[e] = (float)((const P*)run.param)[at], g[e] = (float)((const G*)run.grad)[at];
      m[e] = ((const float*)run.m)[at], v[e] = ((const float*)run.v)[at];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) step_of(r, keep, g[e], m[e], v[e], root, p[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) ((P*)run.param)[i + e] = (P)p[e], ((float*)run.m)[i + e] = m[e], ((float*)run.v)[i + e] = v[e];
    copy_out<G, P>(run, i, n, p);
  }
}

__device__ __forceinline__ unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }   // a NaN's is the largest

__device__ __forceinline__ float wave_most(unsigned u) {
#pragma unroll
  for (int d = 32; d; d >>= 1) u = max(u, (unsigned)__shfl_xor((int)u, d));
  return __builtin_bit_cast(float, u);
}

// x / scale as one of the 8-bit values beside it: up where the part cut off and `random`, of [0, 1), make a whole step.
__device__ __forceinline__ float at_random(float x, float random) {
  const float size = __builtin_fminf(__builtin_fabsf(x), 448.0f);
  const int exponent = max((int)(__builtin_bit_cast(unsigned, size) >> 23) - 127, -6);
  return __builtin_copysignf(__builtin_ldexpf(__builtin_floorf(__builtin_ldexpf(size, 3 - exponent) + random), exponent - 3), x);
}

__device__ __forceinline__ float scale_of(float most) {
  const float s = most / 448.0f;
  return s < 0x1p-126f ? 0x1p-126f : s;
}

__device__ __forceinline__ float value_of(uint8_t code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }
__device__ __forceinline__ uint8_t code_of(float x) { return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false); }

// A wave has a block of 256.
template <typename G, typename P>
__device__ __forceinline__ void run_of_8(const Run& run, const Rates& r) {
  const float keep = (float)(1.0 - r.lr * (double)run.decay);
  const int lane = threadIdx.x % 64;
  for (int k = threadIdx.x / 64; k * kBlock < run.n; k += 4) {
    const int i = k * kBlock + lane * 4, n = min(4, run.n - i);   // 0 or less behind the last element
    const float ms = run.m_scale[k], vs = run.v_scale[k];
    float p[4], m[4], v, g, root[4];
    unsigned most_m = 0, most_v = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      m[e] = root[e] = 0.0f;
      if (e >= n) continue;
      p[e] = (float)((const P*)run.param)[i + e], g = (float)((const G*)run.grad)[i + e];
      m[e] = value_of(((const uint8_t*)run.m)[i + e]) * ms;
      v = value_of(((const uint8_t*)run.v)[i + e]) * vs;
      v *= v;
      step_of(r, keep, g, m[e], v, root[e], p[e]);
      most_m = max(most_m, magnitude(m[e])), most_v = max(most_v, magnitude(root[e]));
    }
    const float new_ms = scale_of(wave_most(most_m)), new_vs = scale_of(wave_most(most_v));
    if (lane == 0) run.m_scale[k] = new_ms, run.v_scale[k] = new_vs;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e >= n) continue;
      float cm = m[e] / new_ms, cv = root[e] / new_vs;
      if (root[e] > 0.0f && cv < 0x1p-9f) cv = 0x1p-9f;
      if (r.key) {
        const uint32_t word = hash(((run.block + k) * kBlock + lane * 4 + e) ^ r.key);
        cm = at_random(cm, ((float)(word >> 16) + 0.5f) * 0x1p-16f);
        cv = at_random(cv, ((float)(word & 65535) + 0.5f) * 0x1p-16f);
      }
      ((uint8_t*)run.m)[i + e] = code_of(cm), ((uint8_t*)run.v)[i + e] = code_of(cv);
      ((P*)run.param)[i + e] = (P)p[e];
    }
    copy_out<G, P>(run, i, n, p);
  }
}

template <bool BITS8, typename G, typename P>
__device__ __forceinline__ void run_of(const Run& run, const Rates& r) {
  if constexpr (BITS8) run_of_8<G, P>(run, r);
  else run_of_32<G, P>(run, r);
}

template <bool BITS8, typename G>
__device__ __forceinline__ void run_of(const Run& run, const Rates& r) {
  if (run.dtype == GBMW_F32) run_of<BITS8, G, float>(run, r);
  else if (run.dtype == GBMW_F16) run_of<BITS8, G, f16>(run, r);
  else run_of<BITS8, G, bf16>(run, r);
}

template <bool BITS8>
__global__ __launch_bounds__(256) void k_adamw(const Run* runs, int count, AdamArgs a) {
  const Rates r = rates_of(a);
  if (r.skip) return;
  for (int k = blockIdx.x; k < count; k += gridDim.x) {
    const Run run = runs[k];
    if (run.grad_dtype == GBMW_F32) run_of<BITS8, float>(run, r);
    else if (run.grad_dtype == GBMW_F16) run_of<BITS8, f16>(run, r);
    else run_of<BITS8, bf16>(run, r);
  }
}

// ---- host ---------------------------------------------------------------------------------

struct Extent {
  uintptr_t begin, end;
  bool written;
  int tensor;
};

// The tensor with an array of which something is written that lies in another array too; -1 if there is none.
int overlap(std::vector<Extent>& all) {
  std::sort(all.begin(), all.end(), [](const Extent& x, const Extent& y) { return x.begin < y.begin; });
  uintptr_t any = 0, written = 0;   // ends of what came before
  for (const Extent& x : all) {
    if (x.begin < (x.written ? any : written)) return x.tensor;
    any = std::max(any, x.end);
    if (x.written) written = std::max(written, x.end);
  }
  return -1;
}

gbmw_status check_adamw(int i, const gbmw_adamw_tensor& t, int bits, std::vector<Extent>& all) {
  if (!known_dtype(t.grad_dtype)) return fail(GBMW_ERR_INVALID_ARG, "grad_dtype of tensor %d is %d", i, t.grad_dtype);
  if (!known_dtype(t.dtype)) return fail(GBMW_ERR_INVALID_ARG, "dtype of tensor %d is %d", i, t.dtype);
  if (t.numel < 0 || t.numel > (1ll << 41)) return fail(GBMW_ERR_INVALID_ARG, "numel of tensor %d is %lld", i, (long long)t.numel);
  if (!(t.weight_decay >= 0.0f) || !std::isfinite(t.weight_decay))
    return fail(GBMW_ERR_INVALID_ARG, "weight_decay of tensor %d is %g", i, (double)t.weight_decay);
  if (t.copy && (t.dtype != GBMW_F32 || (t.copy_dtype != GBMW_F16 && t.copy_dtype != GBMW_BF16)))
    return fail(GBMW_ERR_INVALID_ARG, "tensor %d: a copy is of 16 bits and of a parameter of 32", i);
  if (t.numel == 0) return GBMW_OK;
  const int64_t blocks = (t.numel + kBlock - 1) / kBlock;
  const int state = bits == 8 ? 1 : 4;
  const struct {
    const char* name;
    const void* p;
    int64_t n;
    int size;
    bool written, wanted;
  } arrays[] = {{"grad", t.grad, t.numel, element_size(t.grad_dtype), false, true},
                {"param", t.param, t.numel, element_size(t.dtype), true, true},
                {"copy", t.copy, t.numel, 2, true, t.copy != nullptr},
                {"m", t.m, t.numel, state, true, true},
                {"v", t.v, t.numel, state, true, true},
                {"m_scale", t.m_scale, blocks, 4, true, bits == 8},
                {"v_scale", t.v_scale, blocks, 4, true, bits == 8}};
  for (const auto& x : arrays) {
    if (!x.wanted) continue;
    if (!x.p) return fail(GBMW_ERR_INVALID_ARG, "%s of tensor %d is null", x.name, i);
    if ((uintptr_t)x.p % (unsigned)x.size) return fail(GBMW_ERR_INVALID_ARG, "%s of tensor %d is not aligned to its elements", x.name, i);
    all.push_back({(uintptr_t)x.p, (uintptr_t)x.p + (uintptr_t)(x.n * x.size), x.written, i});
  }
  return GBMW_OK;
}

}  // namespace
}  // namespace gbmw

using namespace gbmw;

struct gbmw_adamw_list {
  gbmw_detail::DevBuf runs;
  int count = 0, device = 0, bits = 32;
};

extern "C" gbmw_status gbmw_adamw_list_create(int32_t n, const gbmw_adamw_tensor* tensors, int32_t state_bits,
                                              gbmw_adamw_list** list) {
  gbmw_detail::clear_error();
  if (!list) return fail(GBMW_ERR_INVALID_ARG, "null list");
  *list = nullptr;
  if (n < 0 || (n > 0 && !tensors)) return fail(GBMW_ERR_INVALID_ARG, "n=%d, or no tensors", n);
  if (state_bits != 8 && state_bits != 32) return fail(GBMW_ERR_INVALID_ARG, "state_bits=%d is neither 8 nor 32", state_bits);
  try {
    std::vector<Extent> all;
    int64_t count = 0;
    for (int i = 0; i < n; ++i) {
      CHECK(check_adamw(i, tensors[i], state_bits, all));
      count += (tensors[i].numel + kRun - 1) / kRun;
    }
    if (count > (1 << 27)) return fail(GBMW_ERR_INVALID_ARG, "more than 2^41 elements");
    const int bad = overlap(all);
    if (bad >= 0) return fail(GBMW_ERR_INVALID_ARG, "tensor %d: an array overlaps another, and one of them is written", bad);
    std::vector<Run> runs;
    runs.reserve((size_t)count);
    uint32_t block = 0;
    for (int i = 0; i < n; ++i) {
      const gbmw_adamw_tensor& t = tensors[i];
      const int gs = element_size(t.grad_dtype), ps = element_size(t.dtype), ss = state_bits == 8 ? 1 : 4;
      for (int64_t at = 0; at < t.numel; at += kRun) {
        Run r{};
        r.grad = (const char*)t.grad + at * gs, r.param = (char*)t.param + at * ps;
        r.copy = t.copy ? (char*)t.copy + at * 2 : nullptr;
        r.m = (char*)t.m + at * ss, r.v = (char*)t.v + at * ss;
        if (state_bits == 8) r.m_scale = t.m_scale + at / kBlock, r.v_scale = t.v_scale + at / kBlock;
        r.n = (int32_t)std::min(kRun, t.numel - at);
        r.block = block + (uint32_t)(at / kBlock);
        r.grad_dtype = t.grad_dtype, r.dtype = t.dtype, r.copy_dtype = t.copy_dtype, r.decay = t.weight_decay;
        runs.push_back(r);
      }
      block += (uint32_t)((t.numel + kBlock - 1) / kBlock);
    }
    gbmw_adamw_list* l = new gbmw_adamw_list;
    l->count = (int)count, l->bits = state_bits;
    gbmw_status st = l->runs.reserve(sizeof(Run) * (size_t)count);
    if (st == GBMW_OK) {
      hipError_t e = hipGetDevice(&l->device);
      if (e == hipSuccess && count) e = hipMemcpy(l->runs.p, runs.data(), sizeof(Run) * (size_t)count, hipMemcpyHostToDevice);
      if (e != hipSuccess) {
        (void)hipGetLastError();
        st = fail(GBMW_ERR_DEVICE, "list: %s", hipGetErrorString(e));
      }
    }
    if (st != GBMW_OK) {
      l->runs.release();
      delete l;
      return st;
    }
    *list = l;
    return GBMW_OK;
  } catch (const std::bad_alloc&) {
    return fail(GBMW_ERR_OOM, "host memory for a list of %d tensors", n);
  }
}

extern "C" gbmw_status gbmw_adamw_step(const gbmw_adamw_list* l, const gbmw_adamw_options* o, void* stream) {
  gbmw_detail::clear_error();
  if (!l || !o) return fail(GBMW_ERR_INVALID_ARG, "null list or options");
  if (!(o->lr >= 0.0) || !std::isfinite(o->lr)) return fail(GBMW_ERR_INVALID_ARG, "lr=%g", o->lr);
  if (!(o->beta1 >= 0.0 && o->beta1 < 1.0)) return fail(GBMW_ERR_INVALID_ARG, "beta1=%g", o->beta1);
  if (!(o->beta2 >= 0.0 && o->beta2 < 1.0)) return fail(GBMW_ERR_INVALID_ARG, "beta2=%g", o->beta2);
  if (!((float)o->eps > 0.0f) || !std::isfinite((float)o->eps)) return fail(GBMW_ERR_INVALID_ARG, "eps=%g", o->eps);
  if (!((float)o->scale > 0.0f) || !std::isfinite((float)o->scale)) return fail(GBMW_ERR_INVALID_ARG, "scale=%g", o->scale);
  if (!(o->max_norm > 0.0)) return fail(GBMW_ERR_INVALID_ARG, "max_norm=%g is not positive", o->max_norm);
  if (!o->step_now && o->step < 1) return fail(GBMW_ERR_INVALID_ARG, "step=%lld is below 1", (long long)o->step);
  if ((uintptr_t)o->norm % 4 || (uintptr_t)o->lr_now % 4 || (uintptr_t)o->step_now % 8)
    return fail(GBMW_ERR_INVALID_ARG, "norm, lr_now or step_now is not aligned to its type");
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != l->device) return fail(GBMW_ERR_INVALID_ARG, "the list is on device %d, device %d is current", l->device, dev);
  if (l->count == 0) return GBMW_OK;
  const AdamArgs a{o->lr, o->beta1, o->beta2, o->scale, o->max_norm, (float)o->eps, o->step, o->seed, o->norm, o->lr_now, o->step_now};
  const dim3 grid(std::min(l->count, kMostGroups)), block(256);
  hipStream_t st = (hipStream_t)stream;
  if (l->bits == 8) hipLaunchKernelGGL(k_adamw<true>, grid, block, 0, st, (const Run*)l->runs.p, l->count, a);
  else hipLaunchKernelGGL(k_adamw<false>, grid, block, 0, st, (const Run*)l->runs.p, l->count, a);
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

extern "C" void gbmw_adamw_list_destroy(gbmw_adamw_list* l) {
  if (!l) return;
  int current = l->device;
  (void)hipGetDevice(&current);
  if (current != l->device) (void)hipSetDevice(l->device);
  (void)hipDeviceSynchronize();
  l->runs.release();
  if (current != l->device) (void)hipSetDevice(current);
  delete l;
}
