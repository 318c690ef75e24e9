// One AdamW step over many tensors, with states in 32 bits or in 8.  Contract: include/gbmw.h.
#include <new>
#include <vector>

#include "gbmw_rows.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

// Bound by HBM: every array is read and written once, and arithmetic (in 8 bits about 80 vector operations an element)
// stays below that.  A workgroup has 1024 elements and ends: the more of them there are, the closer together lies what the chip
// has in flight, and the better memory takes it.  197M parameters, bf16 gradients and copies: states in 32 bits 918 us,
// 6.0 TB/s; 2048 workgroups that walk runs of 16384 elements 1210, with loads and stores through the cache 1361.  States
// in 8 bits 520 us, 6.1 TB/s (with eight elements of a lane next to each other, whose stores are half lines, 6 % more).
// Runs dealt to the dies one by one: 906 us in 32 bits, 1 % more in 8, and 16M parameters with fp32 gradients and no
// copies 80 us, which take 76 in lots.
constexpr int kBlock = 256;         // elements that share a scale
constexpr int kRun = 1024;          // elements of a workgroup
constexpr int kMostRuns = 1 << 23;  // of a launch

template <bool BITS8>
constexpr int kThreads = BITS8 ? 128 : 256;

struct Run {   // elements of one tensor, whose places have the same upper 32 bits
  const void* grad;
  void *param, *copy, *m, *v;
  float *m_scale, *v_scale;
  int64_t block;    // number of the run's first block in the list
  int32_t n;
  uint32_t types;   // the gradient's, the parameter's << 8, the copy's << 16
  float decay;
  __device__ __forceinline__ int grad_type() const { return types & 255; }
  __device__ __forceinline__ int type() const { return types >> 8 & 255; }
  __device__ __forceinline__ int copy_type() const { return types >> 16; }
};

// The numbers that all elements share: computed in fp64, rounded once.
struct Rates {
  double lr;
  float grad, b1, a1, b2, a2, eps, lr_c1, root_c2;
  uint32_t key;   // of the random numbers
};

struct AdamArgs {
  Rates r;   // of the numbers that the host knows
  double beta1, beta2, scale, max_norm, c1;
  uint32_t seed;   // 0: round to nearest
  const float *norm, *lr_now;
  const int64_t* step_now;
};

// The multipliers are xxHash's published primes; what a hash of 0 is (0) is a key like any other.
constexpr uint32_t kHashBy = 0x9E3779B1u;
__host__ __device__ __forceinline__ uint32_t hash_rest(uint32_t x) {
  x = (x ^ (x >> 15)) * 0x85EBCA77u;
  return x ^ (x >> 13);
}
__host__ __device__ __forceinline__ uint32_t hash(uint32_t x) { return hash_rest(x * kHashBy); }

// The key of a step, and of the places of 32 bits that have `high` above them, if that is not 0.
__device__ __forceinline__ uint32_t key_above(uint32_t key, uint32_t high) { return high ? hash(key + high * 0x9E3779B9u) : key; }

__host__ __device__ __forceinline__ uint32_t key_of(uint32_t seed, int64_t step) {
  return hash(seed + (uint32_t)step * 0x9E3779B9u);
}

__host__ __device__ __forceinline__ double power(double x, int64_t n) {
  double p = 1.0;
  for (; n; n >>= 1, x *= x)
    if (n & 1) p *= x;
  return p;
}

// What the device knows alone is read here, with the elements on their way.  False: the step is left out.
__device__ __forceinline__ bool rates_now(const AdamArgs& a, Rates& r) {
  if (a.norm) {
    const double norm = (double)*a.norm;
    if (!(norm < __builtin_inf())) return false;   // a NaN too
    if (norm > a.max_norm) r.grad = (float)(a.scale * (a.max_norm / norm));
  }
  double c1 = a.c1;
  if (a.step_now) {
    int64_t step = *a.step_now;
    if (step < 1) step = 1;
    c1 = 1.0 - power(a.beta1, step);
    r.root_c2 = (float)(1.0 / __builtin_sqrt(1.0 - power(a.beta2, step)));
    r.key = key_of(a.seed, step);
  }
  if (a.lr_now) r.lr = (double)*a.lr_now;
  if (a.lr_now || a.step_now) r.lr_c1 = (float)(r.lr / c1);
  return true;
}

// N elements at p of which n (0..N) are there, loaded or stored at once where all are.  Nothing is
// read or written twice in a step, so all of it passes the cache by.  Arrays that begin in the middle of a
// line (40M parameters: 183 us become 196, in 8 bits 107 become 162) take the same way: through the cache
// they take 280 and 161.
template <typename T, int N>
struct alignas(sizeof(T)) Few {
  T v[N];
};
template <int WORDS>
using Words = uint32_t __attribute__((ext_vector_type(WORDS), aligned(1)));

template <typename T, int N>
__device__ __forceinline__ Few<T, N> load(const void* p, int64_t i, int n) {
  constexpr int kParts = sizeof(Few<T, N>) > 16 ? 2 : 1, kWords = sizeof(Few<T, N>) / (4 * kParts);
  Few<T, N> r;
  if (n >= N) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const auto w = __builtin_nontemporal_load((const Words<kWords>*)((const T*)p + i) + k);
      __builtin_memcpy((char*)&r + 4 * kWords * k, &w, 4 * kWords);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) r.v[e] = e < n ? ((const T*)p)[i + e] : (T)0;
  }
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void store(void* p, int64_t i, const Few<T, N>& x, int n) {
  constexpr int kParts = sizeof(x) > 16 ? 2 : 1, kWords = sizeof(x) / (4 * kParts);
  if (n >= N) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      Words<kWords> w;
      __builtin_memcpy(&w, (const char*)&x + 4 * kWords * k, 4 * kWords);
      __builtin_nontemporal_store(w, (Words<kWords>*)((T*)p + i) + k);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) ((T*)p)[i + e] = x.v[e];
  }
}

template <int N>
__device__ __forceinline__ void store_copy(const Run& run, int i, const float (&p)[N], int n) {
  if (!run.copy) return;
  if (run.copy_type() == GBMW_F16) {
    Few<f16, N> c;
#pragma unroll
    for (int e = 0; e < N; ++e) c.v[e] = (f16)p[e];
    store(run.copy, i, c, n);
  } else {
    Few<bf16, N> c;
#pragma unroll
    for (int e = 0; e < N; ++e) c.v[e] = (bf16)p[e];
    store(run.copy, i, c, n);
  }
}

// States in 32 bits: a thread has four elements.
template <typename G, typename P>
__device__ __forceinline__ void run_of_32(const Run& run, const AdamArgs& a) {
  constexpr int N = kRun / kThreads<false>;
  const int i = threadIdx.x * N, n = run.n - i;   // 0 or less behind the last element
  if (n <= 0) return;
  const Few<G, N> g = load<G, N>(run.grad, i, n);
  Few<P, N> p = load<P, N>(run.param, i, n);
  Few<float, N> m = load<float, N>(run.m, i, n), v = load<float, N>(run.v, i, n);
  Rates r = a.r;
  if (!rates_now(a, r)) return;
  const float keep = (float)(1.0 - r.lr * (double)run.decay);
  float q[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float d = (float)g.v[e] * r.grad;
    m.v[e] = m.v[e] * r.b1 + d * r.a1;
    v.v[e] = v.v[e] * r.b2 + d * d * r.a2;
    q[e] = (float)p.v[e] * keep - m.v[e] / (__builtin_sqrtf(v.v[e]) * r.root_c2 + r.eps) * r.lr_c1;
    p.v[e] = (P)q[e];
  }
  store(run.param, i, p, n), store(run.m, i, m, n), store(run.v, i, v, n);
  store_copy(run, i, q, n);
}

__device__ __forceinline__ unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }   // a NaN's is the largest

template <int CTRL>
__device__ __forceinline__ unsigned max_dpp(unsigned x) {
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float most_of_32(unsigned x) {   // over a half of the wave
  x = max_dpp<0xB1>(x);    // lane ^ 1
  x = max_dpp<0x4E>(x);    // lane ^ 2
  x = max_dpp<0x141>(x);   // the other half of eight
  x = max_dpp<0x140>(x);   // the other half of sixteen
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return __builtin_bit_cast(float, max((unsigned)r[0], (unsigned)r[1]));
}

// Rounded roots, of values from `least` to `most` (as bits): the root by the hardware's reciprocal root is put right by half of
// what its square leaves of x, which a fused operation has exactly.  That is the rounded root of every number of 32 bits
// from 2^-96 on, compared with the one in 64 bits; smaller ones and infinity go the compiler's way.
template <int N>
__device__ __forceinline__ void roots(float (&x)[N], unsigned least, unsigned most) {
  if (least < __builtin_bit_cast(unsigned, 0x1p-96f) || most >= __builtin_bit_cast(unsigned, __builtin_inff())) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = __builtin_sqrtf(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float y = __builtin_amdgcn_rsqf(x[e]), root = x[e] * y;
      x[e] = __builtin_fmaf(__builtin_fmaf(-root, root, x[e]), 0.5f * y, root);
    }
  }
}

// Four values in 8 bits.  By the hash the conversion adds `random` (its upper 20 bits, below the last digit that is
// kept) and cuts off: sixteen bits of the hash, and a half behind them.
__device__ __forceinline__ uint32_t codes_of(const float* x, bool at_random, const uint32_t* random) {
  int c = 0;
  if (at_random) {
    c = __builtin_amdgcn_cvt_sr_fp8_f32(x[0], random[0], c, 0);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(x[1], random[1], c, 1);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(x[2], random[2], c, 2);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(x[3], random[3], c, 3);
  } else {
    c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], c, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], c, true);
  }
  return (uint32_t)c;
}

__device__ __forceinline__ Few<uint8_t, 4> bytes_of(uint32_t c) {
  Few<uint8_t, 4> b;
  __builtin_memcpy(&b, &c, 4);
  return b;
}
__device__ __forceinline__ void values_of(const Few<uint8_t, 4>& code, float* x) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const int c = __builtin_bit_cast(int, code);
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
}

// States in 8 bits: half a wave has a block, a lane four elements of each half of it, so that every store of the wave is
// whole lines.  Moments, scales and codes are the header's formula, each operation rounded: rounding at random carries a
// last place into a whole code now and then, and from there into scales (184 of 10^8 codes a step, had products and sums
// one rounding, and root and quotient a last place to spare).  Vector operations take 0.8 to 0.9 of the cycles, so what is exact
// has to be short: with the compiler's roots, and a key for each block, they take all of them and a kernel 3 % longer; the parameter
// takes the hardware's reciprocal, off by one unit of its last place (with a division 3 % more).  Parameters of 16 bits, which
// move less, are bound by them: 197M bf16 378 us, 5.2 TB/s, with that last place to spare 351.
template <typename G, typename P>
__device__ __forceinline__ void run_of_8(const Run& run, const AdamArgs& a) {
  constexpr int N = 4, U = 2, kApart = kBlock / U;
  static_assert(kRun == kThreads<true> * N * U && kApart == 32 * N, "");
  const int k = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (k * kBlock >= run.n) return;
  const int i = k * kBlock + lane * N;
  Few<G, N> g[U];
  Few<P, N> p[U];
  Few<uint8_t, N> mc[U], vc[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = i + u * kApart, n = run.n - at;   // 0 or less behind the last element
    g[u] = load<G, N>(run.grad, at, n), p[u] = load<P, N>(run.param, at, n);
    mc[u] = load<uint8_t, N>(run.m, at, n), vc[u] = load<uint8_t, N>(run.v, at, n);
  }
  const float ms = run.m_scale[k], vs = run.v_scale[k];
  Rates r = a.r;
  if (!rates_now(a, r)) return;
  const float keep = (float)(1.0 - r.lr * (double)run.decay);
  float m[U * N], root[U * N], q[U][N];
  unsigned most_m = 0, most_v = 0, least_v = ~0u;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    values_of(mc[u], m + u * N), values_of(vc[u], root + u * N);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float &me = m[u * N + e], &ve = root[u * N + e];
      const float d = (float)g[u].v[e] * r.grad, old = ve * vs;
      me = me * ms * r.b1 + d * r.a1;
      ve = old * old * r.b2 + d * d * r.a2;
      // as whole numbers: a NaN is the largest; squares have no sign
      const unsigned bits = __builtin_bit_cast(unsigned, ve);
      most_m = max(most_m, magnitude(me)), most_v = max(most_v, bits), least_v = min(least_v, bits);
    }
  }
  roots(root, least_v, most_v);
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float me = m[u * N + e], ve = root[u * N + e];
      q[u][e] = (float)p[u].v[e] * keep - me * __builtin_amdgcn_rcpf(ve * r.root_c2 + r.eps) * r.lr_c1;
    }
  const float new_ms = scale_of(most_of_32(most_m), 1.0f / 448.0f);
  const float new_vs = scale_of(__builtin_sqrtf(most_of_32(most_v)), 1.0f / 448.0f);
  divide<false>(m, new_ms), divide<false>(root, new_vs);
#pragma unroll
  for (int e = 0; e < U * N; ++e) {
    m[e] = __builtin_amdgcn_fmed3f(m[e], -448.0f, 448.0f);
    root[e] = root[e] > 0.0f ? __builtin_amdgcn_fmed3f(root[e], 0x1p-9f, 448.0f) : 0.0f;
  }
  uint32_t high[U * N] = {}, low[U * N] = {};
  if (a.seed) {
    const uint32_t key = key_above(r.key, (uint32_t)(run.block >> 24)), first = ((uint32_t)run.block + k) * kBlock + lane * N;
    static_assert(kBlock == 256, "");
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // hash(place ^ key) with its first product taken apart: the place of the lane's four, and the two bits below it
      const uint32_t base = ((first + u * kApart) ^ (key & ~3u)) * kHashBy;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint32_t word = hash_rest(base + (e ^ (key & 3u)) * kHashBy);
        high[u * N + e] = (word & 0xffff0000u) | 0x8000, low[u * N + e] = word << 16 | 0x8000;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = i + u * kApart, n = run.n - at;
    const uint32_t mw = codes_of(m + u * N, a.seed != 0, high + u * N), vw = codes_of(root + u * N, a.seed != 0, low + u * N);
    if (n <= 0) continue;
    store(run.m, at, bytes_of(mw), n);
    store(run.v, at, bytes_of(vw), n);
    Few<P, N> to;
#pragma unroll
    for (int e = 0; e < N; ++e) to.v[e] = (P)q[u][e];
    store(run.param, at, to, n);
    store_copy(run, at, q[u], n);
  }
  if (lane == 0) run.m_scale[k] = new_ms, run.v_scale[k] = new_vs;
}

template <bool BITS8, typename G, typename P>
__device__ __forceinline__ void run_of(const Run& run, const AdamArgs& a) {
  if constexpr (BITS8) run_of_8<G, P>(run, a);
  else run_of_32<G, P>(run, a);
}

template <bool BITS8, typename G>
__device__ __forceinline__ void run_of(const Run& run, const AdamArgs& a) {
  if (run.type() == GBMW_F32) run_of<BITS8, G, float>(run, a);
  else if (run.type() == GBMW_F16) run_of<BITS8, G, f16>(run, a);
  else run_of<BITS8, G, bf16>(run, a);
}

template <bool BITS8>
__global__ __launch_bounds__(kThreads<BITS8>) void k_adamw(const Run* runs, AdamArgs a) {
  // workgroups go to the eight dies in turn; lots of 128 runs are one die's, whose cache then holds whole lines of scales
  // and descriptors
  constexpr unsigned kLot = 7, kAll = 8u << kLot;
  unsigned id = blockIdx.x;
  if ((id | (kAll - 1)) < gridDim.x) id = (id & ~(kAll - 1)) | ((id & 7) << kLot) | ((id >> 3) & ((1u << kLot) - 1));
  const Run run = runs[id];
  if (run.grad_type() == GBMW_F32) run_of<BITS8, float>(run, a);
  else if (run.grad_type() == GBMW_F16) run_of<BITS8, f16>(run, a);
  else run_of<BITS8, bf16>(run, a);
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
  int64_t count = 0;
  int device = 0, bits = 32;
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
    int64_t total = 0, count = 0;
    for (int i = 0; i < n; ++i) {
      CHECK(check_adamw(i, tensors[i], state_bits, all));
      total += tensors[i].numel;
      if (total > (1ll << 41)) return fail(GBMW_ERR_INVALID_ARG, "more than 2^41 elements");
    }
    const int bad = overlap(all);
    if (bad >= 0) return fail(GBMW_ERR_INVALID_ARG, "tensor %d: an array overlaps another, and one of them is written", bad);
    std::vector<Run> runs;
    runs.reserve((size_t)(total / kRun + n + (total >> 32) + 1));
    int64_t block = 0;
    for (int i = 0; i < n; ++i) {
      const gbmw_adamw_tensor& t = tensors[i];
      const int gs = element_size(t.grad_dtype), ps = element_size(t.dtype), ss = state_bits == 8 ? 1 : 4;
      for (int64_t at = 0, next; at < t.numel; at = next) {
        Run r{};
        r.grad = (const char*)t.grad + at * gs, r.param = (char*)t.param + at * ps;
        r.copy = t.copy ? (char*)t.copy + at * 2 : nullptr;
        r.m = (char*)t.m + at * ss, r.v = (char*)t.v + at * ss;
        if (state_bits == 8) r.m_scale = t.m_scale + at / kBlock, r.v_scale = t.v_scale + at / kBlock;
        r.block = block + at / kBlock, r.decay = t.weight_decay;
        const int64_t upper = (r.block | ((1 << 24) - 1)) + 1;   // block whose places' upper 32 bits are others
        next = std::min(t.numel, at + std::min<int64_t>(kRun, (upper - r.block) * kBlock));
        r.n = (int32_t)(next - at);
        r.types = t.grad_dtype | t.dtype << 8 | (t.copy ? t.copy_dtype << 16 : 0);
        runs.push_back(r);
      }
      block += (t.numel + kBlock - 1) / kBlock;
    }
    count = (int64_t)runs.size();
    gbmw_adamw_list* l = new gbmw_adamw_list;
    l->count = count, l->bits = state_bits;
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
  if (!((float)o->eps >= 0x1p-126f) || !std::isfinite((float)o->eps)) return fail(GBMW_ERR_INVALID_ARG, "eps=%g", o->eps);
  if (!((float)o->scale > 0.0f) || !std::isfinite((float)o->scale)) return fail(GBMW_ERR_INVALID_ARG, "scale=%g", o->scale);
  if (!(o->max_norm > 0.0)) return fail(GBMW_ERR_INVALID_ARG, "max_norm=%g is not positive", o->max_norm);
  if (!o->step_now && o->step < 1) return fail(GBMW_ERR_INVALID_ARG, "step=%lld is below 1", (long long)o->step);
  if ((uintptr_t)o->norm % 4 || (uintptr_t)o->lr_now % 4 || (uintptr_t)o->step_now % 8)
    return fail(GBMW_ERR_INVALID_ARG, "norm, lr_now or step_now is not aligned to its type");
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != l->device) return fail(GBMW_ERR_INVALID_ARG, "the list is on device %d, device %d is current", l->device, dev);
  if (l->count == 0) return GBMW_OK;
  AdamArgs a{};
  const int64_t step = std::max<int64_t>(1, o->step);   // read on the device if step_now is given
  a.beta1 = o->beta1, a.beta2 = o->beta2, a.scale = o->scale, a.max_norm = o->max_norm, a.seed = o->seed;
  a.norm = o->norm, a.lr_now = o->lr_now, a.step_now = o->step_now;
  a.c1 = 1.0 - power(o->beta1, step);
  a.r.lr = o->lr, a.r.grad = (float)o->scale, a.r.eps = (float)o->eps;
  a.r.b1 = (float)o->beta1, a.r.a1 = (float)(1.0 - o->beta1), a.r.b2 = (float)o->beta2, a.r.a2 = (float)(1.0 - o->beta2);
  a.r.lr_c1 = (float)(o->lr / a.c1), a.r.root_c2 = (float)(1.0 / std::sqrt(1.0 - power(o->beta2, step)));
  a.r.key = key_of(o->seed, step);
  hipStream_t st = (hipStream_t)stream;
  for (int64_t at = 0; at < l->count; at += kMostRuns) {
    const dim3 grid((unsigned)std::min<int64_t>(kMostRuns, l->count - at));
    const Run* runs = (const Run*)l->runs.p + at;
    if (l->bits == 8) hipLaunchKernelGGL(k_adamw<true>, grid, dim3(kThreads<true>), 0, st, runs, a);
    else hipLaunchKernelGGL(k_adamw<false>, grid, dim3(kThreads<false>), 0, st, runs, a);
  }
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
