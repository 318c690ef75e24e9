// Attention, forward and backward (contract: include/gbmw.h), on the matrix cores.
//
// The query heads that read one key head are rows of ONE problem: row r of (sample, key
// head) is query r / share of query head r % share, so shared heads cost no extra reads of
// keys and values, and dk and dv are sums over rows like any other.
//
// All products are 32x32x16 matrix instructions.  Of an A or B operand lane l holds row (or
// column) l % 32 and eight consecutive terms, 8 * (l / 32) on, of the sum; of a result it
// holds column l % 32 and rows 8 * (r / 4) + 4 * (l / 32) + r % 4, r = 0..15.  The order of
// the terms of a sum is free as long as both operands agree, so a result's registers
// 8t .. 8t+7, rounded to 16 bits, ARE a B operand whose terms are the rows
//   16 t + 8 (i / 4) + 4 (l / 32) + i % 4,  i = 0..7:
// probabilities go from one product into the next without leaving their lanes, and the
// other operand is read in the same order (read_cols).
#include <algorithm>
#include <climits>
#include <cmath>

#include "gbmw_ctx.h"
#include "gbmw_dtype.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct AttnArgs {
  const char *q, *k, *v, *dout;
  char *out, *dq, *dk, *dv;
  float *lse, *delta;
  float *vmax, *gmax;   // f16: the largest norms of a value and of a row of dout, for parts of 256 keys and 128 rows
  int64_t qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];
  const int *len_q, *len_k;
  int B, Hq, Hk, Lq, Lk, D, share, causal;
  float c;       // scale * log2(e): probabilities are powers of two
  float scale;
};

template <typename T>
__device__ __forceinline__ f32x16 mma(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (sizeof(T) == 2 && __is_same(T, f16))
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
}

// Registers 8t .. 8t+7 of a result as an operand of the next product.
template <typename T>
__device__ __forceinline__ s16x8 round8(const f32x16& x, int t) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  Tx8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (T)x[8 * t + i];
  return __builtin_bit_cast(s16x8, r);
}

// ---- tiles in LDS: rows of CH 16-byte pieces, the piece swapped by the row -----------------
//
// read_row8 reads one piece of 32 rows, read_cols 32 bytes each of four rows; with the piece
// exclusive-or'ed with this function of the row both touch every bank once per cycle.
__device__ __forceinline__ int swap_of(int row) { return ((row & 3) << 1) | ((row >> 2) & 1); }

template <int CH>
__device__ __forceinline__ int piece_at(int row, int piece) {   // in 16-bit elements
  return (row * CH + (piece ^ swap_of(row))) * 8;
}

// A operand whose rows are the tile's rows row .. row+31 and whose terms are the columns
// 16 step .. 16 step + 15.
template <int CH>
__device__ __forceinline__ s16x8 read_rows(const short* tile, int row, int step) {
  const int l = threadIdx.x % 64;
  return *(const s16x8*)&tile[piece_at<CH>(row + l % 32, 2 * step + l / 32)];
}

// A operand whose rows are the tile's columns col .. col+31 and whose terms are its rows
// row .. row+15 in the order above.  The transposing read gives lane i of 16 element i of each
// of four runs of 16 elements, lanes 4u..4u+3 naming the four quarters of run u.
template <int CH>
__device__ __forceinline__ s16x8 read_cols(const short* tile, int row, int col) {
  typedef __attribute__((address_space(3))) s16x4 lds4;
  const int l = threadIdx.x % 64, i = l % 16;
  const int r = row + 4 * (l / 32) + i / 4, c = col + 16 * ((l / 16) % 2) + 4 * (i % 4);
  s16x4 x[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const short* p = &tile[piece_at<CH>(r + 8 * u, c / 8) + c % 8];
    x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p);
  }
  return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// A piece of a row in global memory; zeros beyond D and where the row is not there.
__device__ __forceinline__ s16x8 load8(const char* row, int piece, int D, bool there) {
  const Pack<bf16> r = load_pack((const bf16*)row + 8 * piece, there ? D - 8 * piece : 0);
  return __builtin_bit_cast(s16x8, r);
}

// Pieces of one 64-row tile that a thread of 256 loads: piece n = threadIdx.x + 256 i is piece
// n % (2 KS) of row n / (2 KS).
template <int KS>
constexpr int kLoads = (64 * 2 * KS + 255) / 256;

template <int KS>
struct Staged {
  s16x8 x[kLoads<KS>];
};

// rows first .. first+63 of an array with one head: row r is at base + r * stride (bytes)
template <int KS>
__device__ __forceinline__ void fetch(Staged<KS>& s, const char* base, int64_t stride, int first, int rows, int D) {
#pragma unroll
  for (int i = 0; i < kLoads<KS>; ++i) {
    const int n = threadIdx.x + 256 * i, r = n / (2 * KS);
    const bool there = first + r < rows && r < 64;
    s.x[i] = load8(base + (there ? (int64_t)(first + r) * stride : 0), n % (2 * KS), D, there);
  }
}

// the same of the rows of a group of heads
template <int KS>
__device__ __forceinline__ void fetch_group(Staged<KS>& s, const char* base, int64_t row_stride, int64_t head_stride,
                                            int share, int first, int rows, int D) {
#pragma unroll
  for (int i = 0; i < kLoads<KS>; ++i) {
    const int n = threadIdx.x + 256 * i, r = n / (2 * KS);
    const bool there = first + r < rows && r < 64;
    const int at = there ? first + r : 0, x = at / share;
    s.x[i] = load8(base + x * row_stride + (at - x * share) * head_stride, n % (2 * KS), D, there);
  }
}

template <int KS, int CH>
__device__ __forceinline__ void put(short* tile, const Staged<KS>& s) {
#pragma unroll
  for (int i = 0; i < kLoads<KS>; ++i) {
    const int n = threadIdx.x + 256 * i, r = n / (2 * KS);
    if (r < 64) *(s16x8*)&tile[piece_at<CH>(r, n % (2 * KS))] = s.x[i];
  }
}

__device__ __forceinline__ int length(const int* len, int b, int most) {
  return len ? max(0, min(len[b], most)) : most;
}

// A row of the result of a product over d: lane l has column (row of the problem) l % 32 and
// the d of its registers, four at a time.
template <typename T>
__device__ __forceinline__ void store4(char* row, int d, int D, const f32x16& x, int r, float f) {
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  Tx4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (T)(x[r + i] * f);
  T* p = (T*)row + d;
  if (d + 4 <= D) {
    __builtin_memcpy(p, &y, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < D) p[i] = y[i];
  }
}

// Probabilities times 2^kUp: float16 loses digits below 2^-14, and a thousand keys have
// probabilities of a thousandth.
template <typename T>
constexpr float kUp = __is_same(T, f16) ? 8.0f : 0.0f;

// ... and score gradients times 2^k, the largest that keeps those of a row under 2^14: with
// |dout_i| <= g and |v_j| <= v they are at most 2 g v, out being a mean of values.
__device__ __forceinline__ int lift_of(float gv) {
  const float bound = 2.0f * gv;
  if (!(bound > 0.0f) || !(bound < kInf)) return 0;
  int e;
  (void)frexpf(bound, &e);
  return max(-100, min(100, 14 - e));
}

__device__ __forceinline__ float max_of(const float* x, int n) {   // n values, the same in every thread of a wave
  float m = 0.0f;
  for (int i = threadIdx.x % 64; i < n; i += 64) m = fmaxf(m, x[i]);
#pragma unroll
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  return m;
}

template <int KS>
constexpr int kChunks = KS <= 4 ? 8 : 16;

// ---- forward --------------------------------------------------------------------------------
//
// A workgroup takes 128 rows of one (sample, key head), 32 a wave, and walks the keys in tiles
// of 64.  A wave computes x^T = K Q^T (lane: one row, 32 keys), so the running maximum and sum
// of a row need one exchange between two lanes a tile, and out^T += V^T p^T with p from its
// own registers.
template <typename T, int KS>
__global__ __launch_bounds__(256, 2) void k_attn_fwd(AttnArgs a) {
  constexpr int CH = kChunks<KS>, DB = (KS + 1) / 2;
  __shared__ __attribute__((aligned(16))) short sK[2][64 * CH * 8], sV[2][64 * CH * 8];
  const int tiles = (a.Lq * a.share + 127) / 128;
  int id = blockIdx.x;
  const int tile = tiles - 1 - id % tiles;   // the longest rows of a causal mask first
  id /= tiles;
  const int hk = id % a.Hk, b = id / a.Hk;
  const int nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk);
  const int l = threadIdx.x % 64, half = l / 32, row0 = tile * 128 + (threadIdx.x / 64) * 32;
  const int rows = a.Lq * a.share, row = row0 + l % 32;
  const int i = row / a.share, hq = hk * a.share + row % a.share;
  // the row sees keys j < sees
  const int sees = i >= nq ? 0 : a.causal ? max(0, min(nk, i + nk - nq + 1)) : nk;
  const int last_i = min((min(tile * 128 + 128, rows) - 1) / a.share, nq - 1);
  const int most = tile * 128 / a.share >= nq ? 0 : a.causal ? max(0, min(nk, last_i + nk - nq + 1)) : nk;
  const char* kb = a.k + 2 * (b * a.ks[0] + hk * a.ks[2]);
  const char* vb = a.v + 2 * (b * a.vs[0] + hk * a.vs[2]);

  s16x8 q[KS];
  {
    const char* p = a.q + 2 * (b * a.qs[0] + (i < nq ? i : 0) * a.qs[1] + hq * a.qs[2]);
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = load8(p, 2 * s + half, a.D, i < nq);
  }
  f32x16 o[DB] = {};
  float m = -kInf, sum = 0.0f;   // m in units of x / scale

  Staged<KS> nextK, nextV;
  if (most > 0) {
    fetch(nextK, kb, 2 * a.ks[1], 0, nk, a.D);
    fetch(nextV, vb, 2 * a.vs[1], 0, nk, a.D);
  }
  for (int j0 = 0, buf = 0; j0 < most; j0 += 64, buf ^= 1) {
    put<KS, CH>(sK[buf], nextK);
    put<KS, CH>(sV[buf], nextV);
    __syncthreads();   // this tile is whole, and nobody reads the other buffer any more
    if (j0 + 64 < most) {
      fetch(nextK, kb, 2 * a.ks[1], j0 + 64, nk, a.D);
      fetch(nextV, vb, 2 * a.vs[1], j0 + 64, nk, a.D);
    }
    f32x16 x[2] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS; ++s) x[u] = mma<T>(read_rows<CH>(sK[buf], 32 * u, s), q[s], x[u]);
    if (!__all(j0 + 64 <= sees)) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (j0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4 >= sees) x[u][r] = -kInf;
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, x[u][r]);
    top = fmaxf(top, __shfl_xor(top, 32));
    if (__any(top > m)) {   // the running sums are in units of the old maximum
      const float f = top > m ? __builtin_amdgcn_exp2f((m - top) * a.c) : 1.0f;
      m = top;
      sum *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= f;
    }
    const float off = (m == -kInf ? 0.0f : m * a.c) - kUp<T>;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[u][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][r], a.c, -off));
        sum += x[u][r];
      }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const s16x8 p = round8<T>(x[u], t);
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = mma<T>(read_cols<CH>(sV[buf], 32 * u + 16 * t, 32 * d), p, o[d]);
      }
  }
  sum += __shfl_xor(sum, 32);
  if (row >= rows) return;
  const bool empty = m == -kInf && !(sum != sum);
  const float f = empty ? 0.0f : 1.0f / sum;
  if (half == 0)
    a.lse[((int64_t)b * a.Hq + hq) * a.Lq + i] = empty ? -kInf : (m * a.c - kUp<T> + __builtin_amdgcn_logf(sum)) * kLn2;
  char* out = a.out + 2 * (b * a.os[0] + i * a.os[1] + hq * a.os[2]);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int at = 32 * d + 8 * (r / 4) + 4 * half;
      if (at < a.D) store4<T>(out, at, a.D, o[d], r, f);
    }
}

// The largest norm of a value among 256 keys of a (sample, key head), for float16's lift.
__global__ __launch_bounds__(256) void k_attn_vmax(AttnArgs a) {
  __shared__ float tops[4];
  const int parts = (a.Lk + 255) / 256, part = blockIdx.x % parts;
  const int hk = blockIdx.x / parts % a.Hk, b = blockIdx.x / parts / a.Hk;
  const int key = part * 256 + threadIdx.x;
  float s = 0.0f;
  if (key < length(a.len_k, b, a.Lk)) {
    const f16* v = (const f16*)a.v + b * a.vs[0] + key * a.vs[1] + hk * a.vs[2];
    for (int d = 0; d < a.D; d += 8) {
      const Pack<f16> x = load_pack(v + d, a.D - d);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)x.v[e], (float)x.v[e], s);
    }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) s = fmaxf(s, __shfl_xor(s, d));
  if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.vmax[blockIdx.x] = __builtin_sqrtf(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
}

// ---- backward, dq -----------------------------------------------------------------------------
//
// Rows and keys as in the forward pass: p^T from K Q^T and the row's log-sum-exp, dp^T = V
// dout^T, ds^T = p^T (dp^T - delta), dq^T += K^T ds^T.  Writes delta = <dout, out> of its rows and,
// for float16, their largest norm for the other kernel.
template <typename T, int KS>
__global__ __launch_bounds__(256, 2) void k_attn_dq(AttnArgs a) {
  constexpr int CH = kChunks<KS>, DB = (KS + 1) / 2;
  constexpr bool kLift = __is_same(T, f16);
  __shared__ __attribute__((aligned(16))) short sK[2][64 * CH * 8], sV[2][64 * CH * 8];
  const int tiles = (a.Lq * a.share + 127) / 128;
  int id = blockIdx.x;
  const int tile = tiles - 1 - id % tiles;
  id /= tiles;
  const int hk = id % a.Hk, b = id / a.Hk;
  const int nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk);
  const int l = threadIdx.x % 64, half = l / 32, row0 = tile * 128 + (threadIdx.x / 64) * 32;
  const int rows = a.Lq * a.share, row = row0 + l % 32;
  const int i = row / a.share, hq = hk * a.share + row % a.share;
  const int sees = i >= nq ? 0 : a.causal ? max(0, min(nk, i + nk - nq + 1)) : nk;
  const int last_i = min((min(tile * 128 + 128, rows) - 1) / a.share, nq - 1);
  const int most = tile * 128 / a.share >= nq ? 0 : a.causal ? max(0, min(nk, last_i + nk - nq + 1)) : nk;
  const char* kb = a.k + 2 * (b * a.ks[0] + hk * a.ks[2]);
  const char* vb = a.v + 2 * (b * a.vs[0] + hk * a.vs[2]);

  s16x8 q[KS], g[KS];
  float delta = 0.0f, lse = kInf, norm = 0.0f;
  {
    const int ii = i < nq ? i : 0;
    const char* p = a.q + 2 * (b * a.qs[0] + ii * a.qs[1] + hq * a.qs[2]);
    const char* d = a.dout + 2 * (b * a.dos[0] + ii * a.dos[1] + hq * a.dos[2]);
    const char* o = a.out + 2 * (b * a.os[0] + ii * a.os[1] + hq * a.os[2]);
    typedef T Tx8 __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = load8(p, 2 * s + half, a.D, i < nq);
      g[s] = load8(d, 2 * s + half, a.D, i < nq);
      const Tx8 x = __builtin_bit_cast(Tx8, g[s]), y = __builtin_bit_cast(Tx8, load8(o, 2 * s + half, a.D, i < nq));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        delta = __builtin_fmaf((float)x[e], (float)y[e], delta);
        if constexpr (kLift) norm = __builtin_fmaf((float)x[e], (float)x[e], norm);
      }
    }
    delta += __shfl_xor(delta, 32);
    if (row < rows) {
      const int64_t at = ((int64_t)b * a.Hq + hq) * a.Lq + i;
      // a row without keys: every probability 2^(x - inf) = 0
      if (sees > 0) lse = a.lse[at] * kLog2e;
      if (lse == -kInf) lse = kInf;
    }
  }
  float up = 1.0f, down = 1.0f;   // powers of two
  if constexpr (kLift) {
    norm = __builtin_sqrtf(norm + __shfl_xor(norm, 32));
    const int parts = (a.Lk + 255) / 256;
    const int k = lift_of(norm * max_of(a.vmax + ((int64_t)b * a.Hk + hk) * parts, (nk + 255) / 256));
    up = __builtin_ldexpf(1.0f, k), down = __builtin_ldexpf(1.0f, -k);
    float top = norm;
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (l == 0) a.gmax[(((int64_t)b * a.Hk + hk) * tiles + tile) * 4 + threadIdx.x / 64] = top;
  }
  f32x16 o[DB] = {};
  float left = 0.0f;
  Staged<KS> nextK, nextV;
  // The score gradients of a row add up to 0: what their sum leaves over is delta's error, the
  // rounding of `out`.  The other kernel gets the corrected delta.  Here it matters where few
  // keys share a row, and there (one tile) a first pass finds it.
  for (int pass = most > 64; pass < 2; ++pass) {
    left = 0.0f;
    if (most > 0) {
      fetch(nextK, kb, 2 * a.ks[1], 0, nk, a.D);
      fetch(nextV, vb, 2 * a.vs[1], 0, nk, a.D);
    }
    for (int j0 = 0, buf = 0; j0 < most; j0 += 64, buf ^= 1) {
      put<KS, CH>(sK[buf], nextK);
      put<KS, CH>(sV[buf], nextV);
      __syncthreads();
      if (j0 + 64 < most) {
        fetch(nextK, kb, 2 * a.ks[1], j0 + 64, nk, a.D);
        fetch(nextV, vb, 2 * a.vs[1], j0 + 64, nk, a.D);
      }
      const bool whole = __all(j0 + 64 <= sees);
      const float shift = delta * up;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x16 x = {}, dp = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) x = mma<T>(read_rows<CH>(sK[buf], 32 * u, s), q[s], x);
#pragma unroll
        for (int s = 0; s < KS; ++s) dp = mma<T>(read_rows<CH>(sV[buf], 32 * u, s), g[s], dp);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.c, -lse)) * __builtin_fmaf(dp[r], up, -shift);
        if (!whole) {   // by choice, not by a product with 0: dp may be anything there
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (j0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4 >= sees) x[r] = 0.0f;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) left += x[r];
        if (pass == 0) continue;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const s16x8 ds = round8<T>(x, t);
#pragma unroll
          for (int d = 0; d < DB; ++d) o[d] = mma<T>(read_cols<CH>(sK[buf], 32 * u + 16 * t, 32 * d), ds, o[d]);
        }
      }
    }
    left += __shfl_xor(left, 32);
    delta = __builtin_fmaf(left, down, delta);
    __syncthreads();   // the next pass begins with the first buffer again
  }
  if (row < rows && half == 0) a.delta[((int64_t)b * a.Hq + hq) * a.Lq + i] = delta;
  if (row >= rows) return;
  char* out = a.dq + 2 * (b * a.dqs[0] + i * a.dqs[1] + hq * a.dqs[2]);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int at = 32 * d + 8 * (r / 4) + 4 * half;
      if (at < a.D) store4<T>(out, at, a.D, o[d], r, a.scale * down);
    }
}

// ---- backward, dk and dv ----------------------------------------------------------------------
//
// A workgroup takes 128 keys of one (sample, key head), 32 a wave, and walks the rows in tiles
// of 64: x = Q K^T (lane: one key, 16 rows), dv^T += dout^T p, dk^T += Q^T ds.  No sums are
// shared between workgroups, so there is nothing to add atomically.
template <typename T, int KS>
__global__ __launch_bounds__(256, 2) void k_attn_dkv(AttnArgs a) {
  constexpr int CH = kChunks<KS>, DB = (KS + 1) / 2;
  __shared__ __attribute__((aligned(16))) short sQ[2][64 * CH * 8], sG[2][64 * CH * 8];
  __shared__ __attribute__((aligned(16))) float sLse[2][64], sDelta[2][64];
  const int tiles = (a.Lk + 127) / 128;
  int id = blockIdx.x;
  const int tile = id % tiles;   // the keys that most rows see first
  id /= tiles;
  const int hk = id % a.Hk, b = id / a.Hk;
  const int nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk);
  const int l = threadIdx.x % 64, half = l / 32, key0 = tile * 128 + (threadIdx.x / 64) * 32;
  const int key = key0 + l % 32;
  const int rows = nq * a.share;
  // the first row that sees key j
  auto first_of = [&](int j) { return a.causal ? max(0, j - (nk - nq)) * a.share : 0; };
  const int first = first_of(key), begin = tile * 128 < nk ? first_of(tile * 128) / 64 * 64 : rows;
  const char* qb = a.q + 2 * (b * a.qs[0] + (int64_t)hk * a.share * a.qs[2]);
  const char* gb = a.dout + 2 * (b * a.dos[0] + (int64_t)hk * a.share * a.dos[2]);
  const int64_t lse0 = ((int64_t)b * a.Hq + hk * a.share) * a.Lq;

  s16x8 k[KS], v[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int64_t j = key < nk ? key : 0;
    k[s] = load8(a.k + 2 * (b * a.ks[0] + j * a.ks[1] + hk * a.ks[2]), 2 * s + half, a.D, key < nk);
    v[s] = load8(a.v + 2 * (b * a.vs[0] + j * a.vs[1] + hk * a.vs[2]), 2 * s + half, a.D, key < nk);
  }
  f32x16 dk[DB] = {}, dv[DB] = {};

  float up = 1.0f, down = 1.0f;   // of score gradients, beyond kUp
  if constexpr (__is_same(T, f16)) {
    const int parts = (a.Lk + 255) / 256, gparts = (a.Lq * a.share + 127) / 128 * 4;
    const int lift = lift_of(max_of(a.gmax + ((int64_t)b * a.Hk + hk) * gparts, gparts) *
                             max_of(a.vmax + ((int64_t)b * a.Hk + hk) * parts, (nk + 255) / 256));
    up = __builtin_ldexpf(1.0f, lift - (int)kUp<T>), down = __builtin_ldexpf(1.0f, -lift);
  }
  Staged<KS> nextQ, nextG;
  float nextL = kInf, nextD = 0.0f;
  auto fetch_all = [&](int r0) {
    fetch_group(nextQ, qb, 2 * a.qs[1], 2 * a.qs[2], a.share, r0, rows, a.D);
    fetch_group(nextG, gb, 2 * a.dos[1], 2 * a.dos[2], a.share, r0, rows, a.D);
    const int r = r0 + threadIdx.x;
    if (threadIdx.x < 64) {
      nextL = kInf, nextD = 0.0f;
      if (r < rows) {
        const int x = r / a.share;
        const int64_t at = lse0 + (int64_t)(r - x * a.share) * a.Lq + x;
        nextL = a.lse[at] * kLog2e - kUp<T>, nextD = a.delta[at] * up;
        if (nextL == -kInf) nextL = kInf;
      }
    }
  };
  if (begin < rows) fetch_all(begin);
  for (int r0 = begin, buf = 0; r0 < rows; r0 += 64, buf ^= 1) {
    put<KS, CH>(sQ[buf], nextQ);
    put<KS, CH>(sG[buf], nextG);
    if (threadIdx.x < 64) sLse[buf][threadIdx.x] = nextL, sDelta[buf][threadIdx.x] = nextD;
    __syncthreads();
    if (r0 + 64 < rows) fetch_all(r0 + 64);
    const bool whole = __all(r0 >= first);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x16 x = {}, dp = {};
#pragma unroll
      for (int s = 0; s < KS; ++s) x = mma<T>(read_rows<CH>(sQ[buf], 32 * u, s), k[s], x);
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 lse = *(const f32x4*)&sLse[buf][32 * u + 2 * r + 4 * half];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[r + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r + e], a.c, -lse[e]));
      }
      if (!whole) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (r0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4 < first) x[r] = 0.0f;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const s16x8 p = round8<T>(x, t);
#pragma unroll
        for (int d = 0; d < DB; ++d) dv[d] = mma<T>(read_cols<CH>(sG[buf], 32 * u + 16 * t, 32 * d), p, dv[d]);
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) dp = mma<T>(read_rows<CH>(sG[buf], 32 * u, s), v[s], dp);
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 delta = *(const f32x4*)&sDelta[buf][32 * u + 2 * r + 4 * half];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[r + e] *= __builtin_fmaf(dp[r + e], up, -delta[e]);
      }
      if (!whole) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (r0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4 < first) x[r] = 0.0f;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const s16x8 ds = round8<T>(x, t);
#pragma unroll
        for (int d = 0; d < DB; ++d) dk[d] = mma<T>(read_cols<CH>(sQ[buf], 32 * u + 16 * t, 32 * d), ds, dk[d]);
      }
    }
  }
  if (key >= a.Lk) return;
  char* ok = a.dk + 2 * (b * a.dks[0] + key * a.dks[1] + hk * a.dks[2]);
  char* ov = a.dv + 2 * (b * a.dvs[0] + key * a.dvs[1] + hk * a.dvs[2]);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (key >= nk) dk[d][r] = dv[d][r] = 0.0f;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int at = 32 * d + 8 * (r / 4) + 4 * half;
      if (at < a.D) {
        store4<T>(ok, at, a.D, dk[d], r, a.scale * down);
        store4<T>(ov, at, a.D, dv[d], r, kUp<T> == 0.0f ? 1.0f : 1.0f / 256.0f);
      }
    }
}

// ---- host ---------------------------------------------------------------------------------------

gbmw_status check_sizes(const gbmw_attention_problem* p) {
  if (!p) return fail(GBMW_ERR_INVALID_ARG, "null problem");
  if (p->dtype != GBMW_F16 && p->dtype != GBMW_BF16)
    return fail(p->dtype == GBMW_F32 ? GBMW_ERR_UNSUPPORTED : GBMW_ERR_INVALID_ARG,
                "dtype=%d: attention takes GBMW_F16 and GBMW_BF16", p->dtype);
  if (p->B < 0 || p->Lq < 0 || p->Lk < 0) return fail(GBMW_ERR_INVALID_ARG, "negative size");
  if (p->Hq < 1 || p->Hk < 1 || p->Hq % p->Hk)
    return fail(GBMW_ERR_INVALID_ARG, "Hq=%d is not a multiple of Hk=%d", p->Hq, p->Hk);
  if (p->D < 1 || p->D > 128) return fail(GBMW_ERR_INVALID_ARG, "D=%d not in 1..128", p->D);
  const int64_t rows = (int64_t)p->Lq * (p->Hq / p->Hk);
  if (rows > INT_MAX - 256 || p->Lk > INT_MAX - 256) return fail(GBMW_ERR_INVALID_ARG, "too many rows");
  const int64_t groups = std::max((rows + 127) / 128, ((int64_t)p->Lk + 127) / 128) * p->Hk;
  if (groups > INT_MAX || groups * p->B > INT_MAX) return fail(GBMW_ERR_INVALID_ARG, "too many rows in all");
  if (p->causal != 0 && p->causal != 1) return fail(GBMW_ERR_INVALID_ARG, "causal=%d", p->causal);
  if (!(p->scale >= 0.0f) || !std::isfinite(p->scale)) return fail(GBMW_ERR_INVALID_ARG, "scale=%g", (double)p->scale);
  return GBMW_OK;
}

gbmw_status check_array(const char* name, const void* ptr, const int64_t* stride, int L, bool written,
                        const gbmw_attention_problem* p, int H) {
  if (L == 0 || p->B == 0) return GBMW_OK;
  if (!ptr) return fail(GBMW_ERR_INVALID_ARG, "%s is null", name);
  if ((uintptr_t)ptr % 2) return fail(GBMW_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
  const int64_t extent[3] = {p->B, L, H};
  for (int i = 0; i < 3; ++i) {
    if (stride[i] < 0 || stride[i] > (1ll << 40)) return fail(GBMW_ERR_INVALID_ARG, "%s: stride %lld", name, (long long)stride[i]);
    if (written && extent[i] > 1 && stride[i] < p->D)
      return fail(GBMW_ERR_INVALID_ARG, "%s: stride %lld lets rows overlap", name, (long long)stride[i]);
  }
  return GBMW_OK;
}

gbmw_status check_common(const gbmw_attention_problem* p, bool backward) {
  gbmw_status st = check_sizes(p);
  if (st == GBMW_OK) st = check_array("q", p->q, p->q_stride, p->Lq, false, p, p->Hq);
  if (st == GBMW_OK) st = check_array("k", p->k, p->k_stride, p->Lk, false, p, p->Hk);
  if (st == GBMW_OK) st = check_array("v", p->v, p->v_stride, p->Lk, false, p, p->Hk);
  if (st == GBMW_OK) st = check_array("out", p->out, p->out_stride, p->Lq, !backward, p, p->Hq);
  if (st != GBMW_OK) return st;
  if (p->B && p->Lq && (!p->lse || (uintptr_t)p->lse % 4)) return fail(GBMW_ERR_INVALID_ARG, "lse is null or not aligned");
  if ((uintptr_t)p->len_q % 4 || (uintptr_t)p->len_k % 4) return fail(GBMW_ERR_INVALID_ARG, "len_q or len_k is not aligned");
  return GBMW_OK;
}

AttnArgs args_of(const gbmw_attention_problem* p) {
  AttnArgs a{};
  a.q = (const char*)p->q, a.k = (const char*)p->k, a.v = (const char*)p->v, a.dout = (const char*)p->dout;
  a.out = (char*)p->out, a.dq = (char*)p->dq, a.dk = (char*)p->dk, a.dv = (char*)p->dv;
  a.lse = p->lse;
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p->q_stride[i], a.ks[i] = p->k_stride[i], a.vs[i] = p->v_stride[i], a.os[i] = p->out_stride[i];
    a.dos[i] = p->dout_stride[i], a.dqs[i] = p->dq_stride[i], a.dks[i] = p->dk_stride[i], a.dvs[i] = p->dv_stride[i];
  }
  a.len_q = p->len_q, a.len_k = p->len_k;
  a.B = p->B, a.Hq = p->Hq, a.Hk = p->Hk, a.Lq = p->Lq, a.Lk = p->Lk, a.D = p->D, a.share = p->Hq / p->Hk;
  a.causal = p->causal, a.scale = p->scale;
  // not 0: a hidden key's -inf has to stay -inf when it is scaled
  a.c = std::max(p->scale * kLog2e, 1e-30f);
  return a;
}

// delta [B][Hq][Lq], and for float16 gmax [B][Hk][tiles][4] and vmax [B][Hk][parts]
struct Scratch {
  int64_t delta, gmax, vmax;   // floats
  int64_t bytes() const { return 4 * (delta + gmax + vmax); }
};
Scratch scratch_of(const gbmw_attention_problem* p) {
  const int64_t groups = (int64_t)p->B * p->Hk, rows = (int64_t)p->Lq * (p->Hq / p->Hk);
  const bool lift = p->dtype == GBMW_F16;
  return {groups * rows, lift ? groups * ((rows + 127) / 128) * 4 : 0, lift ? groups * (((int64_t)p->Lk + 255) / 256) : 0};
}

template <typename T, int KS>
void launch(const AttnArgs& a, bool backward, hipStream_t st) {
  const int64_t rows = (int64_t)a.Lq * a.share;
  const dim3 grid_q((unsigned)((rows + 127) / 128 * a.Hk * a.B)), grid_k((unsigned)(((int64_t)a.Lk + 127) / 128 * a.Hk * a.B));
  if (!backward) {
    hipLaunchKernelGGL((k_attn_fwd<T, KS>), grid_q, dim3(256), 0, st, a);
    return;
  }
  if constexpr (__is_same(T, f16))
    if (a.Lk) hipLaunchKernelGGL(k_attn_vmax, dim3((unsigned)(((int64_t)a.Lk + 255) / 256 * a.Hk * a.B)), dim3(256), 0, st, a);
  if (grid_q.x) hipLaunchKernelGGL((k_attn_dq<T, KS>), grid_q, dim3(256), 0, st, a);
  if (grid_k.x) hipLaunchKernelGGL((k_attn_dkv<T, KS>), grid_k, dim3(256), 0, st, a);
}

template <typename T>
void launch(const AttnArgs& a, bool backward, hipStream_t st) {
  if (a.D <= 32) launch<T, 2>(a, backward, st);
  else if (a.D <= 64) launch<T, 4>(a, backward, st);
  else if (a.D <= 80) launch<T, 5>(a, backward, st);
  else if (a.D <= 96) launch<T, 6>(a, backward, st);
  else launch<T, 8>(a, backward, st);
}

}  // namespace
}  // namespace gbmw

using namespace gbmw;

extern "C" int64_t gbmw_attention_workspace(const gbmw_attention_problem* p, int32_t backward) {
  gbmw_detail::clear_error();
  if (check_sizes(p) != GBMW_OK) return -1;
  return backward ? scratch_of(p).bytes() : 0;
}

extern "C" gbmw_status gbmw_attention_forward(const gbmw_attention_problem* p) {
  gbmw_detail::clear_error();
  const gbmw_status st = check_common(p, false);
  if (st != GBMW_OK) return st;
  if (p->B == 0 || p->Lq == 0) return GBMW_OK;
  const AttnArgs a = args_of(p);
  if (p->dtype == GBMW_F16) launch<f16>(a, false, (hipStream_t)p->stream);
  else launch<bf16>(a, false, (hipStream_t)p->stream);
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

extern "C" gbmw_status gbmw_attention_backward(const gbmw_attention_problem* p) {
  gbmw_detail::clear_error();
  gbmw_status st = check_common(p, true);
  if (st == GBMW_OK) st = check_array("dout", p->dout, p->dout_stride, p->Lq, false, p, p->Hq);
  if (st == GBMW_OK) st = check_array("dq", p->dq, p->dq_stride, p->Lq, true, p, p->Hq);
  if (st == GBMW_OK) st = check_array("dk", p->dk, p->dk_stride, p->Lk, true, p, p->Hk);
  if (st == GBMW_OK) st = check_array("dv", p->dv, p->dv_stride, p->Lk, true, p, p->Hk);
  if (st != GBMW_OK) return st;
  if (p->B == 0 || (p->Lq == 0 && p->Lk == 0)) return GBMW_OK;
  const Scratch sc = scratch_of(p);
  const int64_t need = sc.bytes();
  if (need && (!p->workspace || p->workspace_bytes < need || (uintptr_t)p->workspace % 16))
    return fail(GBMW_ERR_INVALID_ARG, "workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
  AttnArgs a = args_of(p);
  a.delta = (float*)p->workspace, a.gmax = a.delta + sc.delta, a.vmax = a.gmax + sc.gmax;
  if (p->dtype == GBMW_F16) launch<f16>(a, true, (hipStream_t)p->stream);
  else launch<bf16>(a, true, (hipStream_t)p->stream);
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}
