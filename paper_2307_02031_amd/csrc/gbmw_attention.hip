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

#ifndef GBMW_FILL
#define GBMW_FILL 1024
#define GBMW_LEAST 512
#endif
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
  float *lse;
  float *level, *delta;   // [B][Hk][rows]: log2(e) lse - kUp, inf for rows without keys; <dout, out>
  float *vmax, *gmax;   // f16: the largest norms of a value and of a row of dout, for parts of 256 keys and 128 rows
  int64_t qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];
  const int *len_q, *len_k;
  float* partial;   // [parts][2][B][Hk][Lk][D4]: shares of dk and dv
  int B, Hq, Hk, Lq, Lk, D, share, causal;
  int parts, D4;    // D rounded up to 4
  int near;         // heads that a die works on at a time
  unsigned magic;   // 2^32 / share, rounded up
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

// ---- tiles in LDS ---------------------------------------------------------------------------
//
// A tile is 64 rows of CH 16-byte pieces, stored so that the two kinds of reads, a piece of
// each of 32 rows and (transposing) 64 bytes of each of four rows, touch all 64 banks evenly:
// piece p of row r lies at place p ^ swap_of(r) of its row, and rows of 16 pieces have 16 bytes
// between groups of four.  A lane then needs four addresses for each kind (Reader);
// everything else is a constant offset.
typedef __attribute__((address_space(3))) char lds_char;

template <int KS>
constexpr int kChunks = KS <= 4 ? 8 : 16;
template <int CH>
__device__ __forceinline__ constexpr int swap_of(int row) {
  return CH == 16 ? (row & 3) << 2 : ((row & 2) << 1) | ((row >> 2) & 3);
}
template <int CH>
__device__ __forceinline__ constexpr int place_of(int row, int piece) {   // bytes
  return (row * CH + (piece ^ swap_of<CH>(row))) * 16 + (CH == 16 ? row / 4 * 16 : 0);
}
template <int KS>
constexpr int kTile = 64 * 16 * kChunks<KS> + (kChunks<KS> == 16 ? 256 : 0);   // bytes

template <int KS>
struct Reader {
  static constexpr int CH = kChunks<KS>;
  int row[4], col[4];
  __device__ __forceinline__ Reader() {
    const int l = threadIdx.x % 64, i = l % 16, half = l / 32;
#pragma unroll
    for (int s = 0; s < 4; ++s) row[s] = place_of<CH>(l % 32, (CH == 16 ? 4 * s : 2 * s) + half);
    // lanes 4u..4u+3 of sixteen name the quarters of run u of sixteen elements; lane i gets
    // element i of each of the four runs
    const int r = 4 * half + i / 4, c = 16 * ((l / 16) % 2) + 4 * (i % 4);
#pragma unroll
    for (int n = 0; n < 4; ++n)   // of 32 columns each, or of two times 32 columns eight rows apart
      col[n] = (CH == 16 ? place_of<CH>(r, 4 * n + c / 8) : place_of<CH>(r + 8 * (n / 2), 4 * (n % 2) + c / 8)) + (c % 8) * 2;
  }
  static constexpr int down(int r) { return r * CH * 16 + (CH == 16 ? r / 4 * 16 : 0); }   // r a multiple of 16, or of 8 for CH = 16
  // A operand: rows r .. r+31 of the tile (r = 0 or 32), terms 16 step .. 16 step + 15
  __device__ __forceinline__ s16x8 rows(lds_char* tile, int r, int step) const {
    typedef __attribute__((address_space(3))) s16x8 lds8;
    return *(lds8*)(tile + (CH == 16 ? row[step / 2] + (step % 2) * 32 : row[step]) + down(r));
  }
  // A operand: rows = columns 32 d .. 32 d + 31 of the tile, terms = its rows r .. r+15 in the
  // order of a result's registers
  __device__ __forceinline__ s16x8 cols(lds_char* tile, int r, int d) const {
    typedef __attribute__((address_space(3))) s16x4 lds4;
    s16x4 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
      x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(tile + (CH == 16 ? col[d] + down(r + 8 * u) : col[d + 2 * u] + down(r))));
    return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// A piece of a row in global memory; zeros beyond D and where the row is not there.  WHOLE: D is
// a multiple of 8.
template <bool WHOLE>
__device__ __forceinline__ s16x8 load8(const char* row, int piece, int D, bool there) {
  if constexpr (WHOLE) {
    s16x8 r = {};
    if (there && 8 * piece < D) __builtin_memcpy(&r, row + 16 * piece, 16);
    return r;
  } else {
    const Pack<bf16> r = load_pack((const bf16*)row + 8 * piece, there ? D - 8 * piece : 0);
    return __builtin_bit_cast(s16x8, r);
  }
}

// Rows of a group of `share` heads: row r is at base + (r / share) * stride + (r % share) * head.
struct Rows {
  const char* base;
  int64_t stride, head;   // bytes
  int share, count;       // rows beyond count read as zeros
  unsigned magic;         // 2^32 / share, rounded up
  __device__ __forceinline__ int of(int r) const {   // r / share
    if (share == 1) return r;
    int x = (int)__umulhi((unsigned)r, magic);   // at most one too large for r < 2^31
    return x * share > r ? x - 1 : x;
  }
};

// Brings 64 rows into a tile, in two halves: begin() before the tile before it is worked on,
// end() before the barrier that hands it over.
//
// Direct: the loads write to LDS themselves, 64 pieces in lane order; lanes fetch the pieces
// that belong in their places, and what is beyond the buffer's bounds arrives as zeros.  Needs
// 16-byte aligned rows and offsets inside a tile below 2^31.  Otherwise through registers.
//
// A wave brings N runs of kRowsOf rows.  Its lanes' offsets inside a run are the same for all of
// them where rows have 16 pieces; with SPARE every run gets bounds of its own and the lanes keep
// one offset, otherwise N (for the kernel that is short of registers, and those that are not).
template <int KS, bool DIRECT, bool SPARE = false>
struct Loader {
  static constexpr int CH = kChunks<KS>, N = DIRECT ? CH / 4 : (64 * 2 * KS + 255) / 256;
  static constexpr int kRowsOf = 64 / CH;
  static constexpr bool kOne = SPARE && CH == 16;
  static constexpr int NA = kOne ? 1 : N;
  static constexpr unsigned kOut = 0x80000000u;
  s16x8 x[DIRECT ? 1 : N];
  unsigned at[DIRECT ? NA : 1];

  __device__ __forceinline__ static int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }
  __device__ __forceinline__ static int row_of(int i) {   // of this lane, in the tile
    return (wave() * N + i) * kRowsOf + (int)(threadIdx.x % 64) / CH;
  }
  __device__ __forceinline__ void init(const Rows& rows, int D) {
    if constexpr (DIRECT) {
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int piece = ((int)threadIdx.x % CH) ^ swap_of<CH>(row_of(i));
        const int down = kOne ? (int)(threadIdx.x % 64) / CH : row_of(i);
        at[i] = 8 * piece >= D ? kOut : 16 * piece + (rows.share == 1 ? down * (unsigned)rows.stride : 0u);
      }
    }
  }

  __device__ __forceinline__ void begin(lds_char* tile, const Rows& rows, int first, int D) {
    if constexpr (DIRECT) {
      if (rows.share == 1) {   // rows beyond the last one are beyond the bounds
        const int64_t length = (int64_t)(rows.count - first) * rows.stride;
        const int left = (int)min(length, (int64_t)0x7fffffff), run = kRowsOf * (int)rows.stride;
        const char* base = rows.base + first * rows.stride;
        const int skip = kOne ? wave() * N * run : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int off = kOne ? skip + i * run : 0;
          load(tile, __builtin_amdgcn_make_buffer_rsrc((void*)(base + off), 0, max(left - off, 0), 0x00020000), i, at[i % NA]);
        }
      } else {
        const int x0 = rows.of(first);
        __amdgpu_buffer_rsrc_t from =
            __builtin_amdgcn_make_buffer_rsrc((void*)(rows.base + x0 * rows.stride), 0, 0x7fffffff, 0x00020000);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = first + row_of(i), x = rows.of(r);
          load(tile, from, i, (r >= rows.count) | (at[i % NA] == kOut) ? kOut
                                  : at[i % NA] + (unsigned)(x - x0) * (unsigned)rows.stride + (unsigned)(r - x * rows.share) * (unsigned)rows.head);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + 256 * i, r = first + n / (2 * KS);
        const bool there = n < 64 * 2 * KS && r < rows.count;
        const int q = there ? r : first, h = rows.of(q);
        x[i] = load8<false>(rows.base + h * rows.stride + (q - h * rows.share) * rows.head, n % (2 * KS), D, there);
      }
    }
  }
  __device__ __forceinline__ static void load(lds_char* tile, __amdgpu_buffer_rsrc_t from, int i, unsigned offset) {
    lds_char* to = tile + (wave() * N + i) * (CH == 16 ? 1040 : 1024);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, (int)offset, 0, 0, 0);
  }
  __device__ __forceinline__ void end(lds_char* tile) {
    if constexpr (DIRECT) {
      __builtin_amdgcn_s_waitcnt(0x0f70);   // all of this wave's loads have arrived
    } else {
      typedef __attribute__((address_space(3))) s16x8 lds8;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + 256 * i, r = n / (2 * KS);
        if (r < 64) *(lds8*)(tile + place_of<CH>(r, n % (2 * KS))) = x[i];
      }
    }
  }
};

__device__ __forceinline__ int length(const int* len, int b, int most) {
  return len ? max(0, min(len[b], most)) : most;
}

__device__ __forceinline__ float max3(float a, float b, float c) {   // without quieting NaNs first
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

__device__ __forceinline__ float other_half(float x, float* mine) {   // of lane l ^ 32; both sorted by half
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  *mine = __builtin_bit_cast(float, (unsigned)r[0]);
  return __builtin_bit_cast(float, (unsigned)r[1]);
}

// A row of the result of a product over d: lane l has column (row of the problem) l % 32 and
// the d of its registers, four at a time.
template <typename T, bool WHOLE>
__device__ __forceinline__ void store4(char* row, int d, int D, const f32x16& x, int r, float f) {
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  Tx4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float z = x[r + i] * f;
    asm("" : "+v"(z));   // the product is rounded to 32 bits first, in every variant of a kernel
    y[i] = (T)z;
  }
  T* p = (T*)row + d;
  if (WHOLE || d + 4 <= D) {
    __builtin_memcpy(p, &y, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < D) p[i] = y[i];
  }
}

// Which head and which of its `units` pieces of work a workgroup takes.  Workgroups are dealt to
// the eight dies in turn.  A die works on its own heads, `near` of them at a time, so that what
// their units read alike stays in its cache; of those the first units (the longest under a
// causal mask) come first.  Heads that eight does not divide are dealt to all dies at the end.
struct Deal {
  int head, unit;
  __device__ __forceinline__ Deal(int heads, int units, int near) {
    const int per = heads / 8, id = blockIdx.x;
    near = min(near, max(per, 1));
    if (id < 8 * per * units) {
      const int at = id / 8, first = at / (near * units) * near, n = min(near, per - first);
      unit = (at - first * units) / n;
      head = id % 8 * per + first + (at - first * units) % n;
    } else {
      const int n = heads - 8 * per, at = id - 8 * per * units;
      unit = at / n;
      head = 8 * per + at % n;
    }
  }
};

// Where a workgroup of the rows' kernels works, and how many keys a row sees.
struct Place {
  int tile, tiles, hk, b, nq, nk, rows;
  __device__ __forceinline__ Place(const AttnArgs& a, int per) {
    rows = a.Lq * a.share;
    tiles = (rows + per - 1) / per;
    const Deal d(a.Hk * a.B, tiles, a.near);
    tile = tiles - 1 - d.unit;   // the longest rows of a causal mask first
    hk = d.head % a.Hk, b = d.head / a.Hk;
    nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk);
  }
  __device__ __forceinline__ int sees(const AttnArgs& a, int i) const {   // keys j < sees
    return i >= nq ? 0 : a.causal ? max(0, min(nk, i + nk - nq + 1)) : nk;
  }
  __device__ __forceinline__ int most(const AttnArgs& a, int per) const {   // of any row of the tile
    const int first = tile * per / a.share, last = min((min(tile * per + per, rows) - 1) / a.share, nq - 1);
    return first >= nq ? 0 : sees(a, last);
  }
};

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

// ---- forward --------------------------------------------------------------------------------
//
// A workgroup takes 128 NQ rows of one (sample, key head), 32 NQ a wave, and walks the keys in
// tiles of 64.  A wave computes x^T = K Q^T (lane: one row, 32 keys), so the running maximum
// and sum of a row need one exchange between two lanes a tile, and out^T += V^T p^T with p from
// its own registers.  The running sums are in units of 2^(c m); m follows the maximum only
// when that is more than 2^kLag ahead, so they are seldom rescaled.
constexpr float kLag = 6.0f;

template <typename T, int KS, int NQ, bool DIRECT>
__global__ __launch_bounds__(256, NQ == 1 ? 2 : 1) void k_attn_fwd(AttnArgs a) {
  constexpr int DB = (KS + 1) / 2;
  __shared__ __attribute__((aligned(16))) char lds[4 * kTile<KS>];
  lds_char* const tiles = (lds_char*)lds;
  const Place w(a, 128 * NQ);
  const int l = threadIdx.x % 64, half = l / 32;
  const int most = w.most(a, 128 * NQ);
  const Rows kr{a.k + 2 * (w.b * a.ks[0] + w.hk * a.ks[2]), 2 * a.ks[1], 0, 1, w.nk, 0};
  const Rows vr{a.v + 2 * (w.b * a.vs[0] + w.hk * a.vs[2]), 2 * a.vs[1], 0, 1, w.nk, 0};

  s16x8 q[NQ][KS];
  int sees[NQ];
  int fewest = INT_MAX, furthest = 0;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = w.tile * 128 * NQ + ((int)(threadIdx.x / 64) * NQ + n) * 32 + l % 32;
    const int i = row / a.share, hq = w.hk * a.share + row % a.share;
    sees[n] = w.sees(a, i);
    fewest = min(fewest, sees[n]), furthest = max(furthest, sees[n]);
    const char* p = a.q + 2 * (w.b * a.qs[0] + (i < w.nq ? i : 0) * a.qs[1] + hq * a.qs[2]);
#pragma unroll
    for (int s = 0; s < KS; ++s) q[n][s] = load8<DIRECT>(p, 2 * s + half, a.D, i < w.nq);
  }
  f32x16 o[NQ][DB] = {};
  float m[NQ], sum[NQ];   // m in units of x / scale
#pragma unroll
  for (int n = 0; n < NQ; ++n) m[n] = -kInf, sum[n] = 0.0f;

  const Reader<KS> rd;
  Loader<KS, DIRECT> lk, lv;
  lk.init(kr, a.D), lv.init(vr, a.D);
  if (most > 0) {
    lk.begin(tiles, kr, 0, a.D);
    lv.begin(tiles + kTile<KS>, vr, 0, a.D);
  }
  for (int j0 = 0, buf = 0; j0 < most; j0 += 64, buf ^= 1) {
    lds_char *tk = tiles + 2 * buf * kTile<KS>, *tv = tk + kTile<KS>;
    lk.end(tk), lv.end(tv);
    __syncthreads();   // this tile is whole, and nobody reads the other buffer any more
    if (j0 + 64 < most) {
      lds_char* to = tiles + 2 * (buf ^ 1) * kTile<KS>;
      lk.begin(to, kr, j0 + 64, a.D);
      lv.begin(to + kTile<KS>, vr, j0 + 64, a.D);
    }
    if (!__any(j0 < furthest)) continue;   // none of the wave's rows sees this tile
    f32x16 x[NQ][2] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const s16x8 k = rd.rows(tk, 32 * u, s);
#pragma unroll
        for (int n = 0; n < NQ; ++n) x[n][u] = mma<T>(k, q[n][s], x[n][u]);
      }
    if (!__all(j0 + 64 <= fewest)) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (j0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4 >= sees[n]) x[n][u][r] = -kInf;
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      // the matrix results are waited for where the compiler sees them read, before max3
      float top = fmaxf(fmaxf(m[n], x[n][0][15]), x[n][1][15]);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; r += 2) top = max3(top, x[n][u][r], x[n][u][r + 1]);
      float low;
      const float high = other_half(top, &low);
      top = fmaxf(low, high);
      const bool ahead = (top - m[n]) * a.c > kLag;
      if (__any(ahead)) {
        const float f = ahead ? __builtin_amdgcn_exp2f((m[n] - top) * a.c) : 1.0f;
        if (ahead) m[n] = top;
        sum[n] *= f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[n][d][r] *= f;
      }
      const float off = (m[n] == -kInf ? 0.0f : m[n] * a.c) - kUp<T>;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          x[n][u][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][u][r], a.c, -off));
          sum[n] += x[n][u][r];
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s16x8 p[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) p[n] = round8<T>(x[n][u], t);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const s16x8 v = rd.cols(tv, 32 * u + 16 * t, d);
#pragma unroll
          for (int n = 0; n < NQ; ++n) o[n][d] = mma<T>(v, p[n], o[n][d]);
        }
      }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = w.tile * 128 * NQ + ((int)(threadIdx.x / 64) * NQ + n) * 32 + l % 32;
    const int i = row / a.share, hq = w.hk * a.share + row % a.share;
    sum[n] += __shfl_xor(sum[n], 32);
    if (row >= w.rows) continue;
    const bool empty = m[n] == -kInf && !(sum[n] != sum[n]);
    const float f = empty ? 0.0f : 1.0f / sum[n];
    if (half == 0)
      a.lse[((int64_t)w.b * a.Hq + hq) * a.Lq + i] =
          empty ? -kInf : (m[n] * a.c - kUp<T> + __builtin_amdgcn_logf(sum[n])) * kLn2;
    char* out = a.out + 2 * (w.b * a.os[0] + i * a.os[1] + hq * a.os[2]);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int at = 32 * d + 8 * (r / 4) + 4 * half;
        if (at < a.D) store4<T, DIRECT>(out, at, a.D, o[n][d], r, f);
      }
  }
}

// The largest norm of a value among 256 keys of a (sample, key head), for float16's lift.
__global__ __launch_bounds__(256) void k_attn_vmax(AttnArgs a) {
  __shared__ float tops[4];
  const int parts = (a.Lk + 255) / 256, part = blockIdx.x % parts;
  const int hk = blockIdx.x / parts % a.Hk, b = blockIdx.x / parts / a.Hk;
  // sixteen lanes a row, a piece each
  const int last = min(part * 256 + 256, length(a.len_k, b, a.Lk)), d = threadIdx.x % 16 * 8;
  const f16* v = (const f16*)a.v + b * a.vs[0] + hk * a.vs[2] + d;
  float s = 0.0f;
#pragma unroll 4
  for (int key = part * 256 + threadIdx.x / 16; key < last; key += 16) {
    const Pack<f16> x = load_pack(v + key * a.vs[1], a.D - d);
    float n = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) n = __builtin_fmaf((float)x.v[e], (float)x.v[e], n);
#pragma unroll
    for (int i = 8; i; i >>= 1) n += __shfl_xor(n, i);
    s = fmaxf(s, n);
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
template <typename T, int KS, bool DIRECT>
__global__ __launch_bounds__(256, 2) void k_attn_dq(AttnArgs a) {
  constexpr int DB = (KS + 1) / 2;
  constexpr bool kLift = __is_same(T, f16);
  __shared__ __attribute__((aligned(16))) char lds[4 * kTile<KS>];
  lds_char* const tiles = (lds_char*)lds;
  const Place w(a, 128);
  const int l = threadIdx.x % 64, half = l / 32, row = w.tile * 128 + (threadIdx.x / 64) * 32 + l % 32;
  const int i = row / a.share, hq = w.hk * a.share + row % a.share;
  const int b = w.b, hk = w.hk, nq = w.nq, nk = w.nk, rows = w.rows;
  const int sees = w.sees(a, i), most = w.most(a, 128);
  const Rows kr{a.k + 2 * (b * a.ks[0] + hk * a.ks[2]), 2 * a.ks[1], 0, 1, nk, 0};
  const Rows vr{a.v + 2 * (b * a.vs[0] + hk * a.vs[2]), 2 * a.vs[1], 0, 1, nk, 0};

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
      q[s] = load8<DIRECT>(p, 2 * s + half, a.D, i < nq);
      g[s] = load8<DIRECT>(d, 2 * s + half, a.D, i < nq);
      const Tx8 x = __builtin_bit_cast(Tx8, g[s]), y = __builtin_bit_cast(Tx8, load8<DIRECT>(o, 2 * s + half, a.D, i < nq));
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
    if (l == 0) a.gmax[(((int64_t)b * a.Hk + hk) * w.tiles + w.tile) * 4 + threadIdx.x / 64] = top;
  }
  f32x16 o[DB] = {};
  float left = 0.0f;
  const Reader<KS> rd;
  Loader<KS, DIRECT> lk, lv;
  lk.init(kr, a.D), lv.init(vr, a.D);
  // The score gradients of a row add up to 0: what their sum leaves over is delta's error, the
  // rounding of `out`.  The other kernel gets the corrected delta.  Here it matters where few
  // keys share a row, and there (one tile) a first pass finds it.
  for (int pass = most > 64; pass < 2; ++pass) {
    left = 0.0f;
    if (most > 0) {
      lk.begin(tiles, kr, 0, a.D);
      lv.begin(tiles + kTile<KS>, vr, 0, a.D);
    }
    for (int j0 = 0, buf = 0; j0 < most; j0 += 64, buf ^= 1) {
      lds_char *tk = tiles + 2 * buf * kTile<KS>, *tv = tk + kTile<KS>;
      lk.end(tk), lv.end(tv);
      __syncthreads();
      if (j0 + 64 < most) {
        lds_char* to = tiles + 2 * (buf ^ 1) * kTile<KS>;
        lk.begin(to, kr, j0 + 64, a.D);
        lv.begin(to + kTile<KS>, vr, j0 + 64, a.D);
      }
      if (!__any(j0 < sees)) continue;
      const bool whole = __all(j0 + 64 <= sees);
      const float shift = delta * up;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x16 x = {}, dp = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) x = mma<T>(rd.rows(tk, 32 * u, s), q[s], x);
#pragma unroll
        for (int s = 0; s < KS; ++s) dp = mma<T>(rd.rows(tv, 32 * u, s), g[s], dp);
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
          for (int d = 0; d < DB; ++d) o[d] = mma<T>(rd.cols(tk, 32 * u + 16 * t, d), ds, o[d]);
        }
      }
    }
    left += __shfl_xor(left, 32);
    delta = __builtin_fmaf(left, down, delta);
    __syncthreads();   // the next pass begins with the first buffer again
  }
  if (row < rows && half == 0) {
    const int64_t at = ((int64_t)b * a.Hk + hk) * rows + row;
    a.delta[at] = delta, a.level[at] = lse - kUp<T>;
  }
  if (row >= rows) return;
  char* out = a.dq + 2 * (b * a.dqs[0] + i * a.dqs[1] + hq * a.dqs[2]);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int at = 32 * d + 8 * (r / 4) + 4 * half;
      if (at < a.D) store4<T, DIRECT>(out, at, a.D, o[d], r, a.scale * down);
    }
}

// ---- backward, dk and dv ----------------------------------------------------------------------
//
// A workgroup takes 128 keys of one (sample, key head), 32 a wave, and walks the rows in tiles
// of 64: x = Q K^T (lane: one key, 16 rows), dv^T += dout^T p, dk^T += Q^T ds.  No sums are
// shared between workgroups, so there is nothing to add atomically.
template <typename T, int KS, bool DIRECT>
__global__ __launch_bounds__(256, 2) void k_attn_dkv(AttnArgs a) {
  constexpr int DB = (KS + 1) / 2;
  __shared__ __attribute__((aligned(16))) char lds[4 * kTile<KS>];
  lds_char* const buffers = (lds_char*)lds;
  __shared__ __attribute__((aligned(16))) float sRow[2][2][64];   // level, delta
  const int heads = a.Hk * a.B;
  const Deal deal(heads, (a.Lk + 127) / 128 * a.parts, a.near);
  const int part = deal.unit % a.parts, tile = deal.unit / a.parts;   // the keys that most rows see first
  const int hk = deal.head % a.Hk, b = deal.head / a.Hk;
  const int nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk);
  const int l = threadIdx.x % 64, half = l / 32, key0 = tile * 128 + (threadIdx.x / 64) * 32;
  const int key = key0 + l % 32;
  const int rows = nq * a.share;
  // the first row that sees key j
  auto first_of = [&](int j) { return a.causal ? max(0, j - (nk - nq)) * a.share : 0; };
  const int first = first_of(key);
  // the rows that see a key of the tile, in `parts` runs of whole tiles
  int begin = tile * 128 < nk ? min(first_of(tile * 128) / 64 * 64, rows) : rows;
  const int run = ((rows - begin + 63) / 64 + a.parts - 1) / a.parts * 64;
  begin = min((int64_t)begin + (int64_t)part * run, (int64_t)rows);
  const int end = min((int64_t)begin + run, (int64_t)rows);
  const Rows qr{a.q + 2 * (b * a.qs[0] + (int64_t)hk * a.share * a.qs[2]), 2 * a.qs[1], 2 * a.qs[2], a.share, rows, a.magic};
  const Rows gr{a.dout + 2 * (b * a.dos[0] + (int64_t)hk * a.share * a.dos[2]), 2 * a.dos[1], 2 * a.dos[2], a.share, rows, a.magic};
  const int64_t row0 = ((int64_t)b * a.Hk + hk) * a.Lq * a.share;

  s16x8 k[KS], v[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int64_t j = key < nk ? key : 0;
    k[s] = load8<DIRECT>(a.k + 2 * (b * a.ks[0] + j * a.ks[1] + hk * a.ks[2]), 2 * s + half, a.D, key < nk);
    v[s] = load8<DIRECT>(a.v + 2 * (b * a.vs[0] + j * a.vs[1] + hk * a.vs[2]), 2 * s + half, a.D, key < nk);
  }
  f32x16 dk[DB] = {}, dv[DB] = {};

  float up = 1.0f, down = 1.0f;   // of score gradients, beyond kUp
  if constexpr (__is_same(T, f16)) {
    const int parts = (a.Lk + 255) / 256, gparts = (a.Lq * a.share + 127) / 128 * 4;
    const int lift = lift_of(max_of(a.gmax + ((int64_t)b * a.Hk + hk) * gparts, gparts) *
                             max_of(a.vmax + ((int64_t)b * a.Hk + hk) * parts, (nk + 255) / 256));
    up = __builtin_ldexpf(1.0f, lift - (int)kUp<T>), down = __builtin_ldexpf(1.0f, -lift);
  }
  const Reader<KS> rd;
  Loader<KS, DIRECT, true> lq, lg;
  lq.init(qr, a.D), lg.init(gr, a.D);
  auto begin_all = [&](int buf, int r0) {
    lds_char* to = buffers + 2 * buf * kTile<KS>;
    lq.begin(to, qr, r0, a.D);
    lg.begin(to + kTile<KS>, gr, r0, a.D);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if (wave < 2) {   // zeros beyond the last row: nothing comes of them, q and dout being zero there
      __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(
          (void*)((wave ? a.delta : a.level) + row0 + r0), 0, 4 * min(rows - r0, 64), 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(lds_char*)&sRow[buf][wave][0], 4,
                                               4 * l, 0, 0, 0);
    }
  };
  if (begin < end) begin_all(0, begin);
  for (int r0 = begin, buf = 0; r0 < end; r0 += 64, buf ^= 1) {
    lds_char *tq = buffers + 2 * buf * kTile<KS>, *tg = tq + kTile<KS>;
    lq.end(tq), lg.end(tg);
    if constexpr (!DIRECT) __builtin_amdgcn_s_waitcnt(0x0f70);   // sRow
    __syncthreads();
    if (r0 + 64 < end) begin_all(buf ^ 1, r0 + 64);
    if (!__any(r0 + 64 > first)) continue;   // none of these rows sees a key of the wave
    const bool whole = __all(r0 >= first);
#pragma unroll 1
    for (int u = 0; u < 2; ++u, tq += Reader<KS>::down(32), tg += Reader<KS>::down(32)) {
      f32x16 x = {}, dp = {};
#pragma unroll
      for (int s = 0; s < KS; ++s) x = mma<T>(rd.rows(tq, 0, s), k[s], x);
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 lse = *(const f32x4*)&sRow[buf][0][32 * u + 2 * r + 4 * half];
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
        for (int d = 0; d < DB; ++d) dv[d] = mma<T>(rd.cols(tg, 16 * t, d), p, dv[d]);
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) dp = mma<T>(rd.rows(tg, 0, s), v[s], dp);
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 delta = *(const f32x4*)&sRow[buf][1][32 * u + 2 * r + 4 * half];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[r + e] *= __is_same(T, f16) ? (dp[r + e] - delta[e]) * up : dp[r + e] - delta[e];
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
        for (int d = 0; d < DB; ++d) dk[d] = mma<T>(rd.cols(tq, 16 * t, d), ds, dk[d]);
      }
    }
  }
  if (key >= a.Lk) return;
  const float fk = a.scale * down, fv = kUp<T> == 0.0f ? 1.0f : 1.0f / 256.0f;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (key >= nk) dk[d][r] = dv[d][r] = 0.0f;
  if (a.parts == 1) {
    char* ok = a.dk + 2 * (b * a.dks[0] + key * a.dks[1] + hk * a.dks[2]);
    char* ov = a.dv + 2 * (b * a.dvs[0] + key * a.dvs[1] + hk * a.dvs[2]);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int at = 32 * d + 8 * (r / 4) + 4 * half;
        if (at < a.D) {
          store4<T, DIRECT>(ok, at, a.D, dk[d], r, fk);
          store4<T, DIRECT>(ov, at, a.D, dv[d], r, fv);
        }
      }
  } else {
    const int64_t all = (int64_t)heads * a.Lk * a.D4;
    float* o = a.partial + part * 2 * all + (((int64_t)b * a.Hk + hk) * a.Lk + key) * a.D4;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int at = 32 * d + 8 * (r / 4) + 4 * half;
        if (at < a.D4) {
          *(f32x4*)(o + at) = f32x4{dk[d][r] * fk, dk[d][r + 1] * fk, dk[d][r + 2] * fk, dk[d][r + 3] * fk};
          *(f32x4*)(o + all + at) = f32x4{dv[d][r] * fv, dv[d][r + 1] * fv, dv[d][r + 2] * fv, dv[d][r + 3] * fv};
        }
      }
  }
}

// dk and dv from their shares, four values a thread, in the shares' order.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  const int64_t quads = (int64_t)a.B * a.Hk * a.Lk * (a.D4 / 4);
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= quads) return;
  f32x4 s = {};
  for (int k = 0; k < a.parts; ++k) s += *(const f32x4*)(a.partial + (((int64_t)k * 2 + blockIdx.y) * quads + n) * 4);
  const int d = (int)(n % (a.D4 / 4)) * 4;
  int64_t at = n / (a.D4 / 4);
  const int64_t key = at % a.Lk, hk = at / a.Lk % a.Hk, b = at / a.Lk / a.Hk;
  const int64_t* st = blockIdx.y ? a.dvs : a.dks;
  T* o = (T*)(blockIdx.y ? a.dv : a.dk) + b * st[0] + key * st[1] + hk * st[2] + d;
  const Tx4 y = {(T)s[0], (T)s[1], (T)s[2], (T)s[3]};
  if (d + 4 <= a.D) {
    __builtin_memcpy(o, &y, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < a.D) o[i] = y[i];
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
  a.D4 = (p->D + 3) / 4 * 4, a.parts = 1;
  a.causal = p->causal, a.scale = p->scale;
  a.magic = (unsigned)(((1ull << 32) + a.share - 1) / a.share);
  // Without a causal mask units are alike, and four heads at a time (keys and values of a few MB)
  // suit a die's cache: 5 x 32 heads x 2048 x 128 forward 377 us, all at a time 384.  With one the
  // order of their lengths counts more: 2 x 40 heads, all at a time 113 us, four 125; backward 411, 456.
  a.near = p->causal ? INT_MAX : 4;
  // not 0: a hidden key's -inf has to stay -inf when it is scaled
  a.c = std::max(p->scale * kLog2e, 1e-30f);
  return a;
}

// Shares that dk and dv are summed from: where the tiles of keys do not fill the chip a few times
// over (under a causal mask they differ much in length), each tile's rows are dealt to several
// workgroups, as long as each gets enough of them.
int parts_of(const gbmw_attention_problem* p) {
  const int64_t groups = (int64_t)p->B * p->Hk * ((p->Lk + 127) / 128), rows = (int64_t)p->Lq * (p->Hq / p->Hk);
  int parts = 1;
  while (parts < 16 && groups * parts < GBMW_FILL && rows / (2 * parts) >= GBMW_LEAST) parts *= 2;
  return parts;
}

// level and delta [B][Hk][rows], and for float16 gmax [B][Hk][tiles][4] and vmax [B][Hk][parts of 256 keys]
struct Scratch {
  int64_t rows, gmax, vmax, partial;   // floats
  int parts;
  int64_t bytes() const { return 4 * (2 * rows + gmax + vmax + partial); }
};
Scratch scratch_of(const gbmw_attention_problem* p) {
  const int64_t groups = (int64_t)p->B * p->Hk, rows = (int64_t)p->Lq * (p->Hq / p->Hk);
  const bool lift = p->dtype == GBMW_F16;
  const int parts = parts_of(p);
  auto padded = [](int64_t n) { return (n + 3) / 4 * 4; };
  return {padded(groups * rows), padded(lift ? groups * ((rows + 127) / 128) * 4 : 0),
          padded(lift ? groups * (((int64_t)p->Lk + 255) / 256) : 0),
          parts > 1 ? parts * 2 * groups * p->Lk * ((p->D + 3) / 4 * 4) : 0, parts};
}

#ifndef GBMW_NQ
#define GBMW_NQ 1
#endif
template <typename T, int KS, bool DIRECT>
void launch(const AttnArgs& a, bool backward, hipStream_t st) {
  const int64_t rows = (int64_t)a.Lq * a.share, groups = (int64_t)a.Hk * a.B;
  const dim3 grid_q((unsigned)((rows + 127) / 128 * groups)), grid_k((unsigned)(((int64_t)a.Lk + 127) / 128 * groups));
  if (!backward) {
    constexpr int NQ = GBMW_NQ;
    hipLaunchKernelGGL((k_attn_fwd<T, KS, NQ, DIRECT>), dim3((unsigned)((rows + 128 * NQ - 1) / (128 * NQ) * groups)),
                       dim3(256), 0, st, a);
    return;
  }
  if constexpr (__is_same(T, f16))
    if (a.Lk) hipLaunchKernelGGL(k_attn_vmax, dim3((unsigned)(((int64_t)a.Lk + 255) / 256 * groups)), dim3(256), 0, st, a);
  if (grid_q.x) hipLaunchKernelGGL((k_attn_dq<T, KS, DIRECT>), grid_q, dim3(256), 0, st, a);
  if (!grid_k.x) return;
  hipLaunchKernelGGL((k_attn_dkv<T, KS, DIRECT>), dim3(grid_k.x * a.parts), dim3(256), 0, st, a);
  if (a.parts > 1) {
    const int64_t quads = groups * a.Lk * (a.D4 / 4);
    hipLaunchKernelGGL(k_attn_join<T>, dim3((unsigned)((quads + 255) / 256), 2), dim3(256), 0, st, a);
  }
}

// Whether 64 rows of an array can be loaded straight to LDS.
bool direct(const void* ptr, const int64_t* stride, int L, int share, int D) {
  if (L == 0) return true;
  const int64_t row = stride[1] * 2, head = stride[2] * 2;
  if ((uintptr_t)ptr % 16 || (stride[0] * 2) % 16 || row % 16 || head % 16) return false;
  if (row < 2 * D) return false;   // a tile's end is told by its length in bytes
  return 64 * row + share * head < (1ll << 31);
}

template <typename T>
void launch(const AttnArgs& a, bool backward, hipStream_t st) {
  const bool fast = a.D % 8 == 0 && direct(a.k, a.ks, a.Lk, 1, a.D) && direct(a.v, a.vs, a.Lk, 1, a.D) &&
                    (!backward || (direct(a.q, a.qs, a.Lq, a.share, a.D) && direct(a.dout, a.dos, a.Lq, a.share, a.D)));
  if (!fast) {
    if (a.D <= 64) launch<T, 4, false>(a, backward, st);
    else launch<T, 8, false>(a, backward, st);
  }
  else if (a.D <= 32) launch<T, 2, true>(a, backward, st);
  else if (a.D <= 64) launch<T, 4, true>(a, backward, st);
  else if (a.D <= 80) launch<T, 5, true>(a, backward, st);
  else if (a.D <= 96) launch<T, 6, true>(a, backward, st);
  else launch<T, 8, true>(a, backward, st);
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
  a.level = (float*)p->workspace, a.delta = a.level + sc.rows, a.gmax = a.delta + sc.rows, a.vmax = a.gmax + sc.gmax;
  a.partial = a.vmax + sc.vmax, a.parts = sc.parts;
  if (p->dtype == GBMW_F16) launch<f16>(a, true, (hipStream_t)p->stream);
  else launch<bf16>(a, true, (hipStream_t)p->stream);
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}
