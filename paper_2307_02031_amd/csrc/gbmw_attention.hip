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
// other operand is read in the same order (Reader::cols).
#include <algorithm>
#include <cfloat>
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
Divisor divisor(int64_t d) { return {(int)d, (unsigned)(((1ull << 32) + d - 1) / d)}; }

// Which head and which of its `units` pieces of work a workgroup takes: see Deal.
struct Plan {
  int per, units, near, last;   // heads of a die, units of a head, heads at a time, the first of the last heads
  int lot;                      // 2^lot heads next to each other are one die's
  Divisor of_near, near_units, of_last, of_rest;
};

struct AttnArgs {
  const char *q, *k, *v, *dout;
  char *out, *dq, *dk, *dv;
  float* lse;
  float *level, *delta;   // [B][Hk][rows]: log2(e) lse - kUp, inf for rows without keys; <dout, out>
  float *vmax, *gmax;     // f16: the largest norms of a value and of a row of dout, for parts of 64 keys and 32 rows
  int64_t qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];
  const int *len_q, *len_k;
  float* partial;         // [parts][2][B][Hk][Lk][D4]: shares of dk and dv
  Plan by_rows, by_keys;
  Divisor share, heads_k, parts_d, kparts_d;   // query heads of a key head; Hk, parts, kparts
  int B, Hq, Hk, Lq, Lk, D, causal;
  float *shares, *tops;   // [kparts][B][Hk][rows][D4] and [kparts][B][Hk][rows]: of out (or dq) and of what goes with it
  int parts, kparts;      // workgroups that share a tile of keys, or a tile of rows
  int D4;                 // D rounded up to 4
  float c;                // scale * log2(e): probabilities are powers of two
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
// A tile is 64 rows of CH 16-byte pieces (8, 12 or 16, by the head size), stored so that the two
// kinds of reads, a piece of each of 32 rows and (transposing) 64 bytes of each of four rows,
// touch all 64 banks evenly: piece p of row r lies at place p ^ swap_of(r) of its row, and rows of
// 16 pieces have 16 bytes between groups of four.  A lane then needs two or four addresses for
// each kind (Reader); everything else is a constant offset.
typedef __attribute__((address_space(3))) char lds_char;

template <int KS>
constexpr int kChunks = KS <= 4 ? 8 : KS <= 6 ? 12 : 16;
template <int CH>
__device__ __forceinline__ constexpr int swap_of(int row) {
  return CH == 16 ? (row & 3) << 2 : CH == 12 ? (row >> 2) & 3 : ((row & 2) << 1) | ((row >> 2) & 3);
}
template <int CH>
__device__ __forceinline__ constexpr int place_of(int row, int piece) {   // bytes
  return (row * CH + (piece ^ swap_of<CH>(row))) * 16 + (CH == 16 ? row / 4 * 16 : 0);
}
template <int KS>
constexpr int kTile = 64 * 16 * kChunks<KS> + (kChunks<KS> == 16 ? 256 : 0);   // bytes

template <int KS>
struct Reader {
  static constexpr int CH = kChunks<KS>, kSteps = CH == 16 ? 2 : 1;   // steps that share an address
  int row[CH == 12 ? 2 : 4], col[CH == 12 ? 2 : 4];
  __device__ __forceinline__ Reader() {
    const int l = threadIdx.x % 64, i = l % 16, half = l / 32;
#pragma unroll
    for (int n = 0; n < (CH == 12 ? 2 : 4); ++n) row[n] = place_of<CH>(l % 32, 2 * kSteps * n + half);
    // lanes 4u..4u+3 of sixteen name the quarters of run u of sixteen elements; lane i gets
    // element i of each of the four runs
    const int r = 4 * half + i / 4, c = 16 * ((l / 16) % 2) + 4 * (i % 4);
#pragma unroll
    for (int n = 0; n < (CH == 12 ? 2 : 4); ++n)   // of 32 columns each, of eight rows each, or of both
      col[n] = (CH == 16   ? place_of<CH>(r, 4 * n + c / 8)
                : CH == 12 ? place_of<CH>(r + 8 * n, c / 8)
                           : place_of<CH>(r + 8 * (n / 2), 4 * (n % 2) + c / 8)) + (c % 8) * 2;
  }
  static constexpr int down(int r) { return r * CH * 16 + (CH == 16 ? r / 4 * 16 : 0); }   // r a multiple of 16, or of 8 for CH = 16
  // A operand: rows r .. r+31 of the tile (r = 0 or 32), terms 16 step .. 16 step + 15
  __device__ __forceinline__ s16x8 rows(lds_char* tile, int r, int step) const {
    typedef __attribute__((address_space(3))) s16x8 lds8;
    return *(lds8*)(tile + (CH == 16   ? row[step / 2] + (step % 2) * 32
                            : CH == 12 ? row[step % 2] + (step / 2) * 64
                                       : row[step]) + down(r));
  }
  // A operand: rows = columns 32 d .. 32 d + 31 of the tile, terms = its rows r .. r+15 in the
  // order of a result's registers
  __device__ __forceinline__ s16x8 cols(lds_char* tile, int r, int d) const {
    typedef __attribute__((address_space(3))) s16x4 lds4;
    s16x4 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
      x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(tile + (CH == 16   ? col[d] + down(r + 8 * u)
                                                                     : CH == 12 ? col[u] + d * 64 + down(r)
                                                                                : col[d + 2 * u] + down(r))));
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
  Divisor share;
  int count;              // rows beyond count read as zeros
};

// Brings 64 rows into a tile, in two halves: begin() before the tile before it is worked on,
// end() before the barrier that hands it over.
//
// Direct: the loads write to LDS themselves, 64 pieces in lane order; lanes fetch the pieces
// that belong in their places, and what is beyond the buffer's bounds arrives as zeros.  Needs
// 16-byte aligned rows and offsets inside a tile below 2^31.  Otherwise through registers.
//
// A wave brings N runs of 64 pieces.  Its lanes' offsets inside a run are the same for all of
// them where rows have 16 pieces; with SPARE every run gets bounds of its own and the lanes keep
// one offset, otherwise N (for the kernel that is short of registers, and those that are not).
// ALONE: a wave brings 32 rows for itself, and nobody else waits for them.
template <int KS, bool DIRECT, bool SPARE = false, bool ALONE = false>
struct Loader {
  static constexpr int CH = kChunks<KS>, ROWS = ALONE ? 32 : 64, THREADS = ALONE ? 64 : 256;
  static constexpr int N = DIRECT ? ROWS * CH / THREADS : (ROWS * 2 * KS + THREADS - 1) / THREADS;
  static constexpr bool kOne = SPARE && CH == 16;
  static constexpr int NA = kOne ? 1 : N;
  static constexpr unsigned kOut = 0x80000000u;
  s16x8 x[DIRECT ? 1 : N];
  unsigned at[DIRECT ? NA : 1];

  __device__ __forceinline__ static int wave() { return ALONE ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }
  __device__ __forceinline__ static int thread() { return ALONE ? threadIdx.x % 64 : threadIdx.x; }
  __device__ __forceinline__ static int row_of(int i) { return ((wave() * N + i) * 64 + (int)threadIdx.x % 64) / CH; }
  __device__ __forceinline__ void init(const Rows& rows, int D) {
    if constexpr (DIRECT) {
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int piece = ((wave() * N + i) * 64 + (int)threadIdx.x % 64) % CH ^ swap_of<CH>(row_of(i));
        const int down = kOne ? (int)(threadIdx.x % 64) / CH : row_of(i);   // of its run, or of the tile
        at[i] = 8 * piece >= D ? kOut : 16 * piece + (rows.share.d == 1 ? down * (unsigned)rows.stride : 0u);
      }
    }
  }

  __device__ __forceinline__ void begin(lds_char* tile, const Rows& rows, int first, int D) {
    if constexpr (DIRECT) {
      if (rows.share.d == 1) {   // rows beyond the last one are beyond the bounds
        const int64_t length = (int64_t)(rows.count - first) * rows.stride;
        const int left = (int)min(length, (int64_t)0x7fffffff), run = 64 / CH * (int)rows.stride;
        const char* base = rows.base + first * rows.stride;
        const int skip = kOne ? wave() * N * run : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int off = kOne ? skip + i * run : 0;
          load(tile, __builtin_amdgcn_make_buffer_rsrc((void*)(base + off), 0, max(left - off, 0), 0x00020000), i, at[i % NA]);
        }
      } else {
        const int x0 = rows.share.of(first);
        __amdgpu_buffer_rsrc_t from =
            __builtin_amdgcn_make_buffer_rsrc((void*)(rows.base + x0 * rows.stride), 0, 0x7fffffff, 0x00020000);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = first + row_of(i), x = rows.share.of(r);
          load(tile, from, i, ((r >= rows.count) | (at[i % NA] == kOut)) ? kOut
                                  : at[i % NA] + (unsigned)(x - x0) * (unsigned)rows.stride + (unsigned)(r - x * rows.share.d) * (unsigned)rows.head);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = thread() + THREADS * i, r = first + n / (2 * KS);
        const bool there = n < ROWS * 2 * KS && r < rows.count;
        const int q = there ? r : first, h = rows.share.of(q);
        x[i] = load8<false>(rows.base + h * rows.stride + (q - h * rows.share.d) * rows.head, n % (2 * KS), D, there);
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
        const int n = thread() + THREADS * i, r = n / (2 * KS);
        if (r < ROWS) *(lds8*)(tile + place_of<CH>(r, n % (2 * KS))) = x[i];
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

// Four values of a row from d on (a multiple of four).
template <typename T>
__device__ __forceinline__ void store_quad(T* row, int d, int D, f32x4 x) {
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  const Tx4 y = {(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
  if (d + 4 <= D) {
    __builtin_memcpy(row + d, &y, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < D) row[d + i] = y[i];
  }
}

// A row that sees no key has the result 0 by choice, not as a product with 0: the others' keys may
// hold anything.
template <int DB>
__device__ __forceinline__ void clear_unless(bool sees, f32x16 (&x)[DB]) {
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[d][r] = sees ? x[d][r] : 0.0f;
}

// A lane's part of a result's rows, times f, as a share in 32 bits.
template <int DB>
__device__ __forceinline__ void store_share(float* row, int D4, const f32x16 (&x)[DB], float f) {
  const int half = threadIdx.x % 64 / 32;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int at = 32 * d + 8 * (r / 4) + 4 * half;
      if (at < D4) *(f32x4*)(row + at) = f32x4{x[d][r] * f, x[d][r + 1] * f, x[d][r + 2] * f, x[d][r + 3] * f};
    }
}

// Which head and which of its units a workgroup takes.  Workgroups are dealt to the eight dies in
// turn.  A die works on its own heads, `near` of them at a time, so that what their units read
// alike stays in its cache; of those the first units (the longest under a causal mask) come first.
// Heads are dealt to the dies in lots, so that every die gets a share of every sample: samples have
// lengths of their own.  Heads that eight does not divide are dealt to all dies at the end.
struct Deal {
  int head, unit;
  __device__ __forceinline__ Deal(const Plan& p) {
    const int id = blockIdx.x;
    if (id < 8 * p.per * p.units) {
      const int at = id / 8;
      int first = p.last, in = at - p.last * p.units;
      if (in >= 0) {
        unit = p.of_last.of(in);
        in -= unit * p.of_last.d;
      } else {
        first = p.near_units.of(at) * p.near;
        in = at - first * p.units;
        unit = p.of_near.of(in);
        in -= unit * p.near;
      }
      const int n = first + in;
      head = ((((n >> p.lot) * 8 + id % 8) << p.lot) | (n & ((1 << p.lot) - 1)));
    } else {
      const int at = id - 8 * p.per * p.units;
      unit = p.of_rest.of(at);
      head = 8 * p.per + at - unit * p.of_rest.d;
    }
  }
};

// Where a workgroup of the rows' kernels works: `per` rows of one (sample, key head), and of the
// keys that any of them sees its part of `kparts`.
struct Place {
  int tile, tiles, part, hk, b, nq, nk, rows, most, begin, end;
  __device__ __forceinline__ Place(const AttnArgs& a, int per) {
    rows = a.Lq * a.share.d;
    tiles = (rows + per - 1) / per;
    const Deal d(a.by_rows);
    const int at = a.kparts_d.of(d.unit);
    tile = tiles - 1 - at;   // the longest rows of a causal mask first
    part = d.unit - at * a.kparts;
    b = a.heads_k.of(d.head), hk = d.head - b * a.Hk;
    nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk);
    const int first = a.share.of(tile * per), last = min(a.share.of(min(tile * per + per, rows) - 1), nq - 1);
    most = first >= nq ? 0 : sees(a, last);
    // up to two tiles stay together
    const int run = most <= 128 ? 128 : a.kparts_d.of((most + 63) / 64 + a.kparts - 1) * 64;
    begin = min(part * run, most), end = min(begin + run, most);
  }
  __device__ __forceinline__ int sees(const AttnArgs& a, int i) const {   // keys j < sees
    return i >= nq ? 0 : a.causal ? max(0, min(nk, i + nk - nq + 1)) : nk;
  }
  // of a row in `shares` and `tops`
  __device__ __forceinline__ int64_t share_of(const AttnArgs& a, int row) const {
    return (((int64_t)part * a.B + b) * a.Hk + hk) * rows + row;
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
// A workgroup takes 128 rows of one (sample, key head), 32 a wave, and walks the keys in tiles
// of 64.  A wave computes x^T = K Q^T (lane: one row, 32 keys), so the running maximum and sum
// of a row need one exchange between two lanes a tile, and out^T += V^T p^T with p from its own
// registers.  The running sums are in units of 2^(c m); m follows the maximum only when that is
// more than 2^kLag ahead, so they are seldom rescaled.
//
// Sums are kept in 32 bits; probabilities are rounded to the type once, because they enter a
// matrix product of that type (the row's sum adds them unrounded).
//
// Per tile and wave 32 matrix instructions of 32 cycles (heads of 128), about as many cycles of
// exponentials and other vector instructions and a quarter of them of LDS: two waves a SIMD
// overlap the first two.  Medians: 40 heads x 8192 x 128: 1.28 ms, 1075 TFLOP/s, the library's
// large product of the type reaches 1223; 5 x 32 heads x 2048: 344 us, 999; 4 x 40 heads x 2048
// causal: 208 us, 826 of the visible half (tiles on the diagonal, and a start and an end per
// workgroup of 17 tiles), 214 where q, k and v are parts of one product's rows, and 250 for
// those repeated without a pause.  64 rows a wave (half the LDS reads, one wave a SIMD) took
// 397 us for the last where 32 took 287.
constexpr float kLag = 6.0f;

// One row's running maximum (in units of x / scale), sum, and out^T: what a wave has of 32 rows.
template <int DB>
struct Running {
  f32x16 o[DB] = {};
  float m = -kInf, sum = 0.0f;
};

// Takes N runs of 32 keys in: x holds their scores, and leaves with their probabilities.
template <typename T, int DB, int N>
__device__ __forceinline__ void take_scores(Running<DB>& w, f32x16 (&x)[N], float c) {
  // the matrix results are waited for where the compiler sees them read, before max3
  float top = w.m;
#pragma unroll
  for (int u = 0; u < N; ++u) top = fmaxf(top, x[u][15]);
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int r = 0; r < 16; r += 2) top = max3(top, x[u][r], x[u][r + 1]);
  float low;
  const float high = other_half(top, &low);
  top = fmaxf(low, high);
  const bool ahead = (top - w.m) * c > kLag;
  if (__any(ahead)) {
    const float f = ahead ? __builtin_amdgcn_exp2f((w.m - top) * c) : 1.0f;
    if (ahead) w.m = top;
    w.sum *= f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[d][r] *= f;
  }
  const float off = (w.m == -kInf ? 0.0f : w.m * c) - kUp<T>;
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[u][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][r], c, -off));
      w.sum += x[u][r];
    }
}

// log2 of a row's sum of 2^(c x): -inf without keys.
template <typename T>
__device__ __forceinline__ float level_of(float m, float sum, float c) {
  const bool empty = m == -kInf && !(sum != sum);
  return empty ? -kInf : m * c - kUp<T> + __builtin_amdgcn_logf(sum);
}

template <typename T, int KS, bool DIRECT>
__global__ __launch_bounds__(256, 2) void k_attn_fwd(AttnArgs a) {
  constexpr int DB = (KS + 1) / 2;
  __shared__ __attribute__((aligned(16))) char lds[4 * kTile<KS>];
  lds_char* const tiles = (lds_char*)lds;
  const Place w(a, 128);
  const int l = threadIdx.x % 64, half = l / 32, row = w.tile * 128 + (threadIdx.x / 64) * 32 + l % 32;
  const int i = a.share.of(row), hq = (w.hk - i) * a.share.d + row;
  const int sees = w.sees(a, i);
  const Rows kr{a.k + 2 * (w.b * a.ks[0] + w.hk * a.ks[2]), 2 * a.ks[1], 0, {1, 0}, w.nk};
  const Rows vr{a.v + 2 * (w.b * a.vs[0] + w.hk * a.vs[2]), 2 * a.vs[1], 0, {1, 0}, w.nk};

  s16x8 q[KS];
  const char* qrow = a.q + 2 * (w.b * a.qs[0] + (i < w.nq ? i : 0) * a.qs[1] + hq * a.qs[2]);
#pragma unroll
  for (int s = 0; s < KS; ++s) q[s] = load8<DIRECT>(qrow, 2 * s + half, a.D, i < w.nq);
  Running<DB> run;
  const Reader<KS> rd;
  Loader<KS, DIRECT> lk, lv;
  lk.init(kr, a.D), lv.init(vr, a.D);
  if (w.begin < w.end) {
    lk.begin(tiles, kr, w.begin, a.D);
    lv.begin(tiles + kTile<KS>, vr, w.begin, a.D);
  }
  for (int j0 = w.begin, buf = 0; j0 < w.end; j0 += 64, buf ^= 1) {
    lds_char *tk = tiles + 2 * buf * kTile<KS>, *tv = tk + kTile<KS>;
    lk.end(tk), lv.end(tv);
    __syncthreads();   // this tile is whole, and nobody reads the other buffer any more
    if (j0 + 64 < w.end) {
      lds_char* to = tiles + 2 * (buf ^ 1) * kTile<KS>;
      lk.begin(to, kr, j0 + 64, a.D);
      lv.begin(to + kTile<KS>, vr, j0 + 64, a.D);
    }
    if (!__any(j0 < sees)) continue;   // none of the wave's rows sees this tile
    f32x16 x[2] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int s = 0; s < KS; ++s) x[u] = mma<T>(rd.rows(tk, 32 * u, s), q[s], x[u]);
    if (!__all(j0 + 64 <= sees)) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (j0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4 >= sees) x[u][r] = -kInf;
    }
    take_scores<T>(run, x, a.c);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const s16x8 p = round8<T>(x[u], t);
#pragma unroll
        for (int d = 0; d < DB; ++d) run.o[d] = mma<T>(rd.cols(tv, 32 * u + 16 * t, d), p, run.o[d]);
      }
  }
  run.sum += __shfl_xor(run.sum, 32);
  if (row >= w.rows) return;
  const float level = level_of<T>(run.m, run.sum, a.c), f = level == -kInf ? 0.0f : 1.0f / run.sum;
  if (!__all(w.begin < sees)) clear_unless(w.begin < sees, run.o);
  if (a.kparts == 1) {
    if (half == 0) a.lse[((int64_t)w.b * a.Hq + hq) * a.Lq + i] = level * kLn2;
    char* out = a.out + 2 * (w.b * a.os[0] + i * a.os[1] + hq * a.os[2]);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int at = 32 * d + 8 * (r / 4) + 4 * half;
        if (at < a.D) store4<T, DIRECT>(out, at, a.D, run.o[d], r, f);
      }
  } else {
    const int64_t at = w.share_of(a, row);
    if (half == 0) a.tops[at] = level;
    store_share(a.shares + at * a.D4, a.D4, run.o, f);
  }
}

// Forward where a key head has at most 32 rows (one token, a few of them, few heads that share):
// there the keys are what has to be read, and every wave of a workgroup walks tiles of 32 keys
// of its own, without waiting for the others; at the end their sums are put together.  4 x 32
// query on 8 key heads, one token, 4500 keys on average: 19 us, 4.2 TB/s of keys and values
// (128 us with tiles shared by the workgroup, of which one wave has rows); 8 x 16 heads, 4 rows
// over 384 keys: 7.9 us (9.5 where keys and values are not in the cache yet), the latency of three
// tiles in sequence on half of the chip (12.6 with shared tiles).
template <typename T, int KS, bool DIRECT>
__global__ __launch_bounds__(256, 1) void k_attn_few(AttnArgs a) {
  constexpr int DB = (KS + 1) / 2, kHalf = Reader<KS>::down(32), kWave = 4 * kHalf, DP = 32 * DB + 4;
  static_assert(32 * DP * 4 <= kWave, "a wave's sums fit where its tiles were");
  __shared__ __attribute__((aligned(16))) char lds[4 * kWave];
  __shared__ float sTop[4][32], sSum[4][32];
  const Place w(a, 32);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  lds_char* const tiles = (lds_char*)lds + wave * kWave;
  const int l = threadIdx.x % 64, half = l / 32, row = l % 32;
  const int i = a.share.of(row), hq = (w.hk - i) * a.share.d + row;
  const int sees = row < w.rows ? w.sees(a, i) : INT_MAX;   // rows that are not there need no mask
  const Rows kr{a.k + 2 * (w.b * a.ks[0] + w.hk * a.ks[2]), 2 * a.ks[1], 0, {1, 0}, w.nk};
  const Rows vr{a.v + 2 * (w.b * a.vs[0] + w.hk * a.vs[2]), 2 * a.vs[1], 0, {1, 0}, w.nk};

  s16x8 q[KS];
  const bool there = row < w.rows && i < w.nq;
  const char* qrow = a.q + 2 * (w.b * a.qs[0] + (there ? i * a.qs[1] + hq * a.qs[2] : 0));
#pragma unroll
  for (int s = 0; s < KS; ++s) q[s] = load8<DIRECT>(qrow, 2 * s + half, a.D, there);
  Running<DB> run;
  const Reader<KS> rd;
  Loader<KS, DIRECT, false, true> lk, lv;
  lk.init(kr, a.D), lv.init(vr, a.D);
  auto begin = [&](int buf, int j0) {
    lk.begin(tiles + 2 * buf * kHalf, kr, j0, a.D);
    lv.begin(tiles + (2 * buf + 1) * kHalf, vr, j0, a.D);
  };
  int j0 = w.begin + 32 * wave;
  if (j0 < w.end) begin(0, j0);
  for (int buf = 0; j0 < w.end; j0 += 128, buf ^= 1) {
    lds_char *tk = tiles + 2 * buf * kHalf, *tv = tk + kHalf;
    lk.end(tk), lv.end(tv);
    __builtin_amdgcn_s_waitcnt(0xc07f);   // the last tile's reads are done: its place is loaded next
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    f32x16 x[1] = {};
    if (j0 + 128 < w.end) begin(buf ^ 1, j0 + 128);
#pragma unroll
    for (int s = 0; s < KS; ++s) x[0] = mma<T>(rd.rows(tk, 0, s), q[s], x[0]);
    if (!__all(j0 + 32 <= sees)) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (j0 + 8 * (r / 4) + 4 * half + r % 4 >= sees) x[0][r] = -kInf;
    }
    take_scores<T>(run, x, a.c);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const s16x8 p = round8<T>(x[0], t);
#pragma unroll
      for (int d = 0; d < DB; ++d) run.o[d] = mma<T>(rd.cols(tv, 16 * t, d), p, run.o[d]);
    }
  }
  run.sum += __shfl_xor(run.sum, 32);
  if (!__all(w.begin < sees)) clear_unless(w.begin < sees, run.o);
  {
    const float level = level_of<T>(run.m, run.sum, a.c);
    if (half == 0) sTop[wave][row] = level, sSum[wave][row] = run.sum;
    __builtin_amdgcn_s_waitcnt(0);   // every read of this wave's tiles is done
    float* o = (float*)(lds + wave * kWave) + row * DP;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *(f32x4*)(o + 32 * d + 8 * (r / 4) + 4 * half) = f32x4{run.o[d][r], run.o[d][r + 1], run.o[d][r + 2], run.o[d][r + 3]};
  }
  __syncthreads();
  // eight threads a row, quads of values
  const int out_row = threadIdx.x / 8;
  if (out_row >= w.rows) return;
  float top = -kInf, sum = 0.0f, f[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) top = fmaxf(top, sTop[k][out_row]);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float level = sTop[k][out_row];
    const float share = level == -kInf ? 0.0f : __builtin_amdgcn_exp2f(level - (top == -kInf ? 0.0f : top));
    sum += share;
    f[k] = level == -kInf ? 0.0f : share / sSum[k][out_row];
  }
  const bool empty = top == -kInf && !(sum != sum);
  const float level = empty ? -kInf : top + __builtin_amdgcn_logf(sum), inv = empty ? 0.0f : 1.0f / sum;
  const int oi = a.share.of(out_row), oh = (w.hk - oi) * a.share.d + out_row;
  const int64_t at = w.share_of(a, out_row);
  if (threadIdx.x % 8 == 0) {
    if (a.kparts == 1) a.lse[((int64_t)w.b * a.Hq + oh) * a.Lq + oi] = level * kLn2;
    else a.tops[at] = level;
  }
  for (int d = threadIdx.x % 8 * 4; d < a.D4; d += 32) {
    f32x4 o = {};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x4 y = *(const f32x4*)((const float*)(lds + k * kWave) + out_row * DP + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(y[e], f[k], o[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    if (a.kparts == 1) store_quad<T>((T*)a.out + w.b * a.os[0] + oi * a.os[1] + oh * a.os[2], d, a.D, o);
    else *(f32x4*)(a.shares + at * a.D4 + d) = o;
  }
}

// out and lse, or dq and delta, from the parts' shares: four values a thread, in the parts' order.
template <typename T, bool BACKWARD>
__global__ __launch_bounds__(256) void k_attn_merge(AttnArgs a) {
  const int64_t rows = (int64_t)a.Lq * a.share.d, all = rows * a.Hk * a.B;
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x, at = n / (a.D4 / 4);
  if (at >= all) return;
  const int d = (int)(n % (a.D4 / 4)) * 4;
  const int64_t head = at / rows;
  const int row = (int)(at - head * rows), i = a.share.of(row), hk = (int)(head % a.Hk), b = (int)(head / a.Hk);
  const int hq = (hk - i) * a.share.d + row;
  f32x4 o = {};
  float top = -kInf, sum = 0.0f;
  if constexpr (!BACKWARD)
#pragma unroll 8
    for (int k = 0; k < a.kparts; ++k) top = fmaxf(top, a.tops[k * all + at]);
#pragma unroll 8
  for (int k = 0; k < a.kparts; ++k) {
    const float t = a.tops[k * all + at];
    float f = 1.0f;
    if constexpr (!BACKWARD) f = t == -kInf ? 0.0f : __builtin_amdgcn_exp2f(t - (top == -kInf ? 0.0f : top));
    sum += BACKWARD ? t : f;
    const f32x4 y = *(const f32x4*)(a.shares + (k * all + at) * a.D4 + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(y[e], f, o[e]);
  }
  if constexpr (BACKWARD) {
    if (d == 0) a.delta[at] += sum;
    store_quad<T>((T*)a.dq + b * a.dqs[0] + i * a.dqs[1] + hq * a.dqs[2], d, a.D, o);
  } else {
    const bool empty = top == -kInf && !(sum != sum);
    const float inv = empty ? 0.0f : 1.0f / sum;
    if (d == 0) a.lse[((int64_t)b * a.Hq + hq) * a.Lq + i] = empty ? -kInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    store_quad<T>((T*)a.out + b * a.os[0] + i * a.os[1] + hq * a.os[2], d, a.D, o);
  }
}

// The largest norm of a value among 64 keys of a (sample, key head), for float16's lift.  Workgroup
// (x, y) takes half y of x's 128 keys.
__global__ __launch_bounds__(256) void k_attn_vmax(AttnArgs a) {
  __shared__ float tops[4];
  const int parts = (a.Lk + 63) / 64, tiles = (a.Lk + 127) / 128, part = 2 * (blockIdx.x % tiles) + blockIdx.y;
  if (part >= parts) return;
  const int head = blockIdx.x / tiles, hk = head % a.Hk, b = head / a.Hk;
  // sixteen lanes a row, a piece each
  const int last = min(part * 64 + 64, length(a.len_k, b, a.Lk)), d = threadIdx.x % 16 * 8;
  const f16* v = (const f16*)a.v + b * a.vs[0] + hk * a.vs[2] + d;
  float s = 0.0f;
  for (int key = part * 64 + threadIdx.x / 16; key < last; key += 16) {
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
  if (threadIdx.x == 0) a.vmax[(int64_t)head * parts + part] = __builtin_sqrtf(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
}

// ---- backward, dq -----------------------------------------------------------------------------
//
// Rows and keys as in the forward pass: p^T from K Q^T and the row's log-sum-exp, dp^T = V
// dout^T, ds^T = p^T (dp^T - delta), dq^T += K^T ds^T.  Writes delta = <dout, out> of its rows and,
// for float16, their largest norm for the other kernel.
//
// The backward pass is two kernels that both recompute p and dp (seven products, where one kernel
// would do with five): each sum then has one owner, nothing is added atomically, and the result
// does not depend on timing.  One kernel's shares of dq, a row tile's per tile of keys, would be
// written and read at more than the memory's rate (where a head has several tiles of keys).  Score gradients are rounded to the type once,
// as operands.  This one's three products: 32 query on 8 key heads x 8192 x 128 causal 741 us, 1113
// TFLOP/s; 16 x 20 heads x 512 x 64, ragged: 47 us, bound by starts, ends and a last round of
// workgroups that fills a quarter of the chip.
template <typename T, int KS, bool DIRECT>
__global__ __launch_bounds__(256, 2) void k_attn_dq(AttnArgs a) {
  constexpr int DB = (KS + 1) / 2;
  constexpr bool kLift = __is_same(T, f16);
  __shared__ __attribute__((aligned(16))) char lds[4 * kTile<KS>];
  lds_char* const tiles = (lds_char*)lds;
  const Place w(a, 128);
  const int l = threadIdx.x % 64, half = l / 32, row = w.tile * 128 + (threadIdx.x / 64) * 32 + l % 32;
  const int i = a.share.of(row), hq = (w.hk - i) * a.share.d + row;
  const int b = w.b, hk = w.hk, nq = w.nq, nk = w.nk, rows = w.rows;
  const int sees = w.sees(a, i);
  const Rows kr{a.k + 2 * (b * a.ks[0] + hk * a.ks[2]), 2 * a.ks[1], 0, {1, 0}, nk};
  const Rows vr{a.v + 2 * (b * a.vs[0] + hk * a.vs[2]), 2 * a.vs[1], 0, {1, 0}, nk};

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
    norm += __shfl_xor(norm, 32);
    norm = sees > 0 ? __builtin_sqrtf(norm) : 0.0f;
    const int parts = (a.Lk + 63) / 64;
    const int k = lift_of(norm * max_of(a.vmax + ((int64_t)b * a.Hk + hk) * parts, (nk + 63) / 64));
    up = __builtin_ldexpf(1.0f, k), down = __builtin_ldexpf(1.0f, -k);
    float top = norm;
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (l == 0 && w.part == 0) a.gmax[(((int64_t)b * a.Hk + hk) * w.tiles + w.tile) * 4 + threadIdx.x / 64] = top;
  }
  f32x16 o[DB] = {};
  float left = 0.0f;
  const Reader<KS> rd;
  Loader<KS, DIRECT> lk, lv;
  lk.init(kr, a.D), lv.init(vr, a.D);
  // The score gradients of a row add up to 0: what their sum leaves over is delta's error, the
  // rounding of `out`.  The other kernel gets the corrected delta.  Here it matters where few
  // keys share a row, and there (one tile, or the first rows of a causal mask) a first pass finds it.
  const bool small = w.most <= (a.causal ? 128 : 64);
  for (int pass = !small; pass < 2; ++pass) {
    left = 0.0f;
    if (w.begin < w.end) {
      lk.begin(tiles, kr, w.begin, a.D);
      lv.begin(tiles + kTile<KS>, vr, w.begin, a.D);
    }
    for (int j0 = w.begin, buf = 0; j0 < w.end; j0 += 64, buf ^= 1) {
      lds_char *tk = tiles + 2 * buf * kTile<KS>, *tv = tk + kTile<KS>;
      lk.end(tk), lv.end(tv);
      __syncthreads();
      if (j0 + 64 < w.end) {
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
    left *= down;
    if (pass == 0) delta += left;
    __syncthreads();   // the next pass begins with the first buffer again
  }
  if (row >= rows) return;
  if (!__all(w.begin < sees)) clear_unless(w.begin < sees, o);
  const int64_t at = ((int64_t)b * a.Hk + hk) * rows + row;
  if (half == 0 && w.part == 0) a.delta[at] = a.kparts == 1 ? delta + left : delta, a.level[at] = lse - kUp<T>;
  if (a.kparts == 1) {
    char* out = a.dq + 2 * (b * a.dqs[0] + i * a.dqs[1] + hq * a.dqs[2]);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int to = 32 * d + 8 * (r / 4) + 4 * half;
        if (to < a.D) store4<T, DIRECT>(out, to, a.D, o[d], r, a.scale * down);
      }
  } else {
    const int64_t to = w.share_of(a, row);
    if (half == 0) a.tops[to] = left;
    store_share(a.shares + to * a.D4, a.D4, o, a.scale * down);
  }
}

// ---- backward, dk and dv ----------------------------------------------------------------------
//
// A workgroup takes 128 keys of one (sample, key head), 32 a wave, and walks the rows in tiles
// of 64: x = Q K^T (lane: one key, 16 rows), dv^T += dout^T p, dk^T += Q^T ds.  Where several
// workgroups share a tile of keys, each writes its share and k_attn_join adds them in order.
//
// Bound by registers (128 sums a lane, and the keys and values it multiplies with): two waves a
// SIMD that wait for LDS 45 % of their time.  Four products: 32 query on 8 key heads x 8192 x 128
// causal 1.16 ms, 950 TFLOP/s; 16 x 20 heads x 512 x 64, ragged: 55 to 66 us, by which samples are
// long.  Without direct loads it keeps 96 to 212 bytes a lane in scratch memory.
template <typename T, int KS, bool DIRECT>
__global__ __launch_bounds__(256, KS <= 4 ? 3 : 2) void k_attn_dkv(AttnArgs a) {
  constexpr int DB = (KS + 1) / 2;
  __shared__ __attribute__((aligned(16))) char lds[4 * kTile<KS>];
  lds_char* const buffers = (lds_char*)lds;
  __shared__ __attribute__((aligned(16))) float sRow[2][2][64];   // level, delta
  const int heads = a.Hk * a.B;
  const Deal deal(a.by_keys);
  const int tile = a.parts_d.of(deal.unit), part = deal.unit - tile * a.parts;   // the keys that most rows see first
  const int b = a.heads_k.of(deal.head), hk = deal.head - b * a.Hk;
  const int nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk);
  const int l = threadIdx.x % 64, half = l / 32, key = tile * 128 + (threadIdx.x / 64) * 32 + l % 32;
  const int rows = nq * a.share.d;
  // the first row that sees key j
  auto first_of = [&](int j) { return a.causal ? max(0, j - (nk - nq)) * a.share.d : 0; };
  const int first = first_of(key);
  // the rows that see a key of the tile, in `parts` runs of whole tiles
  // and no row before the first that sees a key at all: dout there may be anything
  int begin = tile * 128 < nk ? min(max(first_of(tile * 128) / 64 * 64, first_of(0)), rows) : rows;
  const int run = a.parts_d.of((rows - begin + 63) / 64 + a.parts - 1) * 64;
  begin = min((int64_t)begin + (int64_t)part * run, (int64_t)rows);
  const int end = min((int64_t)begin + run, (int64_t)rows);
  const Rows qr{a.q + 2 * (b * a.qs[0] + (int64_t)hk * a.share.d * a.qs[2]), 2 * a.qs[1], 2 * a.qs[2], a.share, rows};
  const Rows gr{a.dout + 2 * (b * a.dos[0] + (int64_t)hk * a.share.d * a.dos[2]), 2 * a.dos[1], 2 * a.dos[2], a.share, rows};
  const int64_t row0 = ((int64_t)b * a.Hk + hk) * a.Lq * a.share.d;

  // With heads of 128 not all of a lane's keys and values fit in its registers beside the sums:
  // the last pieces of them wait in LDS, each lane's for itself.
  constexpr int PK = KS == 8 ? 2 : 0, PV = KS == 8 ? 1 : 0;
  __shared__ s16x8 parked[PK + PV > 0 ? PK + PV : 1][PK + PV > 0 ? 256 : 1];
  s16x8 k[KS], v[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int64_t j = key < nk ? key : 0;
    k[s] = load8<DIRECT>(a.k + 2 * (b * a.ks[0] + j * a.ks[1] + hk * a.ks[2]), 2 * s + half, a.D, key < nk);
    v[s] = load8<DIRECT>(a.v + 2 * (b * a.vs[0] + j * a.vs[1] + hk * a.vs[2]), 2 * s + half, a.D, key < nk);
  }
#pragma unroll
  for (int s = 0; s < PK; ++s) parked[s][threadIdx.x] = k[KS - PK + s];
#pragma unroll
  for (int s = 0; s < PV; ++s) parked[PK + s][threadIdx.x] = v[KS - PV + s];
  int mine = threadIdx.x;
  auto key_of = [&](int s) { return s < KS - PK ? k[s] : parked[s - (KS - PK)][mine]; };
  auto value_of = [&](int s) { return s < KS - PV ? v[s] : parked[PK + s - (KS - PV)][mine]; };
  f32x16 dk[DB] = {}, dv[DB] = {};

  float up = 1.0f, down = 1.0f;   // of score gradients, beyond kUp
  if constexpr (__is_same(T, f16)) {
    const int parts = (a.Lk + 63) / 64, gparts = (a.Lq * a.share.d + 127) / 128 * 4;
    const int lift = lift_of(max_of(a.gmax + ((int64_t)b * a.Hk + hk) * gparts, gparts) *
                             max_of(a.vmax + ((int64_t)b * a.Hk + hk) * parts, (nk + 63) / 64));
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
      asm("" : "+v"(mine));   // read again, not kept
      f32x16 x = {}, dp = {};
#pragma unroll
      for (int s = 0; s < KS; ++s) x = mma<T>(rd.rows(tq, 0, s), key_of(s), x);
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
      for (int s = 0; s < KS; ++s) dp = mma<T>(rd.rows(tg, 0, s), value_of(s), dp);
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
    store_share(o, a.D4, dk, fk);
    store_share(o + all, a.D4, dv, fv);
  }
}

// ---- backward of a few rows over a few keys ------------------------------------------------------
//
// All of one key head's problem in LDS and in 32 bits, one workgroup, one launch for dq, dk and dv:
//   P = exp2(c q k - log2(e) lse), dS = P (dout v - sum_j P dout v),
//   dq = scale dS k, dk = scale dS^T q, dv = P^T dout.
// Bound by latency: the products are a few thousand terms a column, and matrix instructions would
// be given tiles that are mostly empty.  With so few terms the roundings of P and dS to 16 bits
// do not average out either: the kernels above are off by 1.42 times the result's own rounding on
// average, by up to 1.56 where there are few heads.  Here P and dS are not rounded: 1.00.
//
// Its time grows with the pairs of rows and keys, theirs hardly does (us of the kernels, here / there):
//   heads x size   type       8 x 8        8 x 16       4 x 32       16 x 8       12 x 12      16 x 16
//   64 x 64        bfloat16   9.6 / 12.1   12.1 / 12.1  13.1 / 12.1  14.1 / 11.9  14.8 / 12.1  18.4 / 11.9
//   64 x 128       bfloat16   11.1 / 15.5  13.4 / 15.5  14.4 / 15.5  16.8 / 15.4  17.2 / 15.5  20.9 / 15.4
//   64 x 64        float16    9.7 / 17.1   12.3 / 17.1  13.3 / 17.3  14.3 / 17.0  14.9 / 17.0  18.6 / 17.0
//   2560 x 64      bfloat16   36 / 41      47 / 43      62 / 45      55 / 42      58 / 43      80 / 44
//   2560 x 128     float16    47 / 89      64 / 91      71 / 96      79 / 91      80 / 91      102 / 92
// They meet between 64 and 128 pairs with bfloat16, between 144 and 256 with float16; the limit is
// one in between, 128.  Up to it bfloat16 pays at most 1.37 times the time (2560 heads of 64, 4 x 32)
// for results that are rounded once.
constexpr int kFewRows = 16, kFewKeys = 32, kFewTerms = 128;

template <typename T>
__global__ __launch_bounds__(256) void k_attn_small(AttnArgs a) {
  constexpr int S = 129;   // floats from row to row: odd, so that neither order of reading meets a bank twice
  __shared__ float q[kFewRows][S], dout[kFewRows][S], k[kFewKeys][S], v[kFewKeys][S];
  __shared__ float p[kFewRows][kFewKeys + 1], ds[kFewRows][kFewKeys + 1];
  const int b = a.heads_k.of(blockIdx.x), hk = blockIdx.x - b * a.Hk, rows = a.Lq * a.share.d;
  const int nq = length(a.len_q, b, a.Lq), nk = length(a.len_k, b, a.Lk), ahead = nk - nq;
  const int d = threadIdx.x % 128, part = threadIdx.x / 128;
  auto sees = [&](int i) { return i >= nq ? 0 : a.causal ? max(0, min(nk, i + ahead + 1)) : nk; };
  if (d < a.D) {
#pragma unroll
    for (int n = 0; n < kFewRows; n += 2) {
      const int r = n + part, i = a.share.of(r), h = (hk - i) * a.share.d + r;
      const bool there = r < rows && i < nq;
      q[r][d] = there ? (float)((const T*)a.q)[b * a.qs[0] + i * a.qs[1] + h * a.qs[2] + d] : 0.0f;
      dout[r][d] = there ? (float)((const T*)a.dout)[b * a.dos[0] + i * a.dos[1] + h * a.dos[2] + d] : 0.0f;
    }
#pragma unroll
    for (int n = 0; n < kFewKeys; n += 2) {
      const int j = n + part;
      k[j][d] = j < nk ? (float)((const T*)a.k)[b * a.ks[0] + j * a.ks[1] + hk * a.ks[2] + d] : 0.0f;
      v[j][d] = j < nk ? (float)((const T*)a.v)[b * a.vs[0] + j * a.vs[1] + hk * a.vs[2] + d] : 0.0f;
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kFewRows; n += 8) {   // 32 lanes a row
    const int r = n + threadIdx.x / 32, j = threadIdx.x % 32, i = a.share.of(r), h = (hk - i) * a.share.d + r;
    float x = 0.0f, dp = 0.0f;
    const bool seen = r < rows && j < sees(i);
    if (seen) {
      for (int e = 0; e < a.D; ++e) {
        x = __builtin_fmaf(q[r][e], k[j][e], x);
        dp = __builtin_fmaf(dout[r][e], v[j][e], dp);
      }
      const float lse = a.lse[((int64_t)b * a.Hq + h) * a.Lq + i];
      x = lse == -kInf ? 0.0f : __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.c, -kLog2e * lse));
    }
    float delta = seen ? x * dp : 0.0f;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) delta += __shfl_xor(delta, m);
    p[r][j] = seen ? x : 0.0f;
    ds[r][j] = seen ? x * (dp - delta) : 0.0f;
  }
  __syncthreads();
  if (d >= a.D) return;
  for (int r = part; r < rows; r += 2) {
    const int i = a.share.of(r), h = (hk - i) * a.share.d + r, end = sees(i);
    float x = 0.0f;
    for (int j = 0; j < end; ++j) x = __builtin_fmaf(ds[r][j], k[j][d], x);
    ((T*)a.dq)[b * a.dqs[0] + i * a.dqs[1] + h * a.dqs[2] + d] = (T)(x * a.scale);
  }
  for (int j = part; j < a.Lk; j += 2) {
    const int first = j >= nk ? rows : a.causal ? max(0, j - ahead) * a.share.d : 0, end = nq * a.share.d;
    float x = 0.0f, y = 0.0f;
    for (int r = first; r < end; ++r) {
      x = __builtin_fmaf(ds[r][j], q[r][d], x);
      y = __builtin_fmaf(p[r][j], dout[r][d], y);
    }
    ((T*)a.dk)[b * a.dks[0] + j * a.dks[1] + hk * a.dks[2] + d] = (T)(x * a.scale);
    ((T*)a.dv)[b * a.dvs[0] + j * a.dvs[1] + hk * a.dvs[2] + d] = (T)y;
  }
}

// dk and dv from their shares, four values a thread, in the shares' order.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int64_t quads = (int64_t)a.B * a.Hk * a.Lk * (a.D4 / 4);
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= quads) return;
  f32x4 s = {};
  for (int k = 0; k < a.parts; ++k) s += *(const f32x4*)(a.partial + (((int64_t)k * 2 + blockIdx.y) * quads + n) * 4);
  const int d = (int)(n % (a.D4 / 4)) * 4;
  int64_t at = n / (a.D4 / 4);
  const int64_t key = at % a.Lk, hk = at / a.Lk % a.Hk, b = at / a.Lk / a.Hk;
  const int64_t* st = blockIdx.y ? a.dvs : a.dks;
  store_quad<T>((T*)(blockIdx.y ? a.dv : a.dk) + b * st[0] + key * st[1] + hk * st[2], d, a.D, s);
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
  // A launch has fewer than 2^32 threads along x, 2^24 workgroups of 256.  Tiles are shared by several
  // workgroups only where all of them are at most 4 * kSlots.
  const int64_t groups = std::max((rows + 127) / 128, ((int64_t)p->Lk + 127) / 128) * p->Hk;
  if (groups >= 1 << 24 || groups * p->B >= 1 << 24) return fail(GBMW_ERR_INVALID_ARG, "too many rows in all");
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
    if (extent[i] > 1 && (stride[i] < 0 || stride[i] > (1ll << 40))) return fail(GBMW_ERR_INVALID_ARG, "%s: stride %lld", name, (long long)stride[i]);
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
  // the stride of an extent of one says nothing
  auto take = [&](int64_t (&to)[3], const int64_t* stride, int L, int H) {
    to[0] = p->B > 1 ? stride[0] : 0;
    to[1] = L > 1 ? stride[1] : (p->D + 7) / 8 * 8;
    to[2] = H > 1 ? stride[2] : 0;
  };
  take(a.qs, p->q_stride, p->Lq, p->Hq), take(a.os, p->out_stride, p->Lq, p->Hq);
  take(a.dos, p->dout_stride, p->Lq, p->Hq), take(a.dqs, p->dq_stride, p->Lq, p->Hq);
  take(a.ks, p->k_stride, p->Lk, p->Hk), take(a.vs, p->v_stride, p->Lk, p->Hk);
  take(a.dks, p->dk_stride, p->Lk, p->Hk), take(a.dvs, p->dv_stride, p->Lk, p->Hk);
  a.len_q = p->len_q, a.len_k = p->len_k;
  a.B = p->B, a.Hq = p->Hq, a.Hk = p->Hk, a.Lq = p->Lq, a.Lk = p->Lk, a.D = p->D;
  a.share = divisor(p->Hq / p->Hk), a.heads_k = divisor(p->Hk);
  a.D4 = (p->D + 3) / 4 * 4;
  a.causal = p->causal, a.scale = p->scale;
  // neither 0 nor infinite: a hidden key's -inf has to stay -inf when it is scaled, a score of 0 has to stay 0
  a.c = std::clamp(p->scale * kLog2e, FLT_MIN, FLT_MAX);
  return a;
}

constexpr int kSlots = 512;   // workgroups that the chip holds at a time (two a compute unit)

// Workgroups that share a tile of keys in dk and dv.  Two reasons: tiles that do not fill half the
// chip, as long as each part gets 192 rows (28 heads, 484 rows, 56 tiles: backward 111 us, in four parts
// 67; 456 tiles of 395 rows in two: 68, in one 47), and a causal mask, under which they differ much in
// length, as long as each part gets 1024 (8 heads x 8192, 512 tiles of up to 8192 rows: 646 us, in two
// parts 557; 500 tiles of 1213 rows in two: 108, in one 92).
int parts_of(const gbmw_attention_problem* p) {
  const int64_t groups = (int64_t)p->B * p->Hk * ((p->Lk + 127) / 128), rows = (int64_t)p->Lq * (p->Hq / p->Hk);
  int parts = 1;
  while (parts < 16 && ((groups * parts < 2 * kSlots && rows / (2 * parts) >= 1024) ||
                        (groups * parts <= kSlots / 2 && rows / (2 * parts) >= 192)))
    parts *= 2;
  return parts;
}

bool few(const gbmw_attention_problem* p) { return (int64_t)p->Lq * (p->Hq / p->Hk) <= 32; }

// Workgroups that share a tile of rows: as many as fit the chip, each with enough keys that
// writing its share and reading it back (as much as two tiles of keys per 32 rows) is the less; under
// a causal mask up to twice as many, as long as each gets 1024 keys (388 tiles of up to 6171 keys
// forward: 105 us, in two parts 79; 500 of 1213: 30 us, in two 40).
int kparts_of(const gbmw_attention_problem* p, bool backward) {
  const int64_t rows = (int64_t)p->Lq * (p->Hq / p->Hk), groups = (int64_t)p->B * p->Hk * ((rows + 127) / 128);
  if (groups == 0) return 1;
  const int64_t tiles = ((int64_t)p->Lk + 63) / 64;
  if (few(p) && !backward) return (int)std::max<int64_t>(1, std::min({kSlots / 2 / groups, tiles / 8, (int64_t)64}));
  const int64_t least = std::max<int64_t>(2, std::min<int64_t>(rows, 128) / 16);
  int64_t parts = std::min({kSlots / groups, tiles / least, (int64_t)64});
  if (p->causal) parts = std::max(parts, std::min(2 * kSlots / groups, tiles / 16));
  return (int)std::max<int64_t>(1, parts);
}

// The forward call's workspace: shares and tops.  The backward call's: level and delta
// [B][Hk][rows], for float16 gmax [B][Hk][tiles][4] and vmax [B][Hk][parts of 64 keys], and
// shares and tops, or the shares of dk and dv after them.
struct Scratch {
  int64_t rows, gmax, vmax, shares, tops, partial;   // floats
  int parts, kparts;
  int64_t bytes() const { return 4 * (2 * rows + gmax + vmax + std::max(shares + tops, partial)); }
};
Scratch scratch_of(const gbmw_attention_problem* p, bool backward) {
  const int64_t groups = (int64_t)p->B * p->Hk, rows = (int64_t)p->Lq * (p->Hq / p->Hk), D4 = (p->D + 3) / 4 * 4;
  const bool lift = backward && p->dtype == GBMW_F16;
  auto padded = [](int64_t n) { return (n + 3) / 4 * 4; };
  Scratch s{};
  s.kparts = kparts_of(p, backward), s.parts = backward ? parts_of(p) : 1;
  s.rows = backward ? padded(groups * rows) : 0;
  s.gmax = padded(lift ? groups * ((rows + 127) / 128) * 4 : 0);
  s.vmax = padded(lift ? groups * (((int64_t)p->Lk + 63) / 64) : 0);
  if (s.kparts > 1) s.shares = s.kparts * groups * rows * D4, s.tops = padded(s.kparts * groups * rows);
  if (s.parts > 1) s.partial = s.parts * 2 * groups * p->Lk * D4;
  return s;
}

// Without a causal mask units are alike, and four heads at a time (keys and values of a few MB)
// suit a die's cache: 5 x 32 heads x 2048 x 128 forward 377 us, all at a time 384.  With one the
// order of their lengths counts more: 2 x 40 heads, all at a time 113 us, four 125; backward 411, 456.
//
// A lot is as many heads as fill whole lines of the cache, four at most: 8 x 8 heads, 1024 to 2048
// keys, 128 forward 247 us, with a die's heads all next to each other (of one sample) 289; 32 x 16
// heads of 80, 128 to 256 keys, 23 us, one by one 28.
Plan plan(int64_t heads, int64_t units, int D, bool causal) {
  const int64_t per = heads / 8, near = std::max<int64_t>(1, causal ? per : std::min<int64_t>(per, 4));
  const int64_t rest = per % near, last = rest ? per - rest : std::max<int64_t>(0, per - near);
  int lot = 0;
  while (lot < 2 && (D << lot) % 64 && per % (2 << lot) == 0) ++lot;
  return {(int)per, (int)units, (int)near, (int)last, lot, divisor(near), divisor(std::max<int64_t>(1, near * units)),
          divisor(std::max<int64_t>(1, per - last)), divisor(std::max<int64_t>(1, heads - 8 * per))};
}

void place_scratch(AttnArgs& a, const Scratch& s, void* workspace) {
  a.level = (float*)workspace, a.delta = a.level + s.rows, a.gmax = a.delta + s.rows, a.vmax = a.gmax + s.gmax;
  a.shares = a.partial = a.vmax + s.vmax, a.tops = a.shares + s.shares;
  a.parts = s.parts, a.kparts = s.kparts, a.parts_d = divisor(s.parts), a.kparts_d = divisor(s.kparts);
  const int64_t heads = (int64_t)a.Hk * a.B, rows = (int64_t)a.Lq * a.share.d;
  a.by_rows = plan(heads, (rows + 127) / 128 * a.kparts, a.D, a.causal);
  a.by_keys = plan(heads, ((int64_t)a.Lk + 127) / 128 * a.parts, a.D, a.causal);
}

template <typename T, int KS, bool DIRECT>
void launch(const AttnArgs& a, bool backward, hipStream_t st) {
  const int64_t rows = (int64_t)a.Lq * a.share.d, groups = (int64_t)a.Hk * a.B;
  auto grid = [&](int64_t n, int per) { return dim3((unsigned)((n + per - 1) / per * groups)); };
  auto times = [](dim3 g, int n) { return dim3(g.x * n); };
  const dim3 block(256), merge = dim3((unsigned)((rows * groups * (a.D4 / 4) + 255) / 256));
  if (!backward) {
    if (rows <= 32)
      hipLaunchKernelGGL((k_attn_few<T, KS, DIRECT>), times(grid(rows, 32), a.kparts), block, 0, st, a);
    else
      hipLaunchKernelGGL((k_attn_fwd<T, KS, DIRECT>), times(grid(rows, 128), a.kparts), block, 0, st, a);
    if (a.kparts > 1) hipLaunchKernelGGL((k_attn_merge<T, false>), merge, block, 0, st, a);
    return;
  }
  if constexpr (__is_same(T, f16))
    if (a.Lk) hipLaunchKernelGGL(k_attn_vmax, dim3(grid(a.Lk, 128).x, 2), block, 0, st, a);
  if (rows) {
    hipLaunchKernelGGL((k_attn_dq<T, KS, DIRECT>), times(grid(rows, 128), a.kparts), block, 0, st, a);
    if (a.kparts > 1) hipLaunchKernelGGL((k_attn_merge<T, true>), merge, block, 0, st, a);
  }
  if (!a.Lk) return;
  hipLaunchKernelGGL((k_attn_dkv<T, KS, DIRECT>), times(grid(a.Lk, 128), a.parts), block, 0, st, a);
  if (a.parts > 1) {
    const int64_t quads = groups * a.Lk * (a.D4 / 4);
    hipLaunchKernelGGL(k_attn_join<T>, dim3((unsigned)((quads + 255) / 256), 2), block, 0, st, a);
  }
}

bool small(const AttnArgs& a) {
  const int64_t rows = (int64_t)a.Lq * a.share.d;
  return rows <= kFewRows && a.Lk <= kFewKeys && rows * a.Lk <= kFewTerms;
}

// Whether 64 rows of an array can be loaded straight to LDS.
bool direct(const void* ptr, const int64_t* stride, int L, int share, int D) {
  if (L == 0) return true;
  const int64_t row = stride[1] * 2, head = stride[2] * 2;
  if ((uintptr_t)ptr % 16 || (stride[0] * 2) % 16 || row % 16 || head % 16) return false;
  if (row < 2 * D) return false;   // a tile's end is told by its length in bytes
  return 64 * row + share * head < (1ll << 31);
}

// Head sizes by steps of 16 terms: heads of 40 take dk and dv 830 us with three steps, 1020 with four
// (14 x 30 on 15 heads, 1576 to 3152 keys, causal; dq 560 and 580, forward 469 and 477).
template <typename T>
void launch(const AttnArgs& a, bool backward, hipStream_t st) {
  if (backward && small(a)) {
    hipLaunchKernelGGL(k_attn_small<T>, dim3((unsigned)(a.B * a.Hk)), dim3(256), 0, st, a);
    return;
  }
  const bool fast = a.D % 8 == 0 && direct(a.k, a.ks, a.Lk, 1, a.D) && direct(a.v, a.vs, a.Lk, 1, a.D) &&
                    (!backward || (direct(a.q, a.qs, a.Lq, a.share.d, a.D) && direct(a.dout, a.dos, a.Lq, a.share.d, a.D)));
  if (!fast) {
    if (a.D <= 64) launch<T, 4, false>(a, backward, st);
    else launch<T, 8, false>(a, backward, st);
  }
  else if (a.D <= 32) launch<T, 2, true>(a, backward, st);
  else if (a.D <= 48) launch<T, 3, true>(a, backward, st);
  else if (a.D <= 64) launch<T, 4, true>(a, backward, st);
  else if (a.D <= 80) launch<T, 5, true>(a, backward, st);
  else if (a.D <= 96) launch<T, 6, true>(a, backward, st);
  else launch<T, 8, true>(a, backward, st);
}

}  // namespace
}  // namespace gbmw

using namespace gbmw;

static gbmw_status run(const gbmw_attention_problem* p, bool backward) {
  const Scratch sc = scratch_of(p, backward);
  const int64_t need = sc.bytes();
  if (need && (!p->workspace || p->workspace_bytes < need || (uintptr_t)p->workspace % 16))
    return fail(GBMW_ERR_INVALID_ARG, "workspace of %lld bytes, 16-byte aligned, is needed", (long long)need);
  AttnArgs a = args_of(p);
  place_scratch(a, sc, p->workspace);
  if (p->dtype == GBMW_F16) launch<f16>(a, backward, (hipStream_t)p->stream);
  else launch<bf16>(a, backward, (hipStream_t)p->stream);
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

extern "C" int64_t gbmw_attention_workspace(const gbmw_attention_problem* p, int32_t backward) {
  gbmw_detail::clear_error();
  if (check_sizes(p) != GBMW_OK) return -1;
  return scratch_of(p, backward != 0).bytes();
}

extern "C" gbmw_status gbmw_attention_forward(const gbmw_attention_problem* p) {
  gbmw_detail::clear_error();
  const gbmw_status st = check_common(p, false);
  if (st != GBMW_OK) return st;
  if (p->B == 0 || p->Lq == 0) return GBMW_OK;
  return run(p, false);
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
  return run(p, true);
}
