// Rotary positions of queries and keys.  Contract: include/gbmw.h.
#include "gbmw_rows.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

constexpr int kMostPairs = 256;
constexpr int kTable = 512;    // angles of a wave
constexpr int64_t kMostWaves = (1 << 26) - 8;   // of a launch, whose threads are counted in 32 bits

struct RotaryArgs {
  int B, L, Hq, H, D, rot;   // H: query and key heads
  int pairs;                 // rot / 2
  int turning, pieces;       // pieces of a head that turn, and those with the ones that are handed through
  int tokens, heads, chunks; // of a wave: tokens and heads; waves that share a token's heads
  int begin;                 // the launch's first token
  unsigned units;            // waves' worth of work
  Divisor of_chunk, of_head, of_row, of_pairs;
  float factor, sign;
  const double* freq;
  const int32_t *positions, *len;
  int64_t ps;
  const void *q, *k;
  void *qo, *ko;
  int64_t qs[3], ks[3], qos[3], kos[3];
};

// cos and sin of 2 pi x, |x| <= 1/2, by the quarter turn that x is nearest and the Taylor series of the
// rest (at most pi / 4; the first term left out is below 2^-28 of the result).  The rest is taken in fp64 and rounded
// to fp32 last: rounded before, half a turn less 10^-9 would be half a turn, and angles off by up to 2^-23.
__device__ __forceinline__ void turn_of(double x, float& c, float& s) {
  const double quarter = __builtin_rint(4.0 * x);
  const float r = (float)(6.28318530717958648 * __builtin_fma(-0.25, quarter, x)), r2 = r * r;
  const float sn = r + r * r2 * (-1.0f / 6 + r2 * (1.0f / 120 + r2 * (-1.0f / 5040 + r2 * (1.0f / 362880))));
  const float cs = 1.0f + r2 * (-0.5f + r2 * (1.0f / 24 + r2 * (-1.0f / 720 + r2 * (1.0f / 40320 - r2 * (1.0f / 3628800)))));
  const int n = (int)quarter & 3;
  c = n == 0 ? cs : n == 1 ? -sn : n == 2 ? -cs : sn;
  s = n == 0 ? sn : n == 1 ? cs : n == 2 ? -sn : -cs;
}

template <typename T, int W>
struct alignas(sizeof(T)) Piece {
  T v[W];
};
template <int WORDS>
using Words = uint32_t __attribute__((ext_vector_type(WORDS), aligned(1)));

template <bool STREAM, typename T, int W>
__device__ __forceinline__ void load(Piece<T, W>& r, const T* p) {
  if constexpr (STREAM && sizeof(r) >= 8) {
    const auto w = __builtin_nontemporal_load((const Words<sizeof(r) / 4>*)p);
    __builtin_memcpy(&r, &w, sizeof(r));
  } else {
    __builtin_memcpy(&r, p, sizeof(r));
  }
}
template <bool STREAM, typename T, int W>
__device__ __forceinline__ void store(T* p, const Piece<T, W>& r) {
  if constexpr (STREAM && sizeof(r) >= 8) {
    Words<sizeof(r) / 4> w;
    __builtin_memcpy(&w, &r, sizeof(r));
    __builtin_nontemporal_store(w, (Words<sizeof(r) / 4>*)p);
  } else {
    __builtin_memcpy(p, &r, sizeof(r));
  }
}

// Nothing behind this comes before the piece has been loaded.
template <typename T, int W>
__device__ __forceinline__ void arrived(const Piece<T, W>& r) {
  if constexpr (sizeof(r) >= 4) {
    uint32_t w[sizeof(r) / 4];
    __builtin_memcpy(w, &r, sizeof(r));
#pragma unroll
    for (unsigned i = 0; i < sizeof(r) / 4; ++i) asm volatile("" ::"v"(w[i]) : "memory");
  }
}

template <typename T>
__device__ __forceinline__ void turn(T& x, T& y, float c, float s) {
  const float u = (float)x, v = (float)y;
  x = (T)(u * c - v * s), y = (T)(u * s + v * c);
}

// A lane has two pieces of W values of a head: one and the one rot / 2 further on, or two of pairs next to each
// other (INTER), or two that are handed through.  A wave has as many heads as its lanes have pieces for: some of a
// token's, or all heads of some tokens.  Its loads go out first; then it computes its tokens' angles, in turns and
// in fp64 (a position times a frequency loses the digits of its fraction in fp32), into LDS, once for all heads.
//
// Bound by HBM, and by how much of it is asked for at a time: one load of each piece a lane and many short waves
// (4 x 2048 x 80 heads of 128 in bf16: 54 us, 6.2 TB/s; two rounds of heads a wave 60, a token a wave 68).
//
// Where what turns, or is handed through, is no whole number of pieces, the last piece starts early and shares
// columns with the one before it.  Both lanes have loaded them, by one instruction, before one of them stores:
// also in place (the pieces of a head that turn are at most 64).
template <typename T, int W, bool INTER, bool STREAM, bool ONE>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a) {
  __shared__ float table[4][2][kTable];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = a.rot / 2;
  const unsigned unit = blockIdx.x * 4 + wave;
  if (unit >= a.units) return;
  const int group = a.of_chunk.of((int)unit), chunk = (int)unit - group * a.chunks;
  const int first = a.begin + group * a.tokens, here = min(a.tokens, a.B * a.L - first), first_head = chunk * a.heads;
  const int items = ONE ? min(a.heads, a.H - first_head) : here * a.H;
  float(*angles)[kTable] = table[wave];
  if constexpr (ONE) {
    const int b = a.of_row.of(first);
    if (a.len && first - b * a.L >= a.len[b]) return;
  }
  for (int p0 = 0; p0 < a.pieces; p0 += 64) {
    const int width = min(64, a.pieces - p0), slots = 64 / width, slot = lane / width, piece = p0 + lane % width;
    const bool turns = piece < a.turning;
    int at, other;   // the places of its two pieces in a head
    if (turns) {
      at = INTER ? piece * W : min(piece * W, half - W);
      other = INTER ? min(at + a.turning * W, a.rot - W) : at + half;
    } else {
      at = a.rot + (piece - a.turning) * W, other = min(at + (a.pieces - a.turning) * W, a.D - W);
    }
    const bool few = !turns && a.D - a.rot < W;   // no piece is handed through, but single values
    const int t = ONE ? 0 : a.of_head.of(slot), head = first_head + slot - t * a.H;
    const int token = ONE ? first : min(first + t, a.B * a.L - 1), b = a.of_row.of(token), row = token - b * a.L;
    const bool live = slot < min(slots, items) && (ONE || !(a.len && row >= a.len[b])), key = head >= a.Hq;
    const T* from = key ? (const T*)a.k + (b * a.ks[0] + row * a.ks[1] + (head - a.Hq) * a.ks[2])
                        : (const T*)a.q + (b * a.qs[0] + row * a.qs[1] + head * a.qs[2]);
    T* to = key ? (T*)a.ko + (b * a.kos[0] + row * a.kos[1] + (head - a.Hq) * a.kos[2])
                : (T*)a.qo + (b * a.qos[0] + row * a.qos[1] + head * a.qos[2]);
    Piece<T, W> x, y;
    if (live) load<STREAM>(x, from + min(at, a.D - W)), load<STREAM>(y, from + other);
    if (p0 == 0) {
      for (int i = lane; i < here * a.pairs; i += 64) {
        const int t = ONE ? 0 : a.of_pairs.of(i), token = first + t, b = a.of_row.of(token), row = token - b * a.L;
        const int position = a.positions ? a.positions[b * a.ps + row] : row;
        const double angle = (double)position * (a.freq[i - t * a.pairs] * 0.15915494309189533577);
        float c, s;
        turn_of(angle - __builtin_rint(angle), c, s);
        angles[0][i] = c * a.factor, angles[1][i] = s * a.factor * a.sign;
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    if (!live) continue;
    if (turns) {
      const float *c = angles[0] + t * a.pairs, *s = angles[1] + t * a.pairs;
      if constexpr (INTER) {
        arrived(x), arrived(y);
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
          turn(x.v[2 * i], x.v[2 * i + 1], c[at / 2 + i], s[at / 2 + i]);
          turn(y.v[2 * i], y.v[2 * i + 1], c[other / 2 + i], s[other / 2 + i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < W; ++i) turn(x.v[i], y.v[i], c[at + i], s[at + i]);
      }
    }
    if (few) {
      for (int i = a.rot; i < a.D; ++i) to[i] = from[i];
    } else {
      store<STREAM>(to + at, x), store<STREAM>(to + other, y);
    }
  }
}

// ---- host ---------------------------------------------------------------------------------

gbmw_status check_heads(const char* name, const void* ptr, int size, const int64_t (&s)[3]) {
  if (!ptr) return fail(GBMW_ERR_INVALID_ARG, "%s is null", name);
  if ((uintptr_t)ptr % (unsigned)size) return fail(GBMW_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] > (1ll << 40)) return fail(GBMW_ERR_INVALID_ARG, "%s: stride %lld", name, (long long)s[i]);
  return GBMW_OK;
}

// Whether no two elements of [B][L][H][D] are at one place, by strides that hold one axis inside the next.
bool apart(int B, int L, int H, int D, const int64_t (&s)[3]) {
  struct Axis {
    int64_t n, s;
  } axes[3] = {{B, s[0]}, {L, s[1]}, {H, s[2]}};
  std::sort(axes, axes + 3, [](const Axis& x, const Axis& y) { return x.s < y.s; });
  int64_t reach = D;   // elements from the first to behind the last of the axes so far
  for (const Axis& x : axes) {
    if (x.n <= 1) continue;
    if (x.s < reach) return false;
    reach += (x.n - 1) * x.s;
  }
  return true;
}

template <typename T, int W, bool INTER, bool STREAM>
void launch_rotary(const RotaryArgs& a, hipStream_t st) {
  const dim3 grid((a.units + 3) / 4), block(256);
  if (a.tokens == 1) hipLaunchKernelGGL((k_rotary<T, W, INTER, STREAM, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_rotary<T, W, INTER, STREAM, false>), grid, block, 0, st, a);
}

template <typename T, int W, bool STREAM>
void launch_rotary(const RotaryArgs& a, bool interleaved, hipStream_t st) {
  if constexpr (W > 1) {
    if (interleaved) return launch_rotary<T, W, true, STREAM>(a, st);
  }
  launch_rotary<T, W, false, STREAM>(a, st);
}

template <typename T>
gbmw_status launch_rotary(const RotaryArgs& a, int W, bool interleaved, bool stream, hipStream_t st) {
  constexpr int V = kVec<T>;
  if (W == V && stream) launch_rotary<T, V, true>(a, interleaved, st);
  else if (W == V) launch_rotary<T, V, false>(a, interleaved, st);
  else if (V == 8 && W == 4) launch_rotary<T, 4, false>(a, interleaved, st);
  else if (W == 2) launch_rotary<T, 2, false>(a, interleaved, st);
  else launch_rotary<T, 1, false>(a, interleaved, st);
  HIP_TRY(hipGetLastError());
  return GBMW_OK;
}

gbmw_status rotary(const gbmw_rotary_problem* p, float sign) {
  gbmw_detail::clear_error();
  if (!p) return fail(GBMW_ERR_INVALID_ARG, "null problem");
  if (!known_dtype(p->dtype)) return fail(GBMW_ERR_INVALID_ARG, "dtype=%d", p->dtype);
  if (p->B < 0 || p->L < 0) return fail(GBMW_ERR_INVALID_ARG, "negative size");
  if (p->Hq < 1 || p->Hk < 0 || (int64_t)p->Hq + p->Hk > (1 << 20))
    return fail(GBMW_ERR_INVALID_ARG, "Hq=%d, Hk=%d", p->Hq, p->Hk);
  if (p->D < 1 || p->D > 2 * kMostPairs) return fail(GBMW_ERR_INVALID_ARG, "D=%d not in 1..%d", p->D, 2 * kMostPairs);
  if (p->rot < 0 || p->rot > p->D || p->rot % 2) return fail(GBMW_ERR_INVALID_ARG, "rot=%d is odd or not in 0..D", p->rot);
  if (p->interleaved != 0 && p->interleaved != 1) return fail(GBMW_ERR_INVALID_ARG, "interleaved=%d", p->interleaved);
  if (!std::isfinite(p->factor)) return fail(GBMW_ERR_INVALID_ARG, "factor=%g", (double)p->factor);
  if ((int64_t)p->B * p->L > INT32_MAX - 64) return fail(GBMW_ERR_INVALID_ARG, "too many rows: B=%d, L=%d", p->B, p->L);
  if (p->B == 0 || p->L == 0) return GBMW_OK;
  const int size = element_size(p->dtype);
  if (p->rot > 0 && (!p->freq || (uintptr_t)p->freq % 8)) return fail(GBMW_ERR_INVALID_ARG, "freq is null or not aligned to a double");
  if ((uintptr_t)p->positions % 4) return fail(GBMW_ERR_INVALID_ARG, "positions are not aligned to an int32");
  if (p->position_stride < 0 || p->position_stride > (1ll << 40))
    return fail(GBMW_ERR_INVALID_ARG, "positions: stride %lld", (long long)p->position_stride);
  if ((uintptr_t)p->len % 4) return fail(GBMW_ERR_INVALID_ARG, "len is not aligned to an int32");
  CHECK(check_heads("q", p->q, size, p->q_stride));
  CHECK(check_heads("q_out", p->q_out, size, p->q_out_stride));
  if (!apart(p->B, p->L, p->Hq, p->D, p->q_out_stride)) return fail(GBMW_ERR_INVALID_ARG, "q_out: elements overlap");
  bool in_place = p->q == p->q_out;
  if (in_place && !std::equal(p->q_stride, p->q_stride + 3, p->q_out_stride))
    return fail(GBMW_ERR_INVALID_ARG, "q_out is q, with other strides");
  if (p->Hk) {
    CHECK(check_heads("k", p->k, size, p->k_stride));
    CHECK(check_heads("k_out", p->k_out, size, p->k_out_stride));
    if (!apart(p->B, p->L, p->Hk, p->D, p->k_out_stride)) return fail(GBMW_ERR_INVALID_ARG, "k_out: elements overlap");
    if (p->k == p->k_out && !std::equal(p->k_stride, p->k_stride + 3, p->k_out_stride))
      return fail(GBMW_ERR_INVALID_ARG, "k_out is k, with other strides");
    if (p->k_out == p->q_out) return fail(GBMW_ERR_INVALID_ARG, "q_out and k_out are one array");
    if (p->q_out == p->k) return fail(GBMW_ERR_INVALID_ARG, "q_out is k");   // of which heads are still to be read
    if (p->k_out == p->q) return fail(GBMW_ERR_INVALID_ARG, "k_out is q");
    in_place = in_place && p->k == p->k_out;
  }
  RotaryArgs a{};
  a.B = p->B, a.L = p->L, a.Hq = p->Hq, a.H = p->Hq + p->Hk, a.D = p->D, a.rot = p->rot, a.pairs = p->rot / 2;
  a.factor = p->factor, a.sign = sign, a.freq = p->freq, a.positions = p->positions, a.len = p->len, a.ps = p->position_stride;
  a.q = p->q, a.k = p->k, a.qo = p->q_out, a.ko = p->k_out;
  std::copy(p->q_stride, p->q_stride + 3, a.qs), std::copy(p->k_stride, p->k_stride + 3, a.ks);
  std::copy(p->q_out_stride, p->q_out_stride + 3, a.qos), std::copy(p->k_out_stride, p->k_out_stride + 3, a.kos);
  // the widest piece of up to 16 bytes that what turns has room for
  const int through = in_place ? 0 : p->D - p->rot, unit = p->interleaved ? p->rot : p->rot / 2;
  if (unit == 0 && through == 0) return GBMW_OK;
  int W = 16 / size;
  while ((unit && W > unit) || W > p->D) W /= 2;
  a.turning = p->interleaved ? (unit + 2 * W - 1) / (2 * W) : (unit + W - 1) / W;
  a.pieces = a.turning + (through + 2 * W - 1) / (2 * W);
  // a wave has as many heads as its lanes have pieces for, of several tokens where one has fewer
  const int64_t tokens = (int64_t)p->B * p->L;
  const int items = 64 / std::min(64, a.pieces);
  a.tokens = std::max(1, std::min(items / a.H, kTable / std::max(1, a.pairs)));
  a.heads = a.tokens > 1 ? a.H : std::min(a.H, items);
  a.chunks = (a.H + a.heads - 1) / a.heads;
  a.heads = (a.H + a.chunks - 1) / a.chunks;
  a.of_chunk = divisor(a.chunks), a.of_head = divisor(a.H), a.of_row = divisor(p->L), a.of_pairs = divisor(std::max(1, a.pairs));
  // Loads and stores pass the cache by where it would not hold the results for who reads them next, and where a wave's
  // stores are whole lines of it.  With the attention that reads them, bytes read and written, through the cache and past
  // it: 8192 rows of 40 heads of 128 (168 MB) 212 and 220 us, 12288 (252 MB) 325 and 322, 16384 (336 MB) 431 and 427;
  // 8192 of 80 heads (336 MB) 359 and 349, the call alone 66 and 55.
  const int line = 128 / size;
  auto lines = [line](const void* x, const int64_t (&s)[3]) {
    return (uintptr_t)x % 128 == 0 && s[0] % line == 0 && s[1] % line == 0 && s[2] % line == 0;
  };
  const bool stream = tokens * a.H * (p->rot + through) >= (1ll << 27) / size && p->rot % (2 * line) == 0 &&
                      through % (2 * line) == 0 && lines(p->q_out, p->q_out_stride) &&
                      (!p->Hk || lines(p->k_out, p->k_out_stride));
  hipStream_t st = (hipStream_t)p->stream;
  const int64_t per = kMostWaves / a.chunks * a.tokens;   // tokens of a launch
  for (int64_t begin = 0; begin < tokens; begin += per) {
    a.begin = (int)begin, a.units = (unsigned)((std::min(per, tokens - begin) + a.tokens - 1) / a.tokens * a.chunks);
    if (p->dtype == GBMW_F32) CHECK(launch_rotary<float>(a, W, p->interleaved, stream, st));
    else if (p->dtype == GBMW_F16) CHECK(launch_rotary<f16>(a, W, p->interleaved, stream, st));
    else CHECK(launch_rotary<bf16>(a, W, p->interleaved, stream, st));
  }
  return GBMW_OK;
}

}  // namespace
}  // namespace gbmw

using namespace gbmw;

extern "C" gbmw_status gbmw_rotary_forward(const gbmw_rotary_problem* p) { return rotary(p, 1.0f); }
extern "C" gbmw_status gbmw_rotary_backward(const gbmw_rotary_problem* p) { return rotary(p, -1.0f); }

extern "C" gbmw_status gbmw_rotary_frequencies(int32_t rot, double theta, int32_t scaling, double by, double original,
                                               double slow, double fast, double* freq) {
  gbmw_detail::clear_error();
  if (rot < 0 || rot > 2 * kMostPairs || rot % 2) return fail(GBMW_ERR_INVALID_ARG, "rot=%d", rot);
  if (rot && !freq) return fail(GBMW_ERR_INVALID_ARG, "freq is null");
  if (!(theta > 0.0) || !std::isfinite(theta)) return fail(GBMW_ERR_INVALID_ARG, "theta=%g", theta);
  if (scaling < GBMW_ROTARY_NONE || scaling > GBMW_ROTARY_RAMP) return fail(GBMW_ERR_INVALID_ARG, "scaling=%d", scaling);
  if (scaling != GBMW_ROTARY_NONE && (!(by > 0.0) || !std::isfinite(by))) return fail(GBMW_ERR_INVALID_ARG, "by=%g", by);
  if (scaling == GBMW_ROTARY_BASE && rot == 2) return fail(GBMW_ERR_INVALID_ARG, "rot=2 has one frequency, which no base scales");
  if (scaling == GBMW_ROTARY_RAMP &&
      (!(original > 0.0) || !std::isfinite(original) || !(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast)))
    return fail(GBMW_ERR_INVALID_ARG, "original=%g, slow=%g, fast=%g", original, slow, fast);
  if (scaling == GBMW_ROTARY_BASE) theta *= std::pow(by, (double)rot / (rot - 2));
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / rot);
    if (scaling == GBMW_ROTARY_LINEAR) f /= by;
    if (scaling == GBMW_ROTARY_RAMP) {
      const double turns = original * f / 6.283185307179586477, w = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
      f = w * f + (1.0 - w) * f / by;
    }
    freq[i] = f;
  }
  return GBMW_OK;
}
