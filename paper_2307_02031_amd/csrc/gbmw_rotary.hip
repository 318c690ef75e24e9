// Rotary positions of queries and keys.  Contract: include/gbmw.h.
#include "gbmw_rows.h"

using gbmw_detail::fail;

namespace gbmw {
namespace {

struct RotaryArgs {
  int B, L, Hq, H, D, rot;   // H: query and key heads
  int pairs;                 // rot / 2
  int turning, pieces;       // pieces of a head that turn, and those with the ones that are handed through
  int rounds;                // of 64 / pieces heads that a token's heads take
  int chunks, per_chunk;     // waves that share a token, rounds of each
  unsigned units;            // tokens times chunks
  float factor, sign;
  const double* freq;
  const int32_t *positions, *len;
  int64_t ps;
  const void *q, *k;
  void *qo, *ko;
  int64_t qs[3], ks[3], qos[3], kos[3];
};

// cos and sin of 2 pi x, |x| <= 1/2, by the quarter turn that x is nearest and the Taylor series of the
// rest (at most pi / 4; the first term left out is below 2^-29 of the result).
__device__ __forceinline__ void turn_of(float x, float& c, float& s) {
  const float quarter = __builtin_rintf(4.0f * x);
  const float r = 6.28318530717958648f * __builtin_fmaf(-0.25f, quarter, x), r2 = r * r;
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

constexpr int kMostPairs = 256;

// A wave has one token, or a share of its heads: it computes the token's angles, in turns and in fp64 (a
// position times a frequency loses the digits of its fraction in fp32), and every lane keeps those of its
// piece of W values (or of W values and the W that are rot / 2 further on) for all heads.
template <typename T, int W, bool INTER>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a) {
  constexpr int P = INTER ? W / 2 : W;   // pairs of a piece
  __shared__ float table[4][2][kMostPairs];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  for (unsigned unit = blockIdx.x * 4 + wave; unit < a.units; unit += gridDim.x * 4) {
  const unsigned token = unit / (unsigned)a.chunks;
  const int chunk = (int)(unit % (unsigned)a.chunks), b = (int)(token / (unsigned)a.L), row = (int)(token % (unsigned)a.L);
  if (a.len && row >= a.len[b]) continue;
  const int position = a.positions ? a.positions[b * a.ps + row] : row;
  float(*tab)[kMostPairs] = table[wave];
  for (int i = lane; i < a.pairs; i += 64) {
    const double t = (double)position * (a.freq[i] * 0.15915494309189533577);
    float c, s;
    turn_of((float)(t - __builtin_rint(t)), c, s);
    tab[0][i] = c * a.factor, tab[1][i] = s * a.factor * a.sign;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const int half = a.rot / 2;
  for (int p0 = 0; p0 < a.pieces; p0 += 64) {
    const int width = min(64, a.pieces - p0), slots = 64 / width, slot = lane / width, piece = p0 + lane % width;
    if (slot >= slots) continue;
    const bool turns = piece < a.turning;
    float c[P], s[P];
    if (turns)
#pragma unroll
      for (int i = 0; i < P; ++i) c[i] = tab[0][piece * P + i], s[i] = tab[1][piece * P + i];
    const int at = turns ? piece * W : a.rot + (piece - a.turning) * W;
    const int first = chunk * a.per_chunk * slots, last = min(a.H, first + a.per_chunk * slots);
    for (int head = first + slot; head < last; head += slots) {
      const bool key = head >= a.Hq;
      const int64_t in = key ? b * a.ks[0] + row * a.ks[1] + (head - a.Hq) * a.ks[2] : b * a.qs[0] + row * a.qs[1] + head * a.qs[2];
      const int64_t to = key ? b * a.kos[0] + row * a.kos[1] + (head - a.Hq) * a.kos[2]
                             : b * a.qos[0] + row * a.qos[1] + head * a.qos[2];
      const T* src = (const T*)(key ? a.k : a.q) + in + at;
      T* dst = (T*)(key ? a.ko : a.qo) + to + at;
      Piece<T, W> x, y;
      if (!turns && at + W > a.D) {   // the last of those handed through
        for (int i = 0; at + i < a.D; ++i) dst[i] = src[i];
        continue;
      }
      __builtin_memcpy(&x, src, sizeof(x));
      if (turns) {
        if constexpr (INTER) {
#pragma unroll
          for (int i = 0; i < P; ++i) {
            const float u = (float)x.v[2 * i], v = (float)x.v[2 * i + 1];
            x.v[2 * i] = (T)(u * c[i] - v * s[i]), x.v[2 * i + 1] = (T)(u * s[i] + v * c[i]);
          }
        } else {
          __builtin_memcpy(&y, src + half, sizeof(y));
#pragma unroll
          for (int i = 0; i < P; ++i) {
            const float u = (float)x.v[i], v = (float)y.v[i];
            x.v[i] = (T)(u * c[i] - v * s[i]), y.v[i] = (T)(u * s[i] + v * c[i]);
          }
          __builtin_memcpy(dst + half, &y, sizeof(y));
        }
      }
      __builtin_memcpy(dst, &x, sizeof(x));
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
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

template <typename T>
gbmw_status launch_rotary(const RotaryArgs& a, int W, bool interleaved, int64_t groups, hipStream_t st) {
  const dim3 grid((unsigned)groups), block(256);
  if constexpr (sizeof(T) == 2) {
    if (W == 8) {
      if (interleaved) hipLaunchKernelGGL((k_rotary<T, 8, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((k_rotary<T, 8, false>), grid, block, 0, st, a);
    }
  }
  if (W == 4) {
    if (interleaved) hipLaunchKernelGGL((k_rotary<T, 4, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_rotary<T, 4, false>), grid, block, 0, st, a);
  }
  if (W == 2) {
    if (interleaved) hipLaunchKernelGGL((k_rotary<T, 2, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_rotary<T, 2, false>), grid, block, 0, st, a);
  }
  if (W == 1) hipLaunchKernelGGL((k_rotary<T, 1, false>), grid, block, 0, st, a);
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
  if ((int64_t)p->B * p->L > INT32_MAX) return fail(GBMW_ERR_INVALID_ARG, "too many rows: B=%d, L=%d", p->B, p->L);
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
    in_place = in_place && p->k == p->k_out;
  }
  RotaryArgs a{};
  a.B = p->B, a.L = p->L, a.Hq = p->Hq, a.H = p->Hq + p->Hk, a.D = p->D, a.rot = p->rot, a.pairs = p->rot / 2;
  a.factor = p->factor, a.sign = sign, a.freq = p->freq, a.positions = p->positions, a.len = p->len, a.ps = p->position_stride;
  a.q = p->q, a.k = p->k, a.qo = p->q_out, a.ko = p->k_out;
  std::copy(p->q_stride, p->q_stride + 3, a.qs), std::copy(p->k_stride, p->k_stride + 3, a.ks);
  std::copy(p->q_out_stride, p->q_out_stride + 3, a.qos), std::copy(p->k_out_stride, p->k_out_stride + 3, a.kos);
  // the widest piece of up to 16 bytes of which what turns is a whole number
  const int through = in_place ? 0 : p->D - p->rot, unit = p->interleaved ? p->rot : p->rot / 2;
  if (unit == 0 && through == 0) return GBMW_OK;
  int W = 16 / size;
  while (unit % W) W /= 2;
  a.turning = unit / W, a.pieces = a.turning + (through + W - 1) / W;
  const int slots = 64 / std::min(64, a.pieces);
  a.rounds = (a.H + slots - 1) / slots;
  const int64_t tokens = (int64_t)p->B * p->L;
  a.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(a.rounds, 4096 / tokens));
  a.per_chunk = (a.rounds + a.chunks - 1) / a.chunks;
  a.chunks = (a.rounds + a.per_chunk - 1) / a.per_chunk;
  a.units = (unsigned)(tokens * a.chunks);
  const int64_t groups = std::min<int64_t>(1 << 20, ((int64_t)a.units + 3) / 4);
  hipStream_t st = (hipStream_t)p->stream;
  if (p->dtype == GBMW_F32) return launch_rotary<float>(a, W, p->interleaved && W > 1, groups, st);
  if (p->dtype == GBMW_F16) return launch_rotary<f16>(a, W, p->interleaved && W > 1, groups, st);
  return launch_rotary<bf16>(a, W, p->interleaved && W > 1, groups, st);
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
