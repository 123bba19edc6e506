// Norms of heads and rotation by position, of queries and keys on their own
// (include/lam.h, lam_kv_rotate) and on the way into the 4-bit cache (lam_kv_rotate_append).
//
// A head's row x of N channels with gains g becomes y = g x / sqrt(sum x^2 / N + eps), and its
// channel pair i, at position p, is turned by the angle a = p f_i:
//
//   (u, v) -> A (u cos a - v sin a, u sin a + v cos a)
//
// A lane holds eight channels, the D/8 lanes of a head lie together in a wave, and the pair's other
// channel is in the lane itself (interleaved) or in one D/2 or R/2 channels away (halves).
//
// Angles: p f is taken in binary64 with its rounding error kept, so the fraction of a turn is
// right to 2^-53 at every position; sine and cosine are the Taylor polynomials over an eighth
// of a turn either way, in float32 where the result is rounded to 16 bits.
//
// Bound by memory, a row read and written once: 65,536 rows of 40 heads of 128 channels 253 us,
// 5.3 TB/s, the rate of a copy; 131,072 rows of 32 + 8 + 8 heads into the cache 548 us, 5.2 TB/s.
// Vector instructions are active in two thirds of a SIMD's cycles there, so what is done once a row
// is not done once a head (sines and cosines by every lane for its own channels: 372 and 1,025 us).
#include <algorithm>

#include "kv.h"
#include "kv_rotate.h"
#include "kv_rows.h"
#include "lam_internal.h"
#include "wave.h"

namespace lam {
namespace {

// Where the pair's other channel is: a lane a whole number of lanes away, the lane itself, anywhere.
enum Pairing { kHalves = 0, kInterleaved = 1, kHalvesAnywhere = 2 };

// The angle of position pos at freq radians a position, in turns from the nearest quarter turn.
__device__ __forceinline__ double turns_of(int32_t pos, double freq, int* quarter) {
  constexpr double kInv = 0.15915494309189535, kInvLo = -9.839338337591243e-18;   // 1 / (2 pi)
  const double p = (double)pos, hi = p * freq, lo = fma(p, freq, -hi);
  const double t = hi * kInv, e = fma(hi, kInv, -t) + fma(hi, kInvLo, lo * kInv);
  const double n = rint(4.0 * t);
  *quarter = (int)(n - 4.0 * rint(0.25 * n)) & 3;
  return fma(-0.25, n, t) + e;
}

// From an eighth of a turn either way to the whole circle.
template <typename F>
__device__ __forceinline__ void to_quarter(int quarter, F* c, F* s) {
  const F a = *c, b = *s;
  *c = quarter & 1 ? b : a;
  *s = quarter & 1 ? a : b;
  *c = quarter == 1 || quarter == 2 ? -*c : *c;
  *s = quarter & 2 ? -*s : *s;
}

// (2 pi)^k / k! with the signs of the series
__device__ __forceinline__ void sin_cos(int32_t pos, double freq, double* c, double* s) {
  int quarter;
  const double r = turns_of(pos, freq, &quarter), z = r * r;
  double a = -0.7181223017785006, b = 0.28200596845579123;   // the next terms: 5e-17, 2e-18
  a = fma(a, z, 3.819952584848282), b = fma(b, z, -1.714390711088672);
  a = fma(a, z, -15.09464257682299), b = fma(b, z, 7.903536371318469);
  a = fma(a, z, 42.058693944897655), b = fma(b, z, -26.4262567833744);
  a = fma(a, z, -76.70585975306139), b = fma(b, z, 60.24464137187666);
  a = fma(a, z, 81.60524927607506), b = fma(b, z, -85.45681720669373);
  a = fma(a, z, -41.34170224039976), b = fma(b, z, 64.9393940226683);
  a = fma(a, z, 6.283185307179586), b = fma(b, z, -19.739208802178716);
  *s = a * r;
  *c = fma(b, z, 1.0);
  to_quarter(quarter, c, s);
}

__device__ __forceinline__ void sin_cos(int32_t pos, double freq, float* c, float* s) {
  int quarter;
  const float r = (float)turns_of(pos, freq, &quarter), z = r * r;
  float a = 42.058693944897655f, b = -26.4262567833744f;   // the next terms: 2e-9, 1e-10
  a = fmaf(a, z, -76.70585975306139f), b = fmaf(b, z, 60.24464137187666f);
  a = fmaf(a, z, 81.60524927607506f), b = fmaf(b, z, -85.45681720669373f);
  a = fmaf(a, z, -41.34170224039976f), b = fmaf(b, z, 64.9393940226683f);
  a = fmaf(a, z, 6.283185307179586f), b = fmaf(b, z, -19.739208802178716f);
  *s = a * r;
  *c = fmaf(b, z, 1.0f);
  to_quarter(quarter, c, s);
}

// Which pairs a lane's eight channels from c0 on belong to.
template <int MODE>
struct Lane {
  int c0, pairs;
  __device__ __forceinline__ bool turned(int e) const { return MODE == kInterleaved ? (c0 + e) / 2 < pairs : c0 + e < 2 * pairs; }
  __device__ __forceinline__ bool minus(int e) const { return MODE == kInterleaved ? (e & 1) == 0 : c0 + e < pairs; }
  __device__ __forceinline__ int pair(int e) const {
    if (!turned(e)) return 0;
    return MODE == kInterleaved ? (c0 + e) / 2 : c0 + e < pairs ? c0 + e : c0 + e - pairs;
  }
  // the pair's other channel; a channel that is not turned has none and stands in itself
  __device__ __forceinline__ int other(int e) const {
    if (!turned(e)) return c0 + e;
    return MODE == kInterleaved ? (c0 + e) ^ 1 : c0 + e < pairs ? c0 + e + pairs : c0 + e - pairs;
  }
};

template <bool BF16>
__device__ __forceinline__ float gain_at(const RotateHeads& h, int c) {
  if (h.gain_f32) return static_cast<const float*>(h.gain)[c];
  const uint16_t g = static_cast<const uint16_t*>(h.gain)[c];
  return BF16 ? __uint_as_float((uint32_t)g << 16) : (float)__builtin_bit_cast(_Float16, g);
}

// Gains of eight channels from c on.
template <bool BF16>
__device__ __forceinline__ void gains8(const RotateHeads& h, int c, float g[8]) {
  if (h.gain_wide && h.gain_f32) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const kv_f4 w = reinterpret_cast<const kv_f4*>(static_cast<const float*>(h.gain) + c)[j];
#pragma unroll
      for (int i = 0; i < 4; ++i) g[4 * j + i] = w[i];
    }
  } else if (h.gain_wide) {
    unpack8<BF16>(*reinterpret_cast<const kv_u4*>(static_cast<const uint16_t*>(h.gain) + c), g);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = gain_at<BF16>(h, c + e);
  }
}

// Of a lane's channels and of their pairs' others.
template <int MODE, bool BF16>
__device__ __forceinline__ void gains(const RotateHeads& h, const Lane<MODE>& at, float g[8], float go[8]) {
  gains8<BF16>(h, at.c0, g);
  if constexpr (MODE == kHalves) {
    gains8<BF16>(h, at.other(0), go);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) go[e] = MODE == kInterleaved ? g[e ^ 1] : gain_at<BF16>(h, at.other(e));
  }
}

// A wave's LDS accesses are in order: what its lanes have written is there for the others.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The raw other channels of a lane's eight, given its own (interleaved, also of channels that are not
// turned: their neighbours).  pass: 16 bytes of LDS for each lane, for
// pairs whose channels are no whole number of lanes apart (read from memory once more, 41,569 rows of
// 108 heads of 64 channels and 20 pairs took 384 us, so 233).
template <int MODE, int L>
__device__ __forceinline__ kv_u4 others(const Lane<MODE>& at, kv_u4 own, kv_u4* pass) {
  kv_u4 w = own;
  const int lane = (int)threadIdx.x & 63, group = lane & ~(L - 1);
  if constexpr (MODE == kHalves) {
    const int from = group + at.other(0) / 8;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (uint32_t)__shfl((int)own[j], from);
  } else if constexpr (MODE == kInterleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_alignbit(own[j], own[j], 16);
  } else {
    wave_lds_order();
    pass[lane] = own;
    wave_lds_order();
    if (at.pairs & 1) {
      const uint16_t* const c = reinterpret_cast<const uint16_t*>(pass + group);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = (uint32_t)c[at.other(2 * j)] | ((uint32_t)c[at.other(2 * j + 1)] << 16);
    } else {
      const uint32_t* const c = reinterpret_cast<const uint32_t*>(pass + group);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = c[at.other(2 * j) / 2];
    }
  }
  return w;
}

template <bool BF16>
__device__ __forceinline__ kv_u4 pack8(const float y[8]) {
  kv_u4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16) w[j] = __builtin_bit_cast(uint32_t, kv_b2{(__bf16)y[2 * j], (__bf16)y[2 * j + 1]});
    else w[j] = __builtin_bit_cast(uint32_t, kv_h2{(_Float16)y[2 * j], (_Float16)y[2 * j + 1]});
  }
  return w;
}

__device__ __forceinline__ void store_raw8(void* p, int64_t at, bool wide, kv_u4 w) {
  uint16_t* h = static_cast<uint16_t*>(p) + at;
  if (wide) {
    *reinterpret_cast<kv_u4*>(h) = w;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) h[2 * j] = (uint16_t)w[j], h[2 * j + 1] = (uint16_t)(w[j] >> 16);
}

// A pair's two terms, and a value times its gain, can leave float32's range though what comes of them, by
// the other term or by the norm, is well inside: gains come 2^3 smaller and results are multiplied by it at the end.
constexpr float kDown = 0x1p-3f, kUp = 0x1p3f;

// 1 / sqrt(sum of squares / norm_dim + eps) of a head's eight channels a lane, in float32 where that is well inside
// its range, else (for all heads of the wave) in binary64.  Then float32 may hold neither the factor of bfloat16
// rows nor their product with a gain: true is returned, and its power of two, `by`, is for the channels themselves.
// (Float16 rows get there by zeros or by eps alone, and what a factor beyond float32 multiplies is 0.)
template <int L, bool BF16>
__device__ __forceinline__ bool norm_of(const RotateArgs& a, const float u[8], float* r, int* by) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(u[e], u[e], s);
  s = group_sum_f32<L>(s);
  const float mean = fmaf(s, (float)a.inv_dim, (float)a.eps);
  *r = __builtin_amdgcn_rsqf(mean);
  if (!__any(!(s >= 1e-24f && mean <= 1e37f))) return false;
  double d = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) d = fma((double)u[e], (double)u[e], d);
  const double n = __builtin_amdgcn_rsq(fma(group_sum_f64<L>(d), a.inv_dim, a.eps));
  if constexpr (BF16) {
    *r = (float)__builtin_amdgcn_frexp_mant(n);
    *by = __builtin_amdgcn_frexp_exp(n);
    return true;
  } else {
    *r = n > 1e37 ? 1e37f : (float)n;   // (times kUp still in range)
    return false;
  }
}

// Eight channels times 2^by.
__device__ __forceinline__ void scale8(float x[8], int by) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = ldexpf(x[e], by);
}

// ------------------------------------------------------------------ rows in 16 bits
// Sines and cosines of a row of at most 8 L channels.
template <int L>
struct __align__(16) RowAngles {
  float c[4 * L], s[4 * L];
};

// 16 bytes a lane, where others() needs them.
template <int MODE>
struct Pass {
  kv_u4 w[MODE == kHalvesAnywhere ? 64 : 1];
};

// A wave norms and turns a row, or where rows are few a part of its heads, 64/L heads at a time.
// What a lane needs of the sines and cosines for all heads lies in its registers, multiplied by
// the gains.  kinds: of the queries alone, or of the keys as well.
template <int L, bool BF16, int MODE>
__device__ __forceinline__ void rotate_row(const RotateArgs& a, int kinds, int64_t row, int part, const RowAngles<L>& angles,
                                           kv_u4* pass) {
  constexpr int kAtOnce = 64 / L;
  const int lane = threadIdx.x & 63, sub = lane % L, slot = lane / L;
  const Lane<MODE> at{8 * sub, a.pairs};
  const bool live = at.c0 < a.dim;
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool turned = live && at.turned(e);
    const int i = turned ? at.pair(e) : 0;
    cs[e] = turned ? kDown * angles.c[i] : kDown;
    sn[e] = turned ? kDown * (at.minus(e) ? -angles.s[i] : angles.s[i]) : 0.0f;
  }
  int before = 0;   // rounds of the kind before
#pragma unroll 1
  for (int kind = 0; kind < kinds; ++kind) {
    const RotateHeads& h = a.h[kind];
    const int rounds = (h.heads + kAtOnce - 1) / kAtOnce;
    int i = (part - before % a.parts + a.parts) % a.parts;
    before += rounds;
    if (i >= rounds) continue;
    auto head_of = [&](int i) { return i * kAtOnce + slot; };
    auto row_of = [&](int i) { return h.x + row * h.x_row + (int64_t)min(head_of(i), h.heads - 1) * h.x_head; };
    auto load = [&](int i) {
      kv_u4 w{};
      if (live) w = load_raw8(row_of(i), at.c0, h.x_wide);
      return w;
    };
    kv_u4 next = load(i);
    float ga[8], gb[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) ga[e] = cs[e], gb[e] = sn[e];
    if (h.gain && live) {
      float g[8], go[8];
      gains<MODE, BF16>(h, at, g, go);
#pragma unroll
      for (int e = 0; e < 8; ++e) ga[e] *= g[e], gb[e] *= go[e];
    }
    for (; i < rounds; i += a.parts) {
      const kv_u4 own = next;
      const kv_u4 other = others<MODE, L>(at, own, pass);
      if (i + a.parts < rounds) next = load(i + a.parts);
      float u[8], v[8], y[8], r = 1.0f;
      int by = 0;
      unpack8<BF16>(own, u);
      const bool far = h.gain && norm_of<L, BF16>(a, u, &r, &by);
      unpack8<BF16>(other, v);
      if (far) scale8(u, by), scale8(v, by);
      r *= kUp;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float straight = u[e] * ga[e];
        y[e] = (at.turned(e) ? fmaf(v[e], gb[e], straight) : straight) * r;
      }
      if (live && head_of(i) < h.heads)
        store_raw8(h.y, row * h.y_row + (int64_t)head_of(i) * h.y_head + at.c0, h.y_wide, pack8<BF16>(y));
    }
  }
}

// Few heads leave most of a wave idle while it makes a row's angles and its last heads: there it
// takes four rows, and the heads of all of them in turn.
constexpr int kFewRows = 4;

// i / by for i < 512, by <= 128, inverse = 65536 / by + 1
__device__ __forceinline__ int small_div(int i, uint32_t inverse) { return (int)((uint32_t)i * inverse >> 16); }

// The heads of n rows from row0 on.  none: bit i: row i is of no sequence and gets 0.
template <int L, bool BF16, int MODE>
__device__ __forceinline__ void rotate_few(const RotateArgs& a, int kinds, int64_t row0, int n, uint32_t none,
                                           const RowAngles<L>* angles, kv_u4* pass) {
  constexpr int kAtOnce = 64 / L;
  const int lane = threadIdx.x & 63, sub = lane % L, slot = lane / L;
  const Lane<MODE> at{8 * sub, a.pairs};
  const bool live = at.c0 < a.dim;
#pragma unroll 1
  for (int kind = 0; kind < kinds; ++kind) {
    const RotateHeads& h = a.h[kind];
    if (h.heads == 0) continue;
    const uint32_t inverse = 65536u / (uint32_t)h.heads + 1u;
    const int items = n * h.heads;
    float g[8], go[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = go[e] = 1.0f;
    if (h.gain && live) gains<MODE, BF16>(h, at, g, go);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] *= kDown, go[e] *= at.minus(e) ? -kDown : kDown;
    auto load = [&](int i) {
      const int item = min(i + slot, items - 1), r = small_div(item, inverse);
      kv_u4 w{};
      if (live) w = load_raw8(h.x + (row0 + r) * h.x_row + (int64_t)(item - r * h.heads) * h.x_head, at.c0, h.x_wide);
      return w;
    };
    kv_u4 next = load(0);
    for (int i = 0; i < items; i += kAtOnce) {
      const kv_u4 own = next, other = others<MODE, L>(at, own, pass);
      if (i + kAtOnce < items) next = load(i + kAtOnce);
      const int item = min(i + slot, items - 1), r = small_div(item, inverse);
      float u[8], v[8], y[8], norm = 1.0f;
      int by = 0;
      unpack8<BF16>(own, u);
      const bool far = h.gain && norm_of<L, BF16>(a, u, &norm, &by);
      unpack8<BF16>(other, v);
      if (far) scale8(u, by), scale8(v, by);
      norm *= kUp;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = u[e] * g[e];
      if (MODE != kHalves || at.turned(0)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          kv_f4 c, t;
          if constexpr (MODE == kHalves) {   // all eight are turned or none
            c = *reinterpret_cast<const kv_f4*>(angles[r].c + at.pair(0) + 4 * j);
            t = *reinterpret_cast<const kv_f4*>(angles[r].s + at.pair(0) + 4 * j);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = angles[r].c[at.pair(4 * j + e)], t[e] = angles[r].s[at.pair(4 * j + e)];
          }
#pragma unroll
          for (int e = 4 * j; e < 4 * j + 4; ++e)
            if (MODE == kHalves || at.turned(e)) y[e] = fmaf(v[e] * go[e], t[e - 4 * j], y[e] * c[e - 4 * j]);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= norm;
      kv_u4 w = pack8<BF16>(y);
      if ((none >> r) & 1u) w = kv_u4{0, 0, 0, 0};
      if (live && i + slot < items)
        store_raw8(h.y, (row0 + r) * h.y_row + (int64_t)(item - r * h.heads) * h.y_head + at.c0, h.y_wide, w);
    }
  }
}

// (Held to seven waves a SIMD: else halves take 78 registers for the few rows that norm_of finds out of range, and
// 65,536 rows of 4 + 1 heads of 128 channels 39 us for 38.)
template <int L, bool BF16, int MODE>
__global__ __launch_bounds__(kKvThreads, MODE == kHalvesAnywhere ? 5 : 7) void k_kv_rotate_few(RotateArgs a) {
  __shared__ RowAngles<L> angles[kKvThreads / 64][kFewRows];
  __shared__ Pass<MODE> pass[kKvThreads / 64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row0 = ((int64_t)blockIdx.x * (kKvThreads / 64) + wave) * kFewRows;
  if (row0 >= a.rows) return;
  const int n = (int)min((int64_t)kFewRows, a.rows - row0);
  const uint32_t inverse = a.pairs ? 65536u / (uint32_t)a.pairs + 1u : 0u;
  for (int i = threadIdx.x & 63; i < n * a.pairs; i += 64) {
    const int r = small_div(i, inverse), pair = i - r * a.pairs;
    float c, s;
    sin_cos(a.positions[row0 + r], a.freq[pair], &c, &s);
    angles[wave][r].c[pair] = c * a.amplitude;
    angles[wave][r].s[pair] = s * a.amplitude;
  }
  wave_lds_order();
  rotate_few<L, BF16, MODE>(a, 2, row0, n, 0, angles[wave], pass[wave].w);
}

template <int L, bool BF16, int MODE>
__global__ __launch_bounds__(kKvThreads) void k_kv_rotate(RotateArgs a) {
  __shared__ RowAngles<L> angles[kKvThreads / 64];
  __shared__ Pass<MODE> pass[kKvThreads / 64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t id = blockIdx.x * (kKvThreads / 64) + wave;
  const int64_t row = id / (uint32_t)a.parts;
  if (row >= a.rows) return;
  for (int i = threadIdx.x & 63; i < a.pairs; i += 64) {   // a lane makes a pair's sine and cosine
    float c, s;
    sin_cos(a.positions[row], a.freq[i], &c, &s);
    angles[wave].c[i] = c * a.amplitude;
    angles[wave].s[i] = s * a.amplitude;
  }
  wave_lds_order();
  rotate_row<L, BF16, MODE>(a, 2, row, (int)(id % (uint32_t)a.parts), angles[wave], pass[wave].w);
}

// ------------------------------------------------------------------ rows into the cache
// x rounded to float32 so that it lies on the same side of every number of fewer bits: to the
// odd-numbered neighbour where it is none itself.  What is rounded again, to codes, is then rounded as x is.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  const double d = x - (double)f;
  uint32_t b = __float_as_uint(f);
  if (fabs(d) > 0.0 && !(b & 1u) && fabsf(f) > 1e-30f) b += (d > 0.0) == (f > 0.0f) ? 1u : 0xffffffffu;
  return __uint_as_float(b);
}

// Eight values so.  Codes and scales change at numbers of two fraction bits: where no value is next
// to one, the nearest float32 does as well.
__device__ __forceinline__ void to_odd8(const double y[8], float x[8]) {
  uint32_t least = 0xffffffffu;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = (float)y[e];
    least = min(least, __float_as_uint(x[e]) << 11);
  }
  if (__any(least == 0)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = to_odd(y[e]);
  }
}

// 1 / sqrt(a) to about 2^-52, for a > 0.
__device__ __forceinline__ double inverse_root(double a) {
  double y = __builtin_amdgcn_rsq(a);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-a * y, y, 1.0), y);
  return y;
}

struct AppendArgs {
  KvArgs c;
  int quads;              // of a sequence, where all have as many rows
  uint32_t v_blocks;      // workgroups of values, those of rows after them
  RotateArgs r;
  RowArgs v;
  lam_kv_slots weights, positions;
  const int32_t* first;
  uint32_t* status;
};

// Values as lam_kv_append has them, by quads of slots, D/8 lanes a quad and head.
template <int D, bool BF16>
__device__ __forceinline__ void append_values(const AppendArgs& g) {
  constexpr int kLanes = D / 8;
  const KvArgs& a = g.c;
  const uint32_t item = blockIdx.x * (kKvThreads / kLanes) + threadIdx.x / kLanes;
  const int sub = threadIdx.x % kLanes;
  const int h = (int)(item % (uint32_t)a.heads);
  const Quad q = quad_at<D>(a, g.quads, item / (uint32_t)a.heads, h);
  bool bad = false, over = false;
  if (q.base) {
    kv_u4 raw[4];
    uint32_t w[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // a slot that is not the call's repeats one that is
      const int64_t row = q.row + ((q.rows >> i) & 1u ? i : __builtin_ctz(q.rows));
      raw[i] = load_raw8(g.v.p, row * g.v.row + h * g.v.head + 8 * sub, g.v.wide);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[8];
      unpack8<BF16>(raw[i], x);
      w[i] = quantize8(x, &b[i], &bad, &over);
    }
    put_values<D>(q, 1 << a.page_shift, sub, w, b);
    put_slots(a, q, h, sub, g.weights, g.positions, g.first);
  }
  if (g.status) count_quad(a, q, sub, bad, over, g.status);
}

// What a row's keys are turned by: of every channel the factors of the channel itself and of its
// pair's other one, gains and amplitude in them.
template <int D>
struct __align__(16) Factors {
  double own[D], other[D];
};

// Where a row's token lies.
struct Token {
  int32_t pos;     // its position
  int t;           // its place in the page
  uint8_t* page;   // null: no place
};

// The keys of a row, by a wave (or a part of them, from round i on), 64 / (D/8) heads at a time, in
// binary64, which vector units of this chip run at float32's rate, so that no code is decided by a
// rounding on the way.
template <int D, bool BF16, int MODE>
__device__ __forceinline__ void append_keys(const AppendArgs& g, int64_t row, int i, const Token& token,
                                            const Factors<D>& f, kv_u4* pass) {
  constexpr int kLanes = D / 8, kAtOnce = 64 / kLanes;
  const KvArgs& a = g.c;
  const RotateArgs& r = g.r;
  const RotateHeads& kh = r.h[1];
  const int lane = threadIdx.x & 63, sub = lane % kLanes, slot = lane / kLanes, T = 1 << a.page_shift;
  const Lane<MODE> at{8 * sub, r.pairs};
  bool bad = false, over = false;
  auto row_of = [&](int i) { return kh.x + row * kh.x_row + (int64_t)min(i * kAtOnce + slot, a.heads - 1) * kh.x_head; };
  kv_u4 next = load_raw8(row_of(i), at.c0, kh.x_wide);
  for (; i * kAtOnce < a.heads; i += r.parts) {
    const kv_u4 own = next;
    kv_u4 other = others<MODE, kLanes>(at, own, pass);
    if constexpr (MODE == kInterleaved) {   // what is not turned stands in itself: 0 times a neighbour may be NaN
#pragma unroll
      for (int j = 0; j < 4; ++j) other[j] = at.turned(2 * j) ? other[j] : own[j];
    }
    next = load_raw8(row_of(i + r.parts), at.c0, kh.x_wide);
    float u[8], v[8], x[8];
    unpack8<BF16>(own, u);
    unpack8<BF16>(other, v);
    double y[8], n = 1.0;
    if (kh.gain) {
      double ss = 0.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fma((double)u[e], (double)u[e], ss);
      n = inverse_root(fma(group_sum_f64<kLanes>(ss), r.inv_dim, r.eps));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fma((double)v[e], f.other[at.c0 + e], (double)u[e] * f.own[at.c0 + e]) * n;
    to_odd8(y, x);
    const int h = i * kAtOnce + slot;
    if (h < a.heads) {
      uint32_t b;
      const uint32_t w = quantize8(x, &b, &bad, &over);
      uint8_t* const base = token.page + (int64_t)h * KvLayout<D>::head_bytes(T);
      put_key<D>(base, T, token.t, sub, w, b);
    }
  }
  if (g.status) {
    count_in(g.status, 0, bad);
    count_in(g.status, 1, over);
  }
}

// A row's token, by all lanes of a wave; false: of no sequence.
template <int D>
__device__ __forceinline__ bool row_token(const KvArgs& a, int64_t row, const int32_t* first, Token* token) {
  int s;
  if (!a.starts) {
    s = (int)((uint32_t)row / (uint32_t)a.per_seq);
  } else {
    s = -1;
    for (int b = 0; b < a.n_seqs; b += 64) {
      const int mine = b + (int)(threadIdx.x & 63);
      const unsigned long long in = __ballot(mine < a.n_seqs && a.start(min(mine, a.n_seqs)) <= row);
      if (in == 0) break;
      s = b + (int)__popcll(in) - 1;
      if (~in) break;
    }
    if (s < 0 || row >= a.start(s + 1)) return false;
  }
  const int64_t begin = a.start(s), at = a.lengths[s] - a.start(s + 1) + row;   // its slot
  token->pos = (int32_t)(first ? first[s] + (row - begin) : at);
  token->t = (int)(at & ((1 << a.page_shift) - 1));
  token->page = nullptr;
  if (at >= 0 && (at >> a.page_shift) < a.table_cols) {
    const int64_t page = a.page(s, (int)(at >> a.page_shift));
    if (page >= 0) token->page = a.head_page(page, 0, KvLayout<D>::head_bytes(1 << a.page_shift));
  }
  return true;
}

// What four rows' keys are turned by, the amplitude in it.
template <int D>
struct __align__(16) RowTurns {
  double c[D / 2], s[D / 2];
};

// append_keys for the keys of n rows from row0 on, the heads of all of them in turn.
template <int D, bool BF16, int MODE>
__device__ __forceinline__ void append_few(const AppendArgs& g, int64_t row0, int n, const Token* tokens,
                                           const RowTurns<D>* turns, kv_u4* pass) {
  constexpr int kLanes = D / 8, kAtOnce = 64 / kLanes;
  const RotateArgs& a = g.r;
  const RotateHeads& h = a.h[1];
  const int lane = threadIdx.x & 63, sub = lane % kLanes, slot = lane / kLanes, T = 1 << g.c.page_shift;
  const Lane<MODE> at{8 * sub, a.pairs};
  const uint32_t inverse = 65536u / (uint32_t)h.heads + 1u;
  const int items = n * h.heads;
  bool bad = false, over = false;
  float gn[8], go[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) gn[e] = go[e] = 1.0f;
  if (h.gain) gains<MODE, BF16>(h, at, gn, go);
#pragma unroll
  for (int e = 0; e < 8; ++e) go[e] = at.minus(e) ? -go[e] : go[e];
  auto load = [&](int i) {
    const int item = min(i + slot, items - 1), r = small_div(item, inverse);
    return load_raw8(h.x + (row0 + r) * h.x_row + (int64_t)(item - r * h.heads) * h.x_head, at.c0, h.x_wide);
  };
  kv_u4 next = load(0);
  for (int i = 0; i < items; i += kAtOnce) {
    const kv_u4 own = next, other = others<MODE, kLanes>(at, own, pass);
    next = load(i + kAtOnce);
    const int item = min(i + slot, items - 1), r = small_div(item, inverse), head = item - r * h.heads;
    float u[8], v[8], x[8];
    unpack8<BF16>(own, u);
    unpack8<BF16>(other, v);
    double y[8], norm = 1.0;
    if (h.gain) {
      double ss = 0.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fma((double)u[e], (double)u[e], ss);
      norm = inverse_root(fma(group_sum_f64<kLanes>(ss), a.inv_dim, a.eps));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {   // (a product of a gain and 16 bits is exact)
      y[e] = (double)u[e] * (double)gn[e];
      if (at.turned(e)) y[e] = fma((double)v[e] * (double)go[e], turns[r].s[at.pair(e)], y[e] * turns[r].c[at.pair(e)]);
      y[e] *= norm;
    }
    to_odd8(y, x);
    const Token token = tokens[r];
    if (i + slot < items && token.page) {
      uint32_t b;
      const uint32_t w = quantize8(x, &b, &bad, &over);
      put_key<D>(token.page + (int64_t)head * KvLayout<D>::head_bytes(T), T, token.t, sub, w, b);
    }
  }
  if (g.status) {
    count_in(g.status, 0, bad);
    count_in(g.status, 1, over);
  }
}

// k_kv_rotate_append for few heads.
template <int D, bool BF16, int MODE>
__global__ __launch_bounds__(kKvThreads) void k_kv_rotate_append_few(AppendArgs g) {
  constexpr int kLanes = D / 8, kWaves = kKvThreads / 64;
  __shared__ RowAngles<kLanes> row_angles[kWaves][kFewRows];
  __shared__ RowTurns<D> key_turns[kWaves][kFewRows];
  __shared__ Token row_tokens[kWaves][kFewRows];
  __shared__ Pass<MODE> pass[kWaves];
  if (blockIdx.x < g.v_blocks) {
    append_values<D, BF16>(g);
    return;
  }
  const RotateArgs& r = g.r;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row0 = ((int64_t)(blockIdx.x - g.v_blocks) * kWaves + wave) * kFewRows;
  if (row0 >= g.c.rows) return;
  const int n = (int)min((int64_t)kFewRows, g.c.rows - row0);
  uint32_t none = 0, stored = 0;
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    Token token{0, 0, nullptr};
    none |= row_token<D>(g.c, row0 + i, g.first, &token) ? 0u : 1u << i;
    stored |= token.page ? 1u << i : 0u;
    if (lane == 0) row_tokens[wave][i] = token;
  }
  wave_lds_order();
  const uint32_t inverse = r.pairs ? 65536u / (uint32_t)r.pairs + 1u : 0u;
  for (int i = lane; i < n * r.pairs; i += 64) {
    const int row = small_div(i, inverse), pair = i - row * r.pairs;
    double c, s;
    sin_cos(row_tokens[wave][row].pos, r.freq[pair], &c, &s);
    key_turns[wave][row].c[pair] = c *= r.amplitude64;
    key_turns[wave][row].s[pair] = s *= r.amplitude64;
    row_angles[wave][row].c[pair] = (float)c;
    row_angles[wave][row].s[pair] = (float)s;
  }
  wave_lds_order();
  if (stored) append_few<D, BF16, MODE>(g, row0, n, row_tokens[wave], key_turns[wave], pass[wave].w);
  rotate_few<kLanes, BF16, MODE>(r, 1, row0, n, none, row_angles[wave], pass[wave].w);
}

// Workgroups of values, then waves of a row's queries and keys each (or parts of them).  Keys go by rows
// as the queries do, since their codes are a line of their own for each token, and share the row's
// sines; value codes lie by four tokens and go by quads.  (Keys by quads as well, with the factors of
// four rows in LDS: 140 to 195 registers, 773 to 1,010 us for the rows above.  Workgroups of values by turns
// with those of rows: 65,536 rows of 8 + 8 heads 174 us, after them 164, before them 155.)
template <int D, bool BF16, int MODE>
__global__ __launch_bounds__(kKvThreads) void k_kv_rotate_append(AppendArgs g) {
  constexpr int kLanes = D / 8, kAtOnce = 64 / kLanes, kWaves = kKvThreads / 64;
  __shared__ RowAngles<kLanes> row_angles[kWaves];
  __shared__ Factors<D> key_factors[kWaves];
  __shared__ Pass<MODE> pass[kWaves];
  if (blockIdx.x < g.v_blocks) {
    append_values<D, BF16>(g);
    return;
  }
  const RotateArgs& r = g.r;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const uint32_t id = (blockIdx.x - g.v_blocks) * kWaves + wave;
  const int64_t row = id / (uint32_t)r.parts;
  const int part = (int)(id % (uint32_t)r.parts);
  if (row >= g.c.rows) return;
  const RotateHeads &q = r.h[0], &k = r.h[1];
  Token token;
  if (!row_token<D>(g.c, row, g.first, &token)) {   // queries of no sequence
    for (int head = part * kAtOnce + lane / kLanes; head < q.heads; head += r.parts * kAtOnce)
      store_raw8(q.y, row * q.y_row + (int64_t)head * q.y_head + 8 * (lane % kLanes), q.y_wide, kv_u4{0, 0, 0, 0});
    return;
  }
  const int q_rounds = (q.heads + kAtOnce - 1) / kAtOnce;
  const int k_first = (part - q_rounds % r.parts + r.parts) % r.parts;   // the wave's first round of keys
  const bool keys = token.page && k_first * kAtOnce < g.c.heads;
  RowAngles<kLanes>& angles = row_angles[wave];
  Factors<D>& f = key_factors[wave];
  for (int i = lane; i < D / 2; i += 64) {
    double c = 1.0, s = 0.0;
    int u = 2 * i, v = u + 1;
    if (i < r.pairs) {
      sin_cos(token.pos, r.freq[i], &c, &s);
      c *= r.amplitude64, s *= r.amplitude64;
      if (MODE != kInterleaved) u = i, v = i + r.pairs;
      angles.c[i] = (float)c;
      angles.s[i] = (float)s;
    }
    if (keys) {
      const double gu = k.gain ? (double)gain_at<BF16>(k, u) : 1.0, gv = k.gain ? (double)gain_at<BF16>(k, v) : 1.0;
      f.own[u] = c * gu, f.other[u] = -s * gv;
      f.own[v] = c * gv, f.other[v] = s * gu;
    }
  }
  wave_lds_order();
  if (keys) append_keys<D, BF16, MODE>(g, row, k_first, token, f, pass[wave].w);
  rotate_row<kLanes, BF16, MODE>(r, 1, row, part, angles, pass[wave].w);
}

// Waves that a call of few rows is shared out to, at least for rows on their own, at most on the way
// into the cache, where every part makes the keys' factors again.  Rows of 40 heads of 128 channels (others are not
// measured): 300
// in 10 parts 4.5 us, 1,000 in 4 or 5 7.7 us (1: 10, 8: 9.9), 2,500 in 2 13.8 us (1: 16.5), 4,000 in 2 18.9
// (1: 19.7); into the cache 2,000 in 2 14.1 us (1: 16.0, 3: 17.8), 3,000 in 1 19.4 (2: 21.9).
constexpr int64_t kRotateWaves = 4096;

// Whether a wave takes four rows: for heads so few that the rounds of one leave lanes idle, and so
// many rows that a quarter of the waves fills the chip.  65,536 rows, one and four rows a wave, us:
// 64 channels, 4 + 1 heads 53 and 26 (into the cache 86 and 41), 16 + 4 71 and 61 (113 and 81), 32 + 4 113 and 111
// (146 and 124), 32 + 8 124 and 141 (157 and 152); 128 channels, 4 + 1 heads 56 and 38 (93 and 58), 16 + 2 114 and
// 115 (148 and 131), 16 + 4 124 and 140 (158 and 160).  16,384 rows: 64 channels, 16 + 4 heads 22 and 21 (34 and
// 29), 32 + 8 32 and 34 (44 and 46); 8,192: 4 + 1 heads 9 and 6 (13 and 9), 16 + 4 13 and 15.  Between these the borders
// are not measured.  Heads of 256 channels fill a wave by two.
bool few_heads(int64_t rows, int heads, int lanes) {
  return heads <= (lanes == 8 ? 40 : lanes == 16 ? 18 : 0) && rows >= std::max(8192, 128 * lanes * heads);
}

}  // namespace

// waves of a call's rows; parts: those that share one, `waves` / rows or one for each round of heads
static int64_t row_waves(int64_t waves, int64_t rows, int heads, int other_heads, int lanes, int* parts) {
  const int at_once = 64 / lanes;
  const int rounds = (heads + at_once - 1) / at_once + (other_heads + at_once - 1) / at_once;
  *parts = (int)std::max<int64_t>(1, std::min<int64_t>(rounds, waves / rows));
  return heads + other_heads > 0 ? rows * *parts : 0;
}

lam_status launch_kv_rotate(lam_ctx* ctx, RotateArgs a, int dtype) {
  const int lanes = a.dim <= 64 ? 8 : a.dim <= 128 ? 16 : 32;
  const int64_t waves = row_waves(kRotateWaves + a.rows - 1, a.rows, a.h[0].heads, a.h[1].heads, lanes, &a.parts);
  const bool few = few_heads(a.rows, a.h[0].heads + a.h[1].heads, lanes);
  const int64_t blocks = ((few ? (a.rows + kFewRows - 1) / kFewRows : waves) + kKvThreads / 64 - 1) / (kKvThreads / 64);
  LAM_CHECK(waves < (1LL << 31) && blocks <= most_blocks(kKvThreads), LAM_EINVAL, "too many rows for one launch");
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_rotate", &e0, &e1));
  const dim3 grid((unsigned)blocks);
#define LAM_MODE(L, BF, M)                                                                                  \
  do {                                                                                                      \
    if (L < 32 && few) launch(k_kv_rotate_few<L < 32 ? L : 16, BF, M>, grid, kKvThreads, ctx->stream, e0, e1, a); \
    else launch(k_kv_rotate<L, BF, M>, grid, kKvThreads, ctx->stream, e0, e1, a);                           \
  } while (0)
#define LAM_GO(L, BF)                                          \
  do {                                                         \
    if (a.interleaved) LAM_MODE(L, BF, kInterleaved);          \
    else if (a.pairs % 8 == 0) LAM_MODE(L, BF, kHalves);       \
    else LAM_MODE(L, BF, kHalvesAnywhere);                     \
  } while (0)
  const bool bf = dtype == LAM_BF16;
  if (lanes == 8) { if (bf) LAM_GO(8, true); else LAM_GO(8, false); }
  else if (lanes == 16) { if (bf) LAM_GO(16, true); else LAM_GO(16, false); }
  else { if (bf) LAM_GO(32, true); else LAM_GO(32, false); }
#undef LAM_GO
#undef LAM_MODE
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

lam_status launch_kv_rotate_append(lam_ctx* ctx, const lam_kv_view& v, const RotateArgs& r, const void* val,
                                   int64_t v_row, int64_t v_head, const lam_kv_slots& weights,
                                   const lam_kv_slots& positions, const int32_t* first, uint32_t* status) {
  AppendArgs g{};
  const int lanes = v.head_dim / 8;
  const int64_t values = quad_units(v, &g.quads) * v.kv_heads, per = kKvThreads / lanes;
  const int64_t v_blocks = (values + per - 1) / per;
  g.r = r;
  const int64_t waves = row_waves(kRotateWaves, v.rows, r.h[0].heads, r.h[1].heads, lanes, &g.r.parts);
  const bool few = few_heads(v.rows, r.h[0].heads + r.h[1].heads, lanes);
  const int64_t blocks = v_blocks + ((few ? (v.rows + kFewRows - 1) / kFewRows : waves) + kKvThreads / 64 - 1) / (kKvThreads / 64);
  LAM_CHECK(values < (1LL << 31) && waves < (1LL << 31) && blocks <= most_blocks(kKvThreads), LAM_EINVAL,
            "too many rows or sequences for one launch");
  g.c = KvArgs::of(v);
  g.v_blocks = (uint32_t)v_blocks;
  g.v = RowArgs{val, v_row, v_head, wide_rows(val, v_row, v_head)};
  g.weights = weights;
  g.positions = positions;
  g.first = first;
  g.status = status;
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_rotate_append", &e0, &e1));
  const dim3 grid((unsigned)blocks);
#define LAM_MODE(D, BF, M)                                                                                          \
  do {                                                                                                              \
    if (D < 256 && few) launch(k_kv_rotate_append_few<D < 256 ? D : 128, BF, M>, grid, kKvThreads, ctx->stream, e0, e1, g); \
    else launch(k_kv_rotate_append<D, BF, M>, grid, kKvThreads, ctx->stream, e0, e1, g);                            \
  } while (0)
#define LAM_GO(D, BF)                                          \
  do {                                                         \
    if (r.interleaved) LAM_MODE(D, BF, kInterleaved);          \
    else if (r.pairs % 8 == 0) LAM_MODE(D, BF, kHalves);       \
    else LAM_MODE(D, BF, kHalvesAnywhere);                     \
  } while (0)
  LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
#undef LAM_MODE
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

}  // namespace lam
