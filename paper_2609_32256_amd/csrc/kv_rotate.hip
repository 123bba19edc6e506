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
  float a = 42.058693944897655f, b = -26.4262567833744f;   // the next terms: 2e-9, 3e-9
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

__device__ __forceinline__ float gain_at(const RotateHeads& h, int c, bool bf16) {
  if (h.gain_f32) return static_cast<const float*>(h.gain)[c];
  const uint16_t g = static_cast<const uint16_t*>(h.gain)[c];
  return bf16 ? __uint_as_float((uint32_t)g << 16) : (float)__builtin_bit_cast(_Float16, g);
}

// The raw other channels of a lane's eight, given its own.
template <int MODE, int L>
__device__ __forceinline__ kv_u4 others(const Lane<MODE>& at, kv_u4 own, const uint16_t* head) {
  kv_u4 w = own;
  if constexpr (MODE == kHalves) {
    const int from = ((int)threadIdx.x & 63 & ~(L - 1)) + at.other(0) / 8;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (uint32_t)__shfl((int)own[j], from);
  } else if constexpr (MODE == kInterleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_alignbit(own[j], own[j], 16);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = (uint32_t)head[at.other(2 * j)] | ((uint32_t)head[at.other(2 * j + 1)] << 16);
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

// ------------------------------------------------------------------ rows on their own
// A wave takes a row, or a part of its heads where rows are few, 64/L heads at a time: the sines and
// cosines are made once for all of them and lie in registers, multiplied by the gains.
template <int L, bool BF16, int MODE>
__global__ __launch_bounds__(kKvThreads) void k_kv_rotate(RotateArgs a) {
  constexpr int kAtOnce = 64 / L;
  const uint32_t wave = blockIdx.x * (kKvThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = wave / (uint32_t)a.parts;
  const int part = (int)(wave % (uint32_t)a.parts);
  if (row >= a.rows) return;
  const int sub = threadIdx.x % L, slot = (threadIdx.x & 63) / L;
  const Lane<MODE> at{8 * sub, a.pairs};
  const bool live = at.c0 < a.dim;
  float cs[8], sn[8];
  const int32_t pos = a.pairs ? a.positions[row] : 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (MODE == kInterleaved && (e & 1)) {
      cs[e] = cs[e - 1], sn[e] = -sn[e - 1];
      continue;
    }
    cs[e] = 1.0f, sn[e] = 0.0f;
    if (live && at.turned(e)) {
      sin_cos(pos, a.freq[at.pair(e)], &cs[e], &sn[e]);
      cs[e] *= a.amplitude, sn[e] *= a.amplitude;
      if (at.minus(e)) sn[e] = -sn[e];
    }
  }
  int round0 = 0;
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {
    const RotateHeads& h = a.h[kind];
    const int rounds = (h.heads + kAtOnce - 1) / kAtOnce;
    float ga[8], gb[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      ga[e] = cs[e], gb[e] = sn[e];
      if (h.gain && live) {
        ga[e] *= gain_at(h, at.c0 + e, BF16);
        gb[e] *= gain_at(h, at.other(e), BF16);
      }
    }
    for (int i = (part - round0 % a.parts + a.parts) % a.parts; i < rounds; i += a.parts) {
      const int head = i * kAtOnce + slot;
      const bool there = live && head < h.heads;
      kv_u4 own{}, other{};
      const uint16_t* x = h.x + row * h.x_row + (int64_t)(head < h.heads ? head : 0) * h.x_head;
      if (there) own = load_raw8(x, at.c0, h.x_wide);
      if constexpr (MODE == kHalvesAnywhere) {
        if (there) other = others<MODE, L>(at, own, x);
      } else {
        other = others<MODE, L>(at, own, x);
      }
      float u[8], v[8], y[8];
      unpack8<BF16>(own, u);
      unpack8<BF16>(other, v);
      float r = 1.0f;
      if (h.gain) {
        double ss = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fma((double)u[e], (double)u[e], ss);
        r = (float)__builtin_amdgcn_rsq(fma(group_sum_f64<L>(ss), a.inv_dim, a.eps));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float straight = u[e] * ga[e];
        y[e] = (at.turned(e) ? fmaf(v[e], gb[e], straight) : straight) * r;
      }
      if (there) store_raw8(h.y, row * h.y_row + (int64_t)head * h.y_head + at.c0, h.y_wide, pack8<BF16>(y));
    }
    round0 += rounds;
  }
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

// 1 / sqrt(a) to about 2^-52, for a > 0.
__device__ __forceinline__ double inverse_root(double a) {
  double y = __builtin_amdgcn_rsq(a);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-a * y, y, 1.0), y);
  return y;
}

// Sines and cosines of a quad's rows, with the amplitude in them.
template <int D>
struct __align__(16) Angles {
  double c[4][D / 2], s[4][D / 2];
  float cf[4][D / 2], sf[4][D / 2];
};

// A workgroup takes a quad of slots and 256 / (D/8) heads: the keys and values of a head, or the
// queries of one, by D/8 lanes.  The angles of its rows are made by all threads, for all heads, and
// lie in LDS.  Keys are normed and turned in binary64, which vector units of this chip run at
// float32's rate, so that no code is decided by a rounding on the way.
template <int D, bool BF16, int MODE>
__global__ __launch_bounds__(kKvThreads) void k_kv_rotate_append(KvArgs a, int quads, uint32_t groups, RotateArgs r,
                                                                 RowArgs vals, lam_kv_slots weights,
                                                                 lam_kv_slots positions, const int32_t* first,
                                                                 uint32_t* status) {
  constexpr int kLanes = D / 8, kItems = kKvThreads / kLanes;
  __shared__ Angles<D> angles;
  const uint32_t unit = blockIdx.x / groups;
  const int item = (int)(blockIdx.x % groups) * kItems + (int)threadIdx.x / kLanes, sub = threadIdx.x % kLanes;
  const int h = min(item, a.heads - 1);
  Quad q = quad_at<D>(a, quads, unit, h);
  const uint32_t rows = __builtin_amdgcn_readfirstlane(q.rows);
  bool bad = false, over = false;
  if (rows) {
    for (int i = threadIdx.x; i < 4 * r.pairs; i += kKvThreads) {
      const int row = i / r.pairs, pair = i % r.pairs;
      if (!((rows >> row) & 1u)) continue;
      double c, s;
      sin_cos(quad_pos(q, row, first), r.freq[pair], &c, &s);
      angles.c[row][pair] = c *= r.amplitude64;
      angles.s[row][pair] = s *= r.amplitude64;
      angles.cf[row][pair] = (float)c;
      angles.sf[row][pair] = (float)s;
    }
    __syncthreads();
    const Lane<MODE> at{8 * sub, r.pairs};
    if (item < a.heads) {
      const RotateHeads& kh = r.h[1];
      kv_u4 own[4], val[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // a slot that is not the call's repeats one that is
        const int64_t row = q.row + ((rows >> i) & 1u ? i : __builtin_ctz(rows));
        own[i] = load_raw8(kh.x, row * kh.x_row + (int64_t)h * kh.x_head + at.c0, kh.x_wide);
        val[i] = load_raw8(vals.p, row * vals.row + (int64_t)h * vals.head + at.c0, vals.wide);
      }
      float g[8], go[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[e] = kh.gain ? gain_at(kh, at.c0 + e, BF16) : 1.0f;
        go[e] = kh.gain ? gain_at(kh, at.other(e), BF16) : 1.0f;
      }
      uint32_t kw[4] = {}, vw[4] = {}, kb[4] = {}, vb[4] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!((rows >> i) & 1u)) continue;
        const int64_t row = q.row + i;
        float u[8], v[8], x[8];
        const kv_u4 other = others<MODE, kLanes>(at, own[i], kh.x + row * kh.x_row + (int64_t)h * kh.x_head);
        unpack8<BF16>(own[i], u);
        unpack8<BF16>(other, v);
        double n = 1.0;
        if (kh.gain) {
          double ss = 0.0;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fma((double)u[e], (double)u[e], ss);
          n = inverse_root(fma(group_sum_f64<kLanes>(ss), r.inv_dim, r.eps));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          double y = (double)u[e] * (double)g[e];
          if (at.turned(e)) {
            const double s = angles.s[i][at.pair(e)];
            y = fma((double)v[e] * (double)go[e], at.minus(e) ? -s : s, y * angles.c[i][at.pair(e)]);
          }
          x[e] = to_odd(y * n);
        }
        kw[i] = quantize8(x, &kb[i], &bad, &over);
        unpack8<BF16>(val[i], x);
        vw[i] = quantize8(x, &vb[i], &bad, &over);
      }
      if (q.base) {
        put_quad<D>(q, 1 << a.page_shift, sub, kw, kb, vw, vb);
        put_slots(a, q, h, sub, weights, positions, first);
      } else {
        bad = over = false;   // (not stored, so counted as that alone)
      }
    } else if (item < a.heads + r.h[0].heads) {
      const RotateHeads& qh = r.h[0];
      const int64_t head = item - a.heads;
      kv_u4 own[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t row = q.row + ((rows >> i) & 1u ? i : __builtin_ctz(rows));
        own[i] = load_raw8(qh.x, row * qh.x_row + head * qh.x_head + at.c0, qh.x_wide);
      }
      float g[8], go[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[e] = qh.gain ? gain_at(qh, at.c0 + e, BF16) : 1.0f;
        go[e] = qh.gain ? gain_at(qh, at.other(e), BF16) : 1.0f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!((rows >> i) & 1u)) continue;
        const int64_t row = q.row + i;
        float u[8], v[8], y[8];
        const kv_u4 other = others<MODE, kLanes>(at, own[i], qh.x + row * qh.x_row + head * qh.x_head);
        unpack8<BF16>(own[i], u);
        unpack8<BF16>(other, v);
        float n = 1.0f;
        if (qh.gain) {
          double ss = 0.0;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fma((double)u[e], (double)u[e], ss);
          n = (float)__builtin_amdgcn_rsq(fma(group_sum_f64<kLanes>(ss), r.inv_dim, r.eps));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float t = u[e] * g[e];
          if (at.turned(e)) {
            const float s = angles.sf[i][at.pair(e)];
            t = fmaf(v[e] * go[e], at.minus(e) ? -s : s, t * angles.cf[i][at.pair(e)]);
          }
          y[e] = t * n;
        }
        store_raw8(qh.y, row * qh.y_row + head * qh.y_head + at.c0, qh.y_wide, pack8<BF16>(y));
      }
    }
  }
  if (item >= a.heads) q.rows = 0;   // (counts are of keys and values)
  if (status) count_quad(a, q, sub, bad, over, status);
  if (a.starts && r.h[0].heads) {   // queries of no sequence
    const RotateHeads& qh = r.h[0];
    const int64_t before = a.start(0), after = a.start(a.n_seqs);
    for (int64_t i = blockIdx.x; i < before + a.rows - after; i += gridDim.x) {
      const int64_t row = i < before ? i : after + i - before;
      for (int head = threadIdx.x / kLanes; head < qh.heads; head += kItems)
        store_raw8(qh.y, row * qh.y_row + (int64_t)head * qh.y_head + 8 * sub, qh.y_wide, kv_u4{0, 0, 0, 0});
    }
  }
}

// Waves that a call of few rows is shared out to.
constexpr int64_t kRotateWaves = 4096;

}  // namespace

lam_status launch_kv_rotate(lam_ctx* ctx, RotateArgs a, int dtype) {
  const int lanes = a.dim <= 64 ? 8 : a.dim <= 128 ? 16 : 32, at_once = 64 / lanes;
  const int rounds = (a.h[0].heads + at_once - 1) / at_once + (a.h[1].heads + at_once - 1) / at_once;
  a.parts = (int)std::min<int64_t>(rounds, std::max<int64_t>(1, kRotateWaves / a.rows));
  const int64_t blocks = (a.rows * a.parts + kKvThreads / 64 - 1) / (kKvThreads / 64);
  LAM_CHECK(a.rows * a.parts < (1LL << 31) && blocks <= most_blocks(kKvThreads), LAM_EINVAL, "too many rows for one launch");
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_rotate", &e0, &e1));
  const dim3 grid((unsigned)blocks);
#define LAM_GO(L, BF)                                                                                                  \
  do {                                                                                                                 \
    if (a.interleaved) launch(k_kv_rotate<L, BF, kInterleaved>, grid, kKvThreads, ctx->stream, e0, e1, a);             \
    else if (a.pairs % 8 == 0) launch(k_kv_rotate<L, BF, kHalves>, grid, kKvThreads, ctx->stream, e0, e1, a);          \
    else launch(k_kv_rotate<L, BF, kHalvesAnywhere>, grid, kKvThreads, ctx->stream, e0, e1, a);                        \
  } while (0)
  const bool bf = dtype == LAM_BF16;
  if (lanes == 8) { if (bf) LAM_GO(8, true); else LAM_GO(8, false); }
  else if (lanes == 16) { if (bf) LAM_GO(16, true); else LAM_GO(16, false); }
  else { if (bf) LAM_GO(32, true); else LAM_GO(32, false); }
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

lam_status launch_kv_rotate_append(lam_ctx* ctx, const lam_kv_view& v, const RotateArgs& r, const void* val,
                                   int64_t v_row, int64_t v_head, const lam_kv_slots& weights,
                                   const lam_kv_slots& positions, const int32_t* first, uint32_t* status) {
  int quads;
  const int64_t units = quad_units(v, &quads);
  const int64_t per = kKvThreads / (v.head_dim / 8), groups = (v.kv_heads + r.h[0].heads + per - 1) / per;
  LAM_CHECK(units < (1LL << 31) && units * groups <= most_blocks(kKvThreads), LAM_EINVAL,
            "too many rows or sequences for one launch");
  const KvArgs a = KvArgs::of(v);
  const RowArgs va{val, v_row, v_head, wide_rows(val, v_row, v_head)};
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_rotate_append", &e0, &e1));
  const dim3 grid((unsigned)(units * groups));
#define LAM_MODE(D, BF, M)                                                                                        \
  launch(k_kv_rotate_append<D, BF, M>, grid, kKvThreads, ctx->stream, e0, e1, a, quads, (uint32_t)groups, r, va, weights, \
         positions, first, status)
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
