// The 4-bit key/value cache's own memory: rows quantized into it, values read
// back, and tokens evicted from it (include/lam.h, lam_kv_*).
#include <algorithm>
#include <type_traits>

#include "kv.h"
#include "lam_internal.h"
#include "wave.h"

namespace lam {
namespace {

constexpr int kKvThreads = 256;

// A group of D/8 lanes holds a token of one head, eight channels a lane: one
// 4-byte word of key codes, and the same eight channels' value codes, which lie
// in one run (D = 128), in two (64) or in half of one (256).
template <int D>
__device__ __forceinline__ void put_v_word(uint8_t* base, int T, int t, int sub, uint32_t w) {
  if constexpr (D == 64) {
    *reinterpret_cast<uint16_t*>(base + KvLayout<D>::v_codes(T, t, 2 * sub)) = (uint16_t)w;
    *reinterpret_cast<uint16_t*>(base + KvLayout<D>::v_codes(T, t, 2 * sub + 1)) = (uint16_t)(w >> 16);
  } else if constexpr (D == 128) {
    *reinterpret_cast<uint32_t*>(base + KvLayout<D>::v_codes(T, t, sub)) = w;
  } else {
    *reinterpret_cast<uint32_t*>(base + KvLayout<D>::v_codes(T, t, sub >> 1) + (sub & 1) * 4) = w;
  }
}

template <int D>
__device__ __forceinline__ uint32_t get_v_word(const uint8_t* base, int T, int t, int sub) {
  if constexpr (D == 64) {
    const uint32_t lo = *reinterpret_cast<const uint16_t*>(base + KvLayout<D>::v_codes(T, t, 2 * sub));
    const uint32_t hi = *reinterpret_cast<const uint16_t*>(base + KvLayout<D>::v_codes(T, t, 2 * sub + 1));
    return lo | (hi << 16);
  } else if constexpr (D == 128) {
    return *reinterpret_cast<const uint32_t*>(base + KvLayout<D>::v_codes(T, t, sub));
  } else {
    return *reinterpret_cast<const uint32_t*>(base + KvLayout<D>::v_codes(T, t, sub >> 1) + (sub & 1) * 4);
  }
}

// Eight channels of a row as float32.  Rows are read once here, and written once by
// the read: non-temporal, 284 -> 259 us for 131,072 rows of 8 heads of 128 channels both ways, the rate of a copy.
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t at, bool wide, float x[8]) {
  const uint16_t* h = static_cast<const uint16_t*>(p) + at;
  uint32_t w[4];
  if (wide) {
    const kv_u4 u = __builtin_nontemporal_load(reinterpret_cast<const kv_u4*>(h));
    w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (uint32_t)h[2 * j] | ((uint32_t)h[2 * j + 1] << 16);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    } else {
      const kv_h2 v = __builtin_bit_cast(kv_h2, w[j]);
      x[2 * j] = (float)v[0];
      x[2 * j + 1] = (float)v[1];
    }
  }
}

// The codes of eight channels and their block's scale byte.  Four lanes share
// a block: its largest |x| goes round the quad.  6 * 2^e >= amax with amax =
// m 2^x, m in [1, 2), gives e = x - 2 for m <= 1.5 and x - 1 above; the
// conversion instruction divides by 2^e and rounds to nearest, ties to even.
__device__ __forceinline__ uint32_t quantize8(float x[8], uint32_t* byte, bool* bad, bool* over) {
  float a = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool ok = fabsf(x[j]) < __builtin_inff();
    *bad |= !ok;
    x[j] = ok ? x[j] : 0.0f;
    a = fmaxf(a, fabsf(x[j]));
  }
  a = quad_max_f32(a);
  *over |= a > 49152.0f;
  const uint32_t b = __float_as_uint(a);
  int e = (int)(b >> 23) - 129 + ((b & 0x7fffffu) > 0x400000u ? 1 : 0);
  e = min(max(e, kKvExpLo), kKvExpHi);
  *byte = (uint32_t)(e + 127);
  const float s = kv_scale(*byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}

__device__ __forceinline__ void count_in(uint32_t* status, int i, bool hit) {
  const unsigned long long m = __ballot(hit);
  if (m && (int)__builtin_ctzll(m) == (int)(threadIdx.x & 63)) atomicAdd(status + i, (uint32_t)__popcll(m));
}

struct RowArgs {   // rows of keys or values: strides in elements
  const void* p;
  int64_t row, head;
  int wide;        // every eight channels are a 16-byte load
};

// Four consecutive slots of a head, the unit in which value codes lie, of which the
// call's rows take some.  Units go by sequence: with the same number of rows each, a.quads of
// them a sequence; else those of sequence s begin at floor(start(s) / 4) + 2 s, a
// bound that leaves room for the partial ones at both ends.
struct Quad {
  int s = -1;           // sequence, -1: nothing
  int64_t row = 0;      // row of its first slot (which may be none of the call's)
  int64_t slot = 0;     // its first slot
  int64_t first_row = 0;
  uint32_t rows = 0;    // bit i: slot i is one of the call's rows
  uint8_t* base = nullptr;   // the head's page, null: no place
};

// All lanes of a wave, whose units do not fall: the sequence of the first one is found by
// all at once, 64 sequences a step, with its rows and length in hand (by halves, lane by
// lane, 18,800 rows of 5 sequences took 27 us for 25).
template <int D>
__device__ __forceinline__ Quad quad_at(const KvArgs& a, int quads, uint32_t unit, int h) {
  Quad q;
  uint32_t local;
  int64_t next;
  int len;
  if (!a.starts) {
    q.s = (int)(unit / (uint32_t)quads);
    local = unit % (uint32_t)quads;
    if (q.s >= a.n_seqs) q.s = -1;
    const int s = max(q.s, 0);
    q.first_row = a.start(s);
    next = a.start(s + 1);
    len = a.lengths[s];
  } else {
    const int lane = threadIdx.x & 63;
    const uint32_t unit0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)unit);
    int s = 0;
    q.first_row = next = 0;
    len = 0;
    for (int b = 0; b < a.n_seqs; b += 64) {
      const int mine = min(b + lane, a.n_seqs - 1);
      const int64_t s0 = a.start(mine), s1 = a.start(mine + 1);
      const int l = a.lengths[mine];
      const unsigned long long in = __ballot(b + lane < a.n_seqs && s0 / 4 + 2 * (int64_t)mine <= unit0);
      if (in == 0 && b > 0) break;
      const int last = in == 0 ? 0 : (int)__popcll(in) - 1;
      s = b + last;
      q.first_row = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)s0, last);
      next = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)s1, last);
      len = __builtin_amdgcn_readlane(l, last);
      if (last < 63) break;
    }
    if (s + 1 < a.n_seqs && next / 4 + 2 * (int64_t)(s + 1) <= unit) {   // a lane whose unit is a later sequence's
      do ++s; while (s + 1 < a.n_seqs && a.start(s + 1) / 4 + 2 * (int64_t)(s + 1) <= unit);
      q.first_row = a.start(s);
      next = a.start(s + 1);
      len = a.lengths[s];
    }
    const int64_t at = (int64_t)unit - (q.first_row / 4 + 2 * (int64_t)s);
    q.s = at >= 0 ? s : -1;
    local = (uint32_t)at;
  }
  if (q.s < 0) return q;
  const int64_t n = next - q.first_row;
  const int64_t slot0 = (int64_t)len - n;   // of the first row
  q.slot = (slot0 >> 2) * 4 + 4 * (int64_t)local;
  q.row = q.first_row + (q.slot - slot0);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (q.slot + i >= slot0 && q.slot + i < slot0 + n) q.rows |= 1u << i;
  if (q.rows && q.slot >= 0 && (q.slot >> a.page_shift) < a.table_cols) {
    const int64_t page = a.page(q.s, (int)(q.slot >> a.page_shift));
    if (page >= 0) q.base = a.head_page(page, h, KvLayout<D>::head_bytes(1 << a.page_shift));
  }
  return q;
}

// A lane quantizes eight channels of a quad's four rows: its value codes are then
// one store (of 16 bytes for 128 channels) where all four are the call's, its scales
// of the values one word.  Bound by memory: two rows read and 17/32 of a byte a
// channel written; 131,072 rows of 8 heads of 128 channels take 129 us, 5.3 TB/s.  (A lane for each row, 4-byte stores 16 bytes apart, wrote every
// line in four parts: 175 us.)
template <int D, bool BF16>
__global__ __launch_bounds__(kKvThreads) void k_kv_append(KvArgs a, int quads, RowArgs k, RowArgs v,
                                                          lam_kv_slots weights, lam_kv_slots positions,
                                                          const int32_t* first, uint32_t* status) {
  using L = KvLayout<D>;
  constexpr int kLanes = D / 8;
  const uint32_t item = blockIdx.x * (kKvThreads / kLanes) + threadIdx.x / kLanes;
  const int sub = threadIdx.x % kLanes;
  const int h = (int)(item % (uint32_t)a.heads);
  const Quad q = quad_at<D>(a, quads, item / (uint32_t)a.heads, h);
  const int T = 1 << a.page_shift;
  bool bad = false, over = false;
  if (q.base) {
    float x[4][8], y[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // a slot that is not the call's repeats one that is
      const int64_t row = q.row + ((q.rows >> i) & 1u ? i : __builtin_ctz(q.rows));
      load8<BF16>(k.p, row * k.row + h * k.head + 8 * sub, k.wide, x[i]);
      load8<BF16>(v.p, row * v.row + h * v.head + 8 * sub, v.wide, y[i]);
    }
    uint32_t kw[4], vw[4], kb[4], vb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kw[i] = quantize8(x[i], &kb[i], &bad, &over);
      vw[i] = quantize8(y[i], &vb[i], &bad, &over);
    }
    const int t = (int)(q.slot & (T - 1));
    uint32_t* vs = reinterpret_cast<uint32_t*>(q.base + L::v_scales(T, t, sub >> 2));
    if (q.rows == 0xfu) {
      if constexpr (D == 128) {
        *reinterpret_cast<uint4*>(q.base + L::v_codes(T, t, sub)) = uint4{vw[0], vw[1], vw[2], vw[3]};
      } else if constexpr (D == 64) {   // two runs of four channels: halves of the words
        *reinterpret_cast<uint4*>(q.base + L::v_codes(T, t, 2 * sub)) =
            uint4{__builtin_amdgcn_perm(vw[1], vw[0], 0x05040100u), __builtin_amdgcn_perm(vw[3], vw[2], 0x05040100u),
                  __builtin_amdgcn_perm(vw[1], vw[0], 0x07060302u), __builtin_amdgcn_perm(vw[3], vw[2], 0x07060302u)};
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) put_v_word<D>(q.base, T, t + i, sub, vw[i]);
      }
      if ((sub & 3) == 0) *vs = vb[0] | (vb[1] << 8) | (vb[2] << 16) | (vb[3] << 24);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((q.rows >> i) & 1u) {
          put_v_word<D>(q.base, T, t + i, sub, vw[i]);
          if ((sub & 3) == 0) reinterpret_cast<uint8_t*>(vs)[i] = (uint8_t)vb[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((q.rows >> i) & 1u) {
        *reinterpret_cast<uint32_t*>(q.base + L::k_codes(t + i) + 4 * sub) = kw[i];
        if ((sub & 3) == 0) q.base[L::k_scales(T, t + i) + (sub >> 2)] = (uint8_t)kb[i];
      }
    if (sub < 4 && (q.rows >> sub) & 1u) {   // lane i: token i's weight and position
      const int64_t slot = q.slot + sub;
      if (weights.p_dev && slot < weights.cols)
        static_cast<float*>(weights.p_dev)[q.s * weights.seq_stride + h * weights.head_stride + slot] = 0.0f;
      if (positions.p_dev && slot < positions.cols)
        static_cast<int32_t*>(positions.p_dev)[q.s * positions.seq_stride + h * positions.head_stride + slot] =
            (int32_t)(first[q.s] + (q.row + sub - q.first_row));
    }
  }
  if (status) {
    count_in(status, 0, bad);
    count_in(status, 1, over);
    // rows without a place: of this quad, and (once) those of no sequence
    uint32_t lost = !q.base && sub == 0 ? (uint32_t)__popc(q.rows) : 0u;
    if (a.starts && blockIdx.x == 0 && threadIdx.x == 0)
      lost += (uint32_t)(a.start(0) + a.rows - a.start(a.n_seqs)) * (uint32_t)a.heads;
    if (lost) atomicAdd(status + 2, lost);
  }
}

// The other way, by the same quads.  Bound by memory: the rows above take 103 us, 6.6 TB/s.
template <int D, bool BF16>
__global__ __launch_bounds__(kKvThreads) void k_kv_read(KvArgs a, int quads, uint4* k, uint4* v) {
  using L = KvLayout<D>;
  constexpr int kLanes = D / 8;
  const uint32_t item = blockIdx.x * (kKvThreads / kLanes) + threadIdx.x / kLanes;
  const int sub = threadIdx.x % kLanes;
  const int h = (int)(item % (uint32_t)a.heads);
  const Quad q = quad_at<D>(a, quads, item / (uint32_t)a.heads, h);
  const int T = 1 << a.page_shift;
  uint4 x[4] = {}, y[4] = {};
  if (q.base) {
    const int t = (int)(q.slot & (T - 1));
    uint32_t kw[4], vw[4], kb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kw[i] = *reinterpret_cast<const uint32_t*>(q.base + L::k_codes(t + i) + 4 * sub);
      vw[i] = get_v_word<D>(q.base, T, t + i, sub);   // (of 128 channels: one load)
      kb[i] = q.base[L::k_scales(T, t + i) + (sub >> 2)];
    }
    const uint32_t vb = *reinterpret_cast<const uint32_t*>(q.base + L::v_scales(T, t, sub >> 2));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = kv_values8<BF16>(kw[i], kv_scale(kb[i]));
      y[i] = kv_values8<BF16>(vw[i], kv_scale((vb >> (8 * i)) & 0xffu));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if ((q.rows >> i) & 1u) {
      const int64_t at = ((q.row + i) * a.heads + h) * kLanes + sub;
      __builtin_nontemporal_store(__builtin_bit_cast(kv_u4, x[i]), reinterpret_cast<kv_u4*>(k + at));
      __builtin_nontemporal_store(__builtin_bit_cast(kv_u4, y[i]), reinterpret_cast<kv_u4*>(v + at));
    }
  if (a.starts) {   // rows of no sequence
    const int64_t before = a.start(0), after = a.start(a.n_seqs), row_size = (int64_t)a.heads * kLanes;
    for (int64_t r = blockIdx.x; r < before + a.rows - after; r += gridDim.x) {
      const int64_t row = r < before ? r : after + r - before;
      for (int64_t i = threadIdx.x; i < row_size; i += kKvThreads) k[row * row_size + i] = v[row * row_size + i] = uint4{0, 0, 0, 0};
    }
  }
}

// ------------------------------------------------------------------ eviction
constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;

struct EvictArgs {
  lam_kv_slots scores, positions, scores_out, positions_out;
  int32_t budget, recent, sinks, bound;   // bound: most tokens of a sequence
  int32_t moves;                          // most moves of a sequence's head
  int32_t head_dim;                       // where the selection makes the moves itself, else 0
  int32_t* kept;
  int32_t* lengths_out;
  int32_t* lists;   // of a long cache's holes and extra slots: [seq][head][2][moves]
};

// What one sequence's head selects from and writes to.
struct EvictHead {
  const float* sc;
  const int32_t* ps;   // or null: the slot
  float* so;
  int32_t* po;         // or null
  int32_t* kept;
  int len;

  __device__ __forceinline__ EvictHead(const KvArgs& a, const EvictArgs& e, int bh) {
    const int s = bh / a.heads, h = bh % a.heads;
    auto at = [&](const lam_kv_slots& x) -> int64_t { return s * x.seq_stride + h * x.head_stride; };
    len = min(a.length(s), e.bound);
    sc = static_cast<const float*>(e.scores.p_dev) + at(e.scores);
    ps = e.positions.p_dev ? static_cast<const int32_t*>(e.positions.p_dev) + at(e.positions) : nullptr;
    so = static_cast<float*>(e.scores_out.p_dev) + at(e.scores_out);
    po = e.positions_out.p_dev ? static_cast<int32_t*>(e.positions_out.p_dev) + at(e.positions_out) : nullptr;
    kept = e.kept + (int64_t)bh * e.budget;
  }
  __device__ __forceinline__ int pos(int t) const { return ps ? ps[t] : t; }
  // new slot t holds what old slot `from` held
  __device__ __forceinline__ void keep(int t, int from) const {
    kept[t] = from;
    so[t] = sc[from];
    if (po) po[t] = pos(from);
  }
  // nothing to evict: the tokens stay as they are
  __device__ __forceinline__ void keep_all(int budget) const {
    for (int t = threadIdx.x; t < budget; t += blockDim.x) {
      if (t < len) {
        keep(t, t);
      } else {
        kept[t] = -1;
        so[t] = 0.0f;
        if (po) po[t] = -1;
      }
    }
  }
};

// A wave moves one token: its codes by two bytes (a run has D/32 of them), its scales
// by one.
__device__ __forceinline__ void move_token(const KvArgs& a, int bh, int D, int from, int to) {
  const int s = bh / a.heads, h = bh % a.heads, T = 1 << a.page_shift, lane = threadIdx.x & 63;
  const int64_t pf = a.page(s, from >> a.page_shift), pt = a.page(s, to >> a.page_shift);
  if (pf < 0 || pt < 0) return;
  const int64_t head_bytes = (int64_t)T * (D + D / 16);
  const uint8_t* f = a.head_page(pf, h, head_bytes);
  uint8_t* d = a.head_page(pt, h, head_bytes);
  from &= T - 1;
  to &= T - 1;
  const int run = D / 32, blocks = D / kKvBlock;
  auto code_at = [&](int t, int i) {   // of the token's i-th byte of codes, the keys' D/2 first
    if (i < D / 2) return t * (D / 2) + i;
    i -= D / 2;
    return T * (D / 2) + (((t >> 2) * 16 + i / run) * 4 + (t & 3)) * run + i % run;
  };
  auto scale_at = [&](int t, int i) {
    return T * D + (i < blocks ? t * blocks + i : T * blocks + ((t >> 2) * blocks + i - blocks) * 4 + (t & 3));
  };
  for (int i = 2 * lane; i < D; i += 128)
    *reinterpret_cast<uint16_t*>(d + code_at(to, i)) = *reinterpret_cast<const uint16_t*>(f + code_at(from, i));
  if (lane < 2 * blocks) d[scale_at(to, lane)] = f[scale_at(from, lane)];
}

// Most moves of a head that its selection makes itself, which saves the launch that
// would.  Heads of 128 channels cut to 4,096 tokens, in a recorded graph with a copy of the lengths:
// 24 sequences of 8 heads with 1 move a head 13 us for 19, with 64 18 for 24, with 128
// 24 for 27, with 256 36 for 32; 96 sequences with 64 38 for 61, with 512 143 for 115;
// one sequence with 16 13 for 14, with 64 18 for 15.  (Not where the new lengths replace those
// that the other heads' selections still read.)
constexpr int kOwnMoves = 64;

// The largest of the threads' values (one barrier; tops: of the workgroup's own).
__device__ __forceinline__ int largest(int v, uint32_t* tops) {
  const uint32_t top = wave_max_u32((uint32_t)v ^ 0x80000000u);   // the order of signed numbers
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  uint32_t m = tops[0];
#pragma unroll
  for (int w = 1; w < kSelWaves; ++w) m = max(m, tops[w]);
  return __builtin_amdgcn_readfirstlane((int)(m ^ 0x80000000u));
}

// Order of the scores as unsigned integers: protected slots above all, NaN below all.
// newest: the largest position (an eviction fills holes from the tail, so the last slot
// need not have it).
__device__ __forceinline__ uint32_t evict_key(float s, int pos, int newest, int recent, int sinks) {
  if (pos < sinks || (int64_t)pos > (int64_t)newest - recent) return 0xffffffffu;
  if (s != s) return 0u;
  const uint32_t b = __float_as_uint(s + 0.0f);   // -0 counts as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Digits of a key, from the top: sign, exponent and two bits of the fraction
// spread weights over the counters of a histogram.
constexpr int kDigits = 3, kDigitBits[kDigits] = {11, 11, 10}, kDigitShift[kDigits] = {21, 10, 0};
constexpr int kBins = 1 << 11;

// One workgroup per sequence and head, the keys of up to 1,024 KPT slots in its
// registers (thread i has slots i, i + 1024, ...).  The budget-th largest key is
// found digit by digit with histograms in LDS; a wave whose digits are all the same
// (weights of 0, say) adds them at once; it ends as soon as a digit's keys all stay.
// Then holes below budget and slots kept beyond it are ranked by their place, and the i-th hole
// takes the i-th such slot.  Bound by its reading of scores and positions (the newest position is
// found first, so positions come from memory once and then from the caches) and by
// instructions of the workgroup's one compute unit.
// (A search bit by bit, each a count of all keys, took 25 us more for 32,768 slots.)
template <int KPT>
__global__ __launch_bounds__(kSelThreads) void k_kv_select(KvArgs a, EvictArgs e) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const EvictHead d(a, e, blockIdx.x);
  if (e.head_dim && blockIdx.x % a.heads == 0 && tid == 0)
    e.lengths_out[blockIdx.x / a.heads] = min(d.len, e.budget);
  if (d.len <= e.budget) {
    d.keep_all(e.budget);
    return;
  }
  // Rounds of 1,024 slots past the length are skipped, so that a call pays for its length
  // and not for KPT (4 heads of 43,136 slots cut by half 74 -> 55 us with the moves, 58 with the
  // newest position looked for; one of 14,349 cut to a tenth 26 -> 22).  The counts that are then not written follow all that are used.
  const int len = __builtin_amdgcn_readfirstlane(d.len);
  __shared__ int32_t move_to[kOwnMoves], move_from[kOwnMoves];
  if (tid < kOwnMoves) move_to[tid] = -1;
  constexpr int kCounts = KPT * kSelWaves;   // of 64 slots each, in the order of the slots
  __shared__ uint32_t hist[kBins], found[3];
  __shared__ uint32_t hole_at[kCounts], extra_at[kCounts], sums[2][kSelWaves];
  __shared__ uint16_t extras[KPT * kSelThreads / 2];

  // in batches whose loads are all on their way before the first is used
  constexpr int kBatch = KPT < 16 ? KPT : KPT > 32 ? 8 : 16;   // (16 of 64 spill)
  int newest = len - 1;
  if (d.ps) {   // (read twice, the second time from the caches: held in registers, they spill)
    constexpr int kTops = KPT < 16 ? KPT : 16;
    int top = (int)0x80000000u;
#pragma unroll 1
    for (int t0 = tid; t0 < len; t0 += kTops * kSelThreads) {
      int p[kTops];
#pragma unroll
      for (int j = 0; j < kTops; ++j) p[j] = d.ps[(uint32_t)min(t0 + j * kSelThreads, len - 1)];
#pragma unroll
      for (int j = 0; j < kTops; ++j) top = max(top, p[j]);
    }
    newest = largest(top, sums[0]);
  }
  uint32_t key[KPT];
  auto fill = [&](auto has_positions) {
#pragma unroll
    for (int k0 = 0; k0 < KPT; k0 += kBatch) {
      if (k0 * kSelThreads >= len) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) key[k0 + j] = 0u;
        continue;
      }
      float s[kBatch];
      int p[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t t = min((k0 + j) * kSelThreads + tid, len - 1);
        s[j] = d.sc[t];
        p[j] = has_positions ? d.ps[t] : (int)t;
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        key[k0 + j] = (k0 + j) * kSelThreads + tid < len ? evict_key(s[j], p[j], newest, e.recent, e.sinks) : 0u;
    }
  };
  if (d.ps) fill(std::true_type{}); else fill(std::false_type{});
  // the budget-th largest key: the digits found so far, and how many slots of theirs stay
  uint32_t least = 0;
  int ties = e.budget;
  bool exact = false;   // all of them do
#pragma unroll
  for (int n = 0; n < kDigits; ++n) {
    if (exact) break;
    const int shift = kDigitShift[n];
    const uint32_t above = n == 0 ? 0u : 0xffffffffu << kDigitShift[n == 0 ? 0 : n - 1];
    for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
      if (k * kSelThreads >= len) break;
      const bool in = k * kSelThreads + tid < len && (key[k] & above) == least;
      const unsigned long long m = __ballot(in);
      if (m == 0) continue;
      const uint32_t digit = (key[k] >> shift) & (kBins - 1);
      const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)digit, (int)__builtin_ctzll(m));
      if (__ballot(in && digit != one) == 0) {
        if (lane == 0) atomicAdd(&hist[one], (uint32_t)__popcll(m));
      } else if (in) {
        atomicAdd(&hist[digit], 1u);
      }
    }
    __syncthreads();
    // thread i holds bins kBins - 1 - 2 i and the one below; sums from the top
    const uint32_t c0 = hist[kBins - 1 - 2 * tid], c1 = hist[kBins - 2 - 2 * tid];
    const uint32_t upto = wave_scan_u32(c0 + c1);
    if (lane == 63) sums[0][wave] = upto;
    __syncthreads();
    uint32_t before = upto - c0 - c1;
    for (int w = 0; w < wave; ++w) before += sums[0][w];
    const uint32_t need = (uint32_t)ties;
    if (before < need && before + c0 + c1 >= need) {
      const bool first = before + c0 >= need;
      found[0] = (uint32_t)(kBins - 1 - 2 * tid - (first ? 0 : 1));
      found[1] = need - before - (first ? 0u : c0);
      found[2] = first ? c0 : c1;
    }
    __syncthreads();
    least |= found[0] << shift;
    ties = (int)found[1];
    exact = found[1] == found[2];
  }
  const unsigned long long low = (1ull << lane) - 1;
  // sums of the counts before each group of 64 slots
  auto scan = [&](uint32_t* c, uint32_t* s) {
    const uint32_t mine = tid < kCounts ? c[tid] : 0u;
    const uint32_t upto = wave_scan_u32(mine);
    if (lane == 63) s[wave] = upto;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += s[w];
    if (tid < kCounts) c[tid] = before + upto - mine;
  };
  if (!exact) {   // (hole_at for the ranks of equal keys)
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
      if (k * kSelThreads >= len) break;
      const unsigned long long m = __ballot(key[k] == least && k * kSelThreads + tid < len);
      if (lane == 0) hole_at[k * kSelWaves + wave] = (uint32_t)__popcll(m);
    }
    __syncthreads();
    scan(hole_at, sums[0]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
      if (k * kSelThreads >= len) break;
      const bool eq = key[k] == least && k * kSelThreads + tid < len;
      const int rank = (int)(hole_at[k * kSelWaves + wave] + __popcll(__ballot(eq) & low));
      if (eq && rank >= ties) key[k] = 0;              // evicted
      else if (eq && least == 0) key[k] = 1;           // (a key of 0 that stays)
    }
    __syncthreads();
  }
  least = max(least, 1u);   // (not exact: keys of 0 that stay are 1 now; slots past the length have 0)
#pragma unroll
  for (int k = 0; k < KPT; ++k) {
    if (k * kSelThreads >= len) break;
    const int t = k * kSelThreads + tid;
    const unsigned long long mh = __ballot(t < e.budget && key[k] < least), mx = __ballot(t >= e.budget && key[k] >= least);
    if (lane == 0) {
      hole_at[k * kSelWaves + wave] = (uint32_t)__popcll(mh);
      extra_at[k * kSelWaves + wave] = (uint32_t)__popcll(mx);
    }
  }
  __syncthreads();
  scan(hole_at, sums[0]);
  scan(extra_at, sums[1]);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < KPT; ++k) {
    if (k * kSelThreads >= len) break;
    const int t = k * kSelThreads + tid;
    const bool extra = t >= e.budget && key[k] >= least;
    const unsigned long long m = __ballot(extra);
    if (extra) extras[extra_at[k * kSelWaves + wave] + (uint32_t)__popcll(m & low)] = (uint16_t)(t - e.budget);
  }
  __syncthreads();
#pragma unroll
  for (int k0 = 0; k0 < KPT; k0 += kBatch) {
    if (k0 * kSelThreads >= e.budget) break;
    int from[kBatch], p[kBatch];
    float s[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int k = k0 + j, t = k * kSelThreads + tid;
      const bool hole = t < e.budget && key[k] < least;
      const uint32_t rank = hole_at[k * kSelWaves + wave] + (uint32_t)__popcll(__ballot(hole) & low);
      from[j] = hole ? e.budget + (int)extras[rank] : min(t, e.budget - 1);
      if (hole && e.head_dim) {   // (at most e.moves of them)
        move_to[rank] = t;
        move_from[rank] = from[j];
      }
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) s[j] = d.sc[(uint32_t)from[j]];
    if (d.po) {
#pragma unroll
      for (int j = 0; j < kBatch; ++j) p[j] = d.pos(from[j]);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int t = (k0 + j) * kSelThreads + tid;
      if (t < e.budget) {
        d.kept[t] = from[j];
        d.so[t] = s[j];
        if (d.po) d.po[t] = p[j];
      }
    }
  }
  if (!e.head_dim) return;
  __syncthreads();
  for (int i = wave; i < e.moves; i += kSelWaves) {
    const int to = __builtin_amdgcn_readfirstlane(move_to[i]);
    if (to < 0) break;   // (the i-th hole is there if the one after it is)
    move_token(a, blockIdx.x, e.head_dim, __builtin_amdgcn_readfirstlane(move_from[i]), to);
  }
}

// The same for longer caches, whose keys are made from memory each time: the
// newest position, the budget-th largest key digit by digit (four histograms of 256 counts),
// then one pass over the slots in order, and lists in memory.  Bound by the round trips of one
// workgroup a head: 4 heads of 131,072 slots cut to 60,000 take 438 us (3 for the bytes).
__global__ __launch_bounds__(kSelThreads) void k_kv_select_long(KvArgs a, EvictArgs e) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const EvictHead d(a, e, blockIdx.x);
  if (d.len <= e.budget) {
    d.keep_all(e.budget);
    return;
  }
  int32_t* holes = e.lists + (int64_t)blockIdx.x * 2 * e.moves;
  int32_t* extras = holes + e.moves;
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];
  __shared__ int32_t cnt[2][3][kSelWaves];
  __shared__ uint32_t tops[kSelWaves];
  int newest = d.len - 1;
  if (d.ps) {
    int top = (int)0x80000000u;
    for (int t = tid; t < d.len; t += kSelThreads) top = max(top, d.ps[t]);
    newest = largest(top, tops);
  }
  auto key_of = [&](int t) { return evict_key(d.sc[t], d.pos(t), newest, e.recent, e.sinks); };

  uint32_t prefix = 0, need = (uint32_t)e.budget;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    const uint32_t above = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int t = tid; t < d.len; t += kSelThreads) {
      const uint32_t k = key_of(t);
      if ((k & above) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      // lane l holds the digits 255 - 4 l down to 252 - 4 l; sums from the top
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j] = hist[255 - 4 * lane - j];
      const uint32_t upto = wave_scan_u32(sum);
      uint32_t before = upto - sum;
      if (before < need && upto >= need) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (before < need && before + c[j] >= need) {
            found[0] = 255 - 4 * lane - j;
            found[1] = need - before;
          }
          before += c[j];
        }
      }
    }
    __syncthreads();
    prefix |= found[0] << shift;
    need = found[1];
  }

  // need: how many slots of the threshold's key stay, the lowest ones
  int ties = 0, n_holes = 0, n_extras = 0, buf = 0;
  for (int t0 = 0; t0 < d.len; t0 += kSelThreads, buf ^= 1) {
    const int t = t0 + tid;
    const uint32_t k = t < d.len ? key_of(t) : 0u;
    const bool eq = t < d.len && k == prefix;
    const unsigned long long me = __ballot(eq), low = (1ull << lane) - 1;
    if (lane == 0) cnt[buf][0][wave] = (int)__popcll(me);
    __syncthreads();
    int rank = ties + (int)__popcll(me & low);
    for (int w = 0; w < kSelWaves; ++w) {
      if (w < wave) rank += cnt[buf][0][w];
      ties += cnt[buf][0][w];
    }
    const bool stays = t < d.len && (k > prefix || (eq && rank < (int)need));
    const bool hole = t < e.budget && !stays, extra = t >= e.budget && stays;
    const unsigned long long mh = __ballot(hole), mx = __ballot(extra);
    if (lane == 0) {
      cnt[buf][1][wave] = (int)__popcll(mh);
      cnt[buf][2][wave] = (int)__popcll(mx);
    }
    __syncthreads();
    int ih = n_holes + (int)__popcll(mh & low), ix = n_extras + (int)__popcll(mx & low);
    for (int w = 0; w < kSelWaves; ++w) {
      if (w < wave) {
        ih += cnt[buf][1][w];
        ix += cnt[buf][2][w];
      }
      n_holes += cnt[buf][1][w];
      n_extras += cnt[buf][2][w];
    }
    if (hole) holes[ih] = t;
    if (extra) extras[ix] = t;
    if (t < e.budget && stays) d.keep(t, t);
  }
  __syncthreads();
  for (int i = tid; i < n_holes; i += kSelThreads) d.keep(holes[i], extras[i]);
}

// Moves the tokens that have a new slot: D/8 lanes take four slots, the units in
// which value codes lie.  Sources lie at or beyond budget and destinations below it,
// so no move reads what another wrote.  Bound by memory, at more than the codes'
// bytes: a token's value codes are a quarter of every 16 bytes of 2 D bytes, and
// what is kept of a long tail lies apart.  192 heads' 6,144 moves of 128 channels take 127 to
// 145 us (the bytes alone 62 at a copy's rate, with the lines' other tokens 102); the same with every source token
// next to the last 82 to 90 us for 8,192.  (Tokens that stay reading their own place,
// so that no load hangs on a branch, were 7 % slower, two units a lane group 9 %.)
template <int D>
__global__ __launch_bounds__(kKvThreads) void k_kv_move(KvArgs a, EvictArgs e) {
  using L = KvLayout<D>;
  constexpr int kLanes = D / 8;
  const int bh = blockIdx.y;
  const int s = bh / a.heads, h = bh % a.heads;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0)
    e.lengths_out[s] = min(min(a.length(s), e.bound), e.budget);
  const int T = 1 << a.page_shift;
  const int t0 = 4 * (int)(blockIdx.x * (kKvThreads / kLanes) + threadIdx.x / kLanes);
  const int sub = threadIdx.x % kLanes;
  if (t0 >= e.budget) return;
  const int32_t* kept = e.kept + (int64_t)bh * e.budget;
  int from[4];
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    from[i] = t0 + i < e.budget ? kept[t0 + i] : -1;
    any |= from[i] >= 0 && from[i] != t0 + i;
  }
  if (!any) return;
  const int64_t pd = a.page(s, t0 >> a.page_shift);
  int64_t pf[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) pf[i] = a.page(s, max(from[i], 0) >> a.page_shift);
  const uint8_t* f[4];   // the sources' pages, null: nothing to move
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool move = from[i] >= 0 && from[i] != t0 + i && pd >= 0 && pf[i] >= 0;
    f[i] = move ? a.head_page(pf[i], h, L::head_bytes(T)) : nullptr;
    from[i] &= T - 1;
  }
  uint8_t* d = a.head_page(pd, h, L::head_bytes(T));   // (used only where something moves)
  const int td = t0 & (T - 1);
  uint32_t kw[4], vw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!f[i]) continue;
    kw[i] = *reinterpret_cast<const uint32_t*>(f[i] + L::k_codes(from[i]) + 4 * sub);
    vw[i] = get_v_word<D>(f[i], T, from[i], sub);
  }
  // the lane's scales: block b of the i-th token
  const int i = sub / (D / 32), b = sub % (D / 32);
  const uint8_t* fi = i == 0 ? f[0] : i == 1 ? f[1] : i == 2 ? f[2] : f[3];
  const int ti = i == 0 ? from[0] : i == 1 ? from[1] : i == 2 ? from[2] : from[3];
  uint8_t ks = 0, vs = 0;
  if (fi) {
    ks = fi[L::k_scales(T, ti) + b];
    vs = fi[L::v_scales(T, ti, b)];
  }
  if (D == 128 && f[0] && f[1] && f[2] && f[3]) {
    *reinterpret_cast<uint4*>(d + L::v_codes(T, td, sub)) = uint4{vw[0], vw[1], vw[2], vw[3]};
  } else {
#pragma unroll
    for (int n = 0; n < 4; ++n)
      if (f[n]) put_v_word<D>(d, T, td + n, sub, vw[n]);
  }
#pragma unroll
  for (int n = 0; n < 4; ++n)
    if (f[n]) *reinterpret_cast<uint32_t*>(d + L::k_codes(td + n) + 4 * sub) = kw[n];
  if (fi) {
    d[L::k_scales(T, td + i) + b] = ks;
    d[L::v_scales(T, td + i, b)] = vs;
  }
}

bool wide_rows(const void* p, int64_t row, int64_t head) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && row % 8 == 0 && head % 8 == 0;
}

// workgroups of kKvThreads lanes, D/8 lanes a quad and head; quads: of a sequence, where all have as many rows
lam_status quad_grid(const lam_kv_view& v, int* quads, unsigned* grid) {
  int64_t units;
  *quads = 0;
  if (v.starts_dev) {
    units = v.rows / 4 + 2 * (int64_t)v.n_seqs;
  } else {
    const int64_t n = v.rows / v.n_seqs;
    *quads = (int)(n / 4 + (n % 4 > 1 ? 2 : 1));   // n rows from any slot on touch no more
    units = *quads * (int64_t)v.n_seqs;
  }
  const int64_t per = kKvThreads / (v.head_dim / 8), items = units * v.kv_heads, blocks = (items + per - 1) / per;
  LAM_CHECK(items < (1LL << 31) && blocks <= most_blocks(kKvThreads), LAM_EINVAL,
            "too many rows or sequences for one launch");
  *grid = (unsigned)blocks;
  return LAM_OK;
}

}  // namespace

lam_status launch_kv_append(lam_ctx* ctx, const lam_kv_view& v, const void* k, int64_t k_row, int64_t k_head,
                            const void* val, int64_t v_row, int64_t v_head, const lam_kv_slots& weights,
                            const lam_kv_slots& positions, const int32_t* first, uint32_t* status) {
  unsigned grid;
  int quads;
  LAM_TRY(quad_grid(v, &quads, &grid));
  const KvArgs a = KvArgs::of(v);
  const RowArgs ka{k, k_row, k_head, wide_rows(k, k_row, k_head)}, va{val, v_row, v_head, wide_rows(val, v_row, v_head)};
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_append", &e0, &e1));
#define LAM_GO(D, BF)                                                                                             \
  launch(k_kv_append<D, BF>, dim3(grid), kKvThreads, ctx->stream, e0, e1, a, quads, ka, va, weights, positions, first, \
         status)
  LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

lam_status launch_kv_read(lam_ctx* ctx, const lam_kv_view& v, void* k, void* val) {
  unsigned grid;
  int quads;
  LAM_TRY(quad_grid(v, &quads, &grid));
  const KvArgs a = KvArgs::of(v);
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_read", &e0, &e1));
#define LAM_GO(D, BF)                                                                          \
  launch(k_kv_read<D, BF>, dim3(grid), kKvThreads, ctx->stream, e0, e1, a, quads, static_cast<uint4*>(k), \
         static_cast<uint4*>(val))
  LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

lam_status launch_kv_evict(lam_ctx* ctx, const lam_kv_view& v, const lam_kv_slots& scores,
                           const lam_kv_slots& positions, int32_t budget, int32_t recent, int32_t sinks,
                           int32_t* kept, const lam_kv_slots& scores_out, const lam_kv_slots& positions_out,
                           int32_t* lengths_out) {
  const KvArgs a = KvArgs::of(v);
  const int64_t pairs = (int64_t)v.n_seqs * v.kv_heads;
  LAM_CHECK(pairs < 65536, LAM_EINVAL, "n_seqs * kv_heads must be below 65536");
  EvictArgs e{scores, positions, scores_out, positions_out, budget, recent, sinks};
  const int64_t cap = (int64_t)v.table_cols * v.page_size;
  e.bound = (int32_t)std::min<int64_t>(cap, scores.cols);
  if (positions.p_dev) e.bound = std::min(e.bound, positions.cols);
  e.moves = std::max(0, std::min(budget, e.bound - budget));
  e.kept = kept;
  e.lengths_out = lengths_out;
  const bool apart = lengths_out + v.n_seqs <= v.lengths_dev || v.lengths_dev + v.n_seqs <= lengths_out;
  if (e.moves <= kOwnMoves && e.bound <= 64 * kSelThreads && apart) e.head_dim = v.head_dim;
  const int per = kKvThreads / (v.head_dim / 8) * 4;   // slots a workgroup of the move
  const int64_t move_blocks = ((int64_t)std::min(budget, std::max(e.bound, 1)) + per - 1) / per;
  LAM_CHECK(move_blocks <= most_blocks(kKvThreads), LAM_EINVAL, "too many slots for one launch");
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_select", &e0, &e1));
#define LAM_GO(KPT) launch(k_kv_select<KPT>, dim3((unsigned)pairs), kSelThreads, ctx->stream, e0, e1, a, e)
  if (e.bound <= 2 * kSelThreads) LAM_GO(2);
  else if (e.bound <= 8 * kSelThreads) LAM_GO(8);
  else if (e.bound <= 32 * kSelThreads) LAM_GO(32);
  else if (e.bound <= 64 * kSelThreads) LAM_GO(64);
#undef LAM_GO
  else {
    void* lists;
    LAM_TRY(kv_scratch(ctx, (size_t)pairs * 2 * (size_t)e.moves * 4, &lists));
    e.lists = static_cast<int32_t*>(lists);
    launch(k_kv_select_long, dim3((unsigned)pairs), kSelThreads, ctx->stream, e0, e1, a, e);
  }
  LAM_HIP(hipGetLastError());
  if (e.head_dim) return LAM_OK;
  LAM_TRY(prof_launch_events(ctx, "kv_move", &e0, &e1));
  const dim3 grid((unsigned)move_blocks, (unsigned)pairs);
#define LAM_GO(D) launch(k_kv_move<D>, grid, kKvThreads, ctx->stream, e0, e1, a, e)
  if (v.head_dim == 64) LAM_GO(64); else if (v.head_dim == 128) LAM_GO(128); else LAM_GO(256);
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

}  // namespace lam
