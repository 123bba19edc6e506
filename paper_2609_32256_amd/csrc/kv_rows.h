// What the calls that write rows into the 4-bit cache share: rows of 16-bit values on their
// way to codes, the quads of slots that a workgroup's lanes take, and the launch over them.
#pragma once

#include <hip/hip_runtime.h>

#include "kv.h"
#include "lam_internal.h"
#include "wave.h"

namespace lam {

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

// Eight channels of a row.  Rows are read once here, and written once by
// the read: non-temporal, 284 -> 259 us for 131,072 rows of 8 heads of 128 channels both ways, the rate of a copy.
__device__ __forceinline__ kv_u4 load_raw8(const void* p, int64_t at, bool wide) {
  const uint16_t* h = static_cast<const uint16_t*>(p) + at;
  if (wide) return __builtin_nontemporal_load(reinterpret_cast<const kv_u4*>(h));
  kv_u4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = (uint32_t)h[2 * j] | ((uint32_t)h[2 * j + 1] << 16);
  return w;
}

// They as float32.
template <bool BF16>
__device__ __forceinline__ void unpack8(kv_u4 w, float x[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t u = w[j];   // (a bit cast of w[j] itself takes the first element)
    if constexpr (BF16) {
      x[2 * j] = __uint_as_float(u << 16);
      x[2 * j + 1] = __uint_as_float(u & 0xffff0000u);
    } else {
      const kv_h2 v = __builtin_bit_cast(kv_h2, u);
      x[2 * j] = (float)v[0];
      x[2 * j + 1] = (float)v[1];
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t at, bool wide, float x[8]) {
  unpack8<BF16>(load_raw8(p, at, wide), x);
}

// The codes of eight channels and their block's scale byte.  Four lanes share
// a block: its largest |x| goes round the quad.  6 * 2^e >= amax with amax =
// m 2^x, m in [1, 2), gives e = x - 2 for m <= 1.5 and x - 1 above; the
// conversion instruction divides by 2^e and rounds to nearest, ties to even.
__device__ __forceinline__ uint32_t quantize8(float x[8], uint32_t* byte, bool* bad, bool* over) {
  // sizes in the order of their bits, what is not finite above all
  constexpr uint32_t kInf = 0x7f800000u, kLargest = 0x47400000u;   // 49152
  auto size = [&](int j) { return __float_as_uint(x[j]) & 0x7fffffffu; };
  uint32_t b = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) b = max(b, size(j));
  if (__any(b >= kInf)) {
    *bad |= b >= kInf;
    b = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = size(j) < kInf ? x[j] : 0.0f;
      b = max(b, size(j));
    }
  }
  b = quad_max_u32(b);
  *over |= b > kLargest;
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

// Stores a quad's value codes and scale bytes of eight channels, of the slots that are the call's.
template <int D>
__device__ __forceinline__ void put_values(const Quad& q, int T, int sub, const uint32_t vw[4], const uint32_t vb[4]) {
  using L = KvLayout<D>;
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
}

// And the key codes and scale byte of place t of a head's page.
template <int D>
__device__ __forceinline__ void put_key(uint8_t* base, int T, int t, int sub, uint32_t w, uint32_t b) {
  using L = KvLayout<D>;
  *reinterpret_cast<uint32_t*>(base + L::k_codes(t) + 4 * sub) = w;
  if ((sub & 3) == 0) base[L::k_scales(T, t) + (sub >> 2)] = (uint8_t)b;
}

// Position of the quad's i-th slot: what its sequence begins with and the row, or the slot.
__device__ __forceinline__ int32_t quad_pos(const Quad& q, int i, const int32_t* first) {
  return first ? (int32_t)(first[q.s] + (q.row + i - q.first_row)) : (int32_t)(q.slot + i);
}

// Weights and positions of a head's new tokens: lane i has token i's.
__device__ __forceinline__ void put_slots(const KvArgs& a, const Quad& q, int h, int sub, const lam_kv_slots& weights,
                                          const lam_kv_slots& positions, const int32_t* first) {
  if (sub >= 4 || !((q.rows >> sub) & 1u)) return;
  const int64_t slot = q.slot + sub;
  if (weights.p_dev && slot < weights.cols)
    static_cast<float*>(weights.p_dev)[q.s * weights.seq_stride + h * weights.head_stride + slot] = 0.0f;
  if (positions.p_dev && slot < positions.cols)
    static_cast<int32_t*>(positions.p_dev)[q.s * positions.seq_stride + h * positions.head_stride + slot] =
        quad_pos(q, sub, first);
}

// What lam_kv_append counts.  All lanes of the wave.
__device__ __forceinline__ void count_quad(const KvArgs& a, const Quad& q, int sub, bool bad, bool over, uint32_t* status) {
  count_in(status, 0, bad);
  count_in(status, 1, over);
  // rows without a place: of this quad, and (once) those of no sequence
  uint32_t lost = !q.base && sub == 0 ? (uint32_t)__popc(q.rows) : 0u;
  if (a.starts && blockIdx.x == 0 && threadIdx.x == 0)
    lost += (uint32_t)(a.start(0) + a.rows - a.start(a.n_seqs)) * (uint32_t)a.heads;
  if (lost) atomicAdd(status + 2, lost);
}

inline bool wide_rows(const void* p, int64_t row, int64_t head) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && row % 8 == 0 && head % 8 == 0;
}

// Units of quads that cover a call's rows; quads: those of a sequence, where all have as many rows.
inline int64_t quad_units(const lam_kv_view& v, int* quads) {
  *quads = 0;
  if (v.starts_dev) return v.rows / 4 + 2 * (int64_t)v.n_seqs;
  const int64_t n = v.rows / v.n_seqs;
  *quads = (int)(n / 4 + (n % 4 > 1 ? 2 : 1));   // n rows from any slot on touch no more
  return *quads * (int64_t)v.n_seqs;
}

}  // namespace lam
