// Attention over the 4-bit key/value cache (include/lam.h, lam_kv_attend).
//
// A workgroup takes 16 query rows that share a key/value head (the rows of the
// group's heads for one token, or of several tokens) and a part of the length.
// Its waves walk the part in strips of 32 tokens with the running maximum and
// sum of a softmax, all on the matrix units:
//
//   S^T = K Q^T   A operand: 16 tokens' keys, converted from their codes in
//                 registers; B operand: the 16 query rows.  A lane supplies the
//                 D/4 channels of its quarter of the row, which are consecutive
//                 in memory: the order of the reduction is free as long as both
//                 operands have the same.
//   O^T += V^T P^T   A lane's scores are those of tokens 4 g + i and 16 + 4 g + i
//                 (g = lane / 16, i < 4) and one query: taken as they lie they are
//                 a B operand whose reduction runs over those tokens, so no lane
//                 exchanges anything.  The value codes are stored by four tokens
//                 and runs of D/16 channels for the A operand of the same order.
//
// Conversions are one instruction per two values with the scale applied; values
// of two tokens are then paired by one move each.
#include <hip/hip_ext.h>

#include <algorithm>

#include "kv.h"
#include "lam_internal.h"
#include "wave.h"

namespace lam {
namespace {

constexpr int kAttThreads = 256;
constexpr int kAttWaves = kAttThreads / 64;
constexpr int kAttRows = 16;

// The reference of a row's exponentials is at least its maximum so far less
// 2^kSpan and at most 2^-kLift of it when it was set: the weights reach 2^15,
// within float16, and those 2^-21 below the maximum are still normal numbers.
constexpr float kLift = 7.0f, kSpan = 15.0f;
constexpr float kNoMax = -3.0e38f;   // no token seen yet

struct AttendArgs {
  KvArgs c;
  const uint16_t* q;
  int64_t q_row, q_head;
  int q_wide;             // every eight channels of q are a 16-byte load
  int q_heads, group;
  int causal;
  float scale2;           // scale * log2(e)
  int64_t cut;            // lengths are cut to it
  int tiles_per_seq;      // where every sequence has the same number of rows
  int splits, part;       // parts of the length, and their tokens (a multiple of kKvStrip * kAttWaves)
  lam_kv_slots mask, weights;
  uint16_t* out;
  float* lse;             // natural logarithm, the caller's
  float* lse2;            // base 2, for the weights
  float* part_m;          // [row * q_heads + head][splits]
  float* part_l;
  float* part_o;          // [row * q_heads + head][splits][D]
};

// The rows of a tile: tile `t` of the call, in order of sequences.
struct TileRows {
  int s;             // sequence, -1: an empty tile
  int64_t first;     // its first row of the call
  int n;             // its rows
  int r0;            // first of the tile's 16 (row, head of the group) pairs, row-major
  int pairs;         // pairs of the sequence
  int len, end_full; // cached tokens, cut and not
};

__device__ __forceinline__ TileRows tile_rows(const AttendArgs& a, int64_t t) {
  TileRows w;
  if (!a.c.starts) {
    w.s = (int)(t / a.tiles_per_seq);
    w.r0 = (int)(t % a.tiles_per_seq) * kAttRows;
  } else {
    // sequence s has its tiles from floor(start(s) * group / 16) + s on, a bound
    // that leaves room for every partial tile and that a search can use
    int lo = 0, hi = a.c.n_seqs;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (a.c.start(m) * a.group / kAttRows + m <= t) lo = m; else hi = m;
    }
    w.s = lo;
    w.r0 = (int)min((t - (a.c.start(lo) * a.group / kAttRows + lo)) * kAttRows, (int64_t)0x7fffff00);
  }
  w.first = a.c.start(w.s);
  w.n = (int)max((int64_t)0, a.c.start(w.s + 1) - w.first);
  w.pairs = w.n * a.group;
  w.end_full = a.c.length(w.s);
  w.len = (int)min((int64_t)w.end_full, a.cut);
  if (w.r0 < 0 || w.r0 >= w.pairs) w.s = -1;
  return w;
}

// Tokens that pair r of the sequence sees: those below this.
__device__ __forceinline__ int pair_end(const AttendArgs& a, const TileRows& w, int r) {
  if (!a.causal) return w.len;
  return max(0, min(w.len, w.end_full - w.n + r / a.group + 1));
}

// B operands of the 16 query rows: lane (c, g) holds channels g D/4 + 8 j + 0..7
// of pair r0 + c as step j.
template <int D>
__device__ __forceinline__ void load_q(const AttendArgs& a, const TileRows& w, int h, int r0, uint4 q[D / 32]) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int r = r0 + c;
  const int rr = min(r, w.pairs - 1);
  const uint16_t* p =
      a.q + (w.first + rr / a.group) * a.q_row + (int64_t)(h * a.group + rr % a.group) * a.q_head + g * (D / 4);
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    uint4 u;
    if (a.q_wide) {
      u = *reinterpret_cast<const uint4*>(p + 8 * j);
    } else {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (uint32_t)p[8 * j + 2 * i] | ((uint32_t)p[8 * j + 2 * i + 1] << 16);
      u = uint4{x[0], x[1], x[2], x[3]};
    }
    q[j] = r < w.pairs ? u : uint4{0, 0, 0, 0};
  }
}

template <bool BF16>
__device__ __forceinline__ kv_f4 mfma(uint4 x, uint4 y, kv_f4 z) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_b8, x), __builtin_bit_cast(kv_b8, y), z, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(kv_h8, x), __builtin_bit_cast(kv_h8, y), z, 0, 0, 0);
}

// One lane's codes and scales of a strip's keys or values, as they lie in memory.
template <int D>
struct Codes {
  uint32_t w[2][D / 32];
  uint32_t s[2];
};

template <int D>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t w[D / 32]) {
  if constexpr (D == 64) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x, w[1] = u.y;
  } else {
#pragma unroll
    for (int j = 0; j < D / 128; ++j) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + 16 * j);
      w[4 * j] = u.x, w[4 * j + 1] = u.y, w[4 * j + 2] = u.z, w[4 * j + 3] = u.w;
    }
  }
}

// Keys: tile kt of a strip, token t + 16 kt + c, the lane's quarter of the channels.
template <int D>
__device__ __forceinline__ void load_keys(const uint8_t* page, int T, int t, Codes<D>& k) {
  using L = KvLayout<D>;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const int tt = t + 16 * kt + c;
    load_words<D>(page + L::k_codes(tt) + g * (D / 8), k.w[kt]);
    const uint8_t* s = page + L::k_scales(T, tt);
    if constexpr (D == 64) k.s[kt] = s[g >> 1];
    else if constexpr (D == 128) k.s[kt] = s[g];
    else k.s[kt] = *reinterpret_cast<const uint16_t*>(s + 2 * g);
  }
}

// Values: half `half` of a strip, tokens t + 16 half + 4 g + 0..3, run c of the channels.
template <int D>
__device__ __forceinline__ void load_vals(const uint8_t* page, int T, int t, Codes<D>& v) {
  using L = KvLayout<D>;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int tt = t + 16 * half + 4 * g;
    load_words<D>(page + L::v_codes(T, tt, c), v.w[half]);
    v.s[half] = *reinterpret_cast<const uint32_t*>(page + L::v_scales(T, tt, c * (D / 16) / kKvBlock));
  }
}

// A operands of a strip's keys times the queries: scores of tokens 16 kt + 4 g + i.
template <int D, bool BF16>
__device__ __forceinline__ void key_operand(const Codes<D>& k, int kt, uint4 x[D / 32]) {
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const uint32_t byte = D == 256 ? (j < 4 ? k.s[kt] & 0xffu : k.s[kt] >> 8) : k.s[kt];
    x[j] = kv_values8<BF16>(k.w[kt][j], kv_scale(byte));
  }
}

// Two values of token TOK (of four) of a half's codes: channels 2 JP and 2 JP + 1 of the run.
template <int D, int TOK, int JP>
__device__ __forceinline__ uint32_t val_pair(const uint32_t w[D / 32], float s) {
  constexpr int byte = TOK * (D / 32) + JP;
  return kv_values<false, byte % 4>(w[byte / 4], s);
}

// O^T += V^T P^T of a strip: one product per channel of the lane's run.
template <int D, int JP>
__device__ __forceinline__ void add_values(const Codes<D>& v, const float s[2][4], uint4 p, kv_f4* o) {
  if constexpr (JP < D / 32) {
    uint4 even, odd;
    const uint32_t a0 = val_pair<D, 0, JP>(v.w[0], s[0][0]), a1 = val_pair<D, 1, JP>(v.w[0], s[0][1]);
    const uint32_t a2 = val_pair<D, 2, JP>(v.w[0], s[0][2]), a3 = val_pair<D, 3, JP>(v.w[0], s[0][3]);
    const uint32_t b0 = val_pair<D, 0, JP>(v.w[1], s[1][0]), b1 = val_pair<D, 1, JP>(v.w[1], s[1][1]);
    const uint32_t b2 = val_pair<D, 2, JP>(v.w[1], s[1][2]), b3 = val_pair<D, 3, JP>(v.w[1], s[1][3]);
    even = uint4{__builtin_amdgcn_perm(a1, a0, 0x05040100u), __builtin_amdgcn_perm(a3, a2, 0x05040100u),
                 __builtin_amdgcn_perm(b1, b0, 0x05040100u), __builtin_amdgcn_perm(b3, b2, 0x05040100u)};
    odd = uint4{__builtin_amdgcn_perm(a1, a0, 0x07060302u), __builtin_amdgcn_perm(a3, a2, 0x07060302u),
                __builtin_amdgcn_perm(b1, b0, 0x07060302u), __builtin_amdgcn_perm(b3, b2, 0x07060302u)};
    o[2 * JP] = mfma<false>(even, p, o[2 * JP]);
    o[2 * JP + 1] = mfma<false>(odd, p, o[2 * JP + 1]);
    add_values<D, JP + 1>(v, s, p, o);
  }
}

// Which of a strip's tokens the lane's query sees: bit 4 half + i for token t0 + 16 half + 4 g + i.
__device__ __forceinline__ uint32_t seen_bits(const AttendArgs& a, int s, int h, int t0, int end) {
  const int g = (threadIdx.x & 63) >> 4;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int t = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
    bool in = t < end;
    if (a.mask.p_dev)
      in = in && t < a.mask.cols &&
           static_cast<const uint8_t*>(a.mask.p_dev)[s * a.mask.seq_stride + h * a.mask.head_stride + t] != 0;
    m |= (in ? 1u : 0u) << i;
  }
  return m;
}

__device__ __forceinline__ uint32_t pack_half(float x, float y) {
  const kv_h2 v{(_Float16)x, (_Float16)y};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ uint16_t to_out(float x, bool bf16) {
  if (bf16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  return __builtin_bit_cast(uint16_t, (_Float16)x);
}

template <int D, bool BF16>
__global__ __launch_bounds__(kAttThreads) void k_kv_attend(AttendArgs a) {
  constexpr int kRun = D / 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  int64_t id = blockIdx.x;
  const int split = (int)(id % a.splits);
  id /= a.splits;
  const int h = (int)(id % a.c.heads);
  const TileRows w = tile_rows(a, id / a.c.heads);
  if (w.s < 0) return;
  const int T = 1 << a.c.page_shift;
  const int64_t head_bytes = KvLayout<D>::head_bytes(T);

  uint4 q[D / 32];
  load_q<D>(a, w, h, w.r0, q);
  const int end = pair_end(a, w, min(w.r0 + c, w.pairs - 1));
  const int end_first = pair_end(a, w, w.r0), end_last = pair_end(a, w, min(w.r0 + kAttRows, w.pairs) - 1);

  kv_f4 o[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) o[j] = kv_f4{0, 0, 0, 0};
  float m = kNoMax, l = 0.0f;

  const int from = split * a.part, to = (int)min((int64_t)from + a.part, (int64_t)end_last);
  for (int t0 = from + wave * kKvStrip; t0 < to; t0 += kKvStrip * kAttWaves) {
    const int64_t page = a.c.page(w.s, t0 >> a.c.page_shift);
    if (page < 0) continue;
    const uint8_t* base = a.c.head_page(page, h, head_bytes);
    Codes<D> k, v;
    load_keys<D>(base, T, t0 & (T - 1), k);
    load_vals<D>(base, T, t0 & (T - 1), v);

    float x[8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      uint4 y[D / 32];
      key_operand<D, BF16>(k, kt, y);
      kv_f4 sc{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < D / 32; ++j) sc = mfma<BF16>(y[j], q[j], sc);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * kt + i] = sc[i] * a.scale2;
    }
    const bool edge = t0 + kKvStrip > end_first || a.mask.p_dev != nullptr;
    if (edge) {
      const uint32_t in = seen_bits(a, w.s, h, t0, end);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (in >> i) & 1u ? x[i] : -__builtin_inff();
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
    if (__any(top > m + kSpan)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = top > m + kSpan ? top - kLift : m;
      const float f = __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int j = 0; j < kRun; ++j) o[j] *= f;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(x[i] - m);
      l += p[i];
    }
    const uint4 pb{pack_half(p[0], p[1]), pack_half(p[2], p[3]), pack_half(p[4], p[5]), pack_half(p[6], p[7])};
    float s[2][4];
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[half][i] = kv_scale((v.s[half] >> (8 * i)) & 0xffu);
    if (t0 + kKvStrip > w.len) {   // memory past the last token may hold anything: 0 times it must be 0
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + 16 * half + 4 * g + i >= w.len) {
            s[half][i] = 1.0f;
#pragma unroll
            for (int b = i * (D / 32); b < (i + 1) * (D / 32); ++b) v.w[half][b >> 2] &= ~(0xffu << (8 * (b & 3)));
          }
    }
    add_values<D, 0>(v, s, pb, o);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // the waves' parts: every wave's sums relative to the largest maximum
  __shared__ float sm[kAttWaves][kAttRows], sl[kAttWaves][kAttRows];
  __shared__ __align__(16) float so[kAttWaves][kAttRows][D + 4];
  if (g == 0) {
    sm[wave][c] = m;
    sl[wave][c] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < kRun; j += 4)
      *reinterpret_cast<kv_f4*>(&so[wave][c][(4 * g + i) * kRun + j]) =
          kv_f4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
  __syncthreads();
  const int col = threadIdx.x >> 4, run = threadIdx.x & 15;
  const int r = w.r0 + col;
  if (r >= w.pairs) return;
  float M = sm[0][col];
#pragma unroll
  for (int i = 1; i < kAttWaves; ++i) M = fmaxf(M, sm[i][col]);
  float f[kAttWaves], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kAttWaves; ++i) {
    f[i] = __builtin_amdgcn_exp2f(sm[i][col] - M);
    sum += f[i] * sl[i][col];
  }
  float acc[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    acc[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < kAttWaves; ++i) acc[j] += f[i] * so[i][col][run * kRun + j];
  }
  const int64_t at = (w.first + r / a.group) * a.q_heads + h * a.group + r % a.group;
  if (a.splits > 1) {
    const int64_t p = at * a.splits + split;
    if (run == 0) {
      a.part_m[p] = M;
      a.part_l[p] = sum;
    }
    float* d = a.part_o + p * D + run * kRun;
#pragma unroll
    for (int j = 0; j < kRun; j += 4) *reinterpret_cast<kv_f4*>(d + j) = kv_f4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
    return;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t* d = a.out + at * D + run * kRun;
#pragma unroll
  for (int j = 0; j < kRun; j += 4) {
    uint2 u;
    u.x = (uint32_t)to_out(acc[j] * inv, BF16) | ((uint32_t)to_out(acc[j + 1] * inv, BF16) << 16);
    u.y = (uint32_t)to_out(acc[j + 2] * inv, BF16) | ((uint32_t)to_out(acc[j + 3] * inv, BF16) << 16);
    *reinterpret_cast<uint2*>(d + j) = u;
  }
  if (run == 0) {
    const float e = sum == 0.0f ? -__builtin_inff() : M + __builtin_amdgcn_logf(sum);
    if (a.lse2) a.lse2[at] = e;
    if (a.lse) a.lse[at] = e * 0.6931471805599453f;
  }
}

// Joins the parts of the length: D/4 lanes per query row and head.
template <int D, bool BF16>
__global__ __launch_bounds__(kAttThreads) void k_kv_join(AttendArgs a) {
  constexpr int kLanes = D / 4;
  const int64_t at = (int64_t)blockIdx.x * (kAttThreads / kLanes) + threadIdx.x / kLanes;
  const int sub = threadIdx.x % kLanes;
  if (at >= a.c.rows * a.q_heads) return;
  if (a.c.starts && a.c.seq_of(at / a.q_heads) < 0) return;   // a row of no sequence: no part was written
  const float* pm = a.part_m + at * a.splits;
  const float* pl = a.part_l + at * a.splits;
  float M = kNoMax;
  for (int i = 0; i < a.splits; ++i) M = fmaxf(M, pm[i]);
  float sum = 0.0f;
  kv_f4 acc{0, 0, 0, 0};
  for (int i = 0; i < a.splits; ++i) {
    const float f = __builtin_amdgcn_exp2f(pm[i] - M);
    sum += f * pl[i];
    acc += f * *reinterpret_cast<const kv_f4*>(a.part_o + (at * a.splits + i) * D + 4 * sub);
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint2 u;
  u.x = (uint32_t)to_out(acc[0] * inv, BF16) | ((uint32_t)to_out(acc[1] * inv, BF16) << 16);
  u.y = (uint32_t)to_out(acc[2] * inv, BF16) | ((uint32_t)to_out(acc[3] * inv, BF16) << 16);
  *reinterpret_cast<uint2*>(a.out + at * D + 4 * sub) = u;
  if (sub == 0) {
    const float e = sum == 0.0f ? -__builtin_inff() : M + __builtin_amdgcn_logf(sum);
    if (a.lse2) a.lse2[at] = e;
    if (a.lse) a.lse[at] = e * 0.6931471805599453f;
  }
}

// Accumulated weights: a wave owns 32 tokens of one head, whose keys it converts
// once, and walks the call's rows; p = 2^(s - lse).  Every token is summed by one
// wave in the order of the rows, so the result does not depend on timing.
template <int D, bool BF16>
__global__ __launch_bounds__(kAttThreads) void k_kv_weights(AttendArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  int64_t id = blockIdx.x;
  const int64_t chunks = (a.cut + kKvStrip * kAttWaves - 1) / (kKvStrip * kAttWaves);
  const int t0 = (int)(id % chunks) * (kKvStrip * kAttWaves) + wave * kKvStrip;
  id /= chunks;
  const int h = (int)(id % a.c.heads);
  TileRows w;
  w.s = (int)(id / a.c.heads);
  w.first = a.c.start(w.s);
  w.n = (int)max((int64_t)0, a.c.start(w.s + 1) - w.first);
  w.pairs = w.n * a.group;
  w.end_full = a.c.length(w.s);
  w.len = (int)min((int64_t)w.end_full, a.cut);
  if (t0 >= w.len || w.pairs == 0) return;
  const int T = 1 << a.c.page_shift;
  const int64_t page = a.c.page(w.s, t0 >> a.c.page_shift);
  if (page < 0) return;
  Codes<D> k;
  load_keys<D>(a.c.head_page(page, h, KvLayout<D>::head_bytes(T)), T, t0 & (T - 1), k);
  uint4 y[2][D / 32];
  key_operand<D, BF16>(k, 0, y[0]);
  key_operand<D, BF16>(k, 1, y[1]);
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  // with a causal limit the first row that sees token t0 is row t0 - (end_full - n)
  int r0 = a.causal ? max(0, t0 - (w.end_full - w.n)) * a.group / kAttRows * kAttRows : 0;
  for (; r0 < w.pairs; r0 += kAttRows) {
    uint4 q[D / 32];
    load_q<D>(a, w, h, r0, q);
    const int r = r0 + c, rr = min(r, w.pairs - 1);
    const float e = a.lse2[(w.first + rr / a.group) * a.q_heads + h * a.group + rr % a.group];
    const int end = pair_end(a, w, rr);
    const uint32_t in = r < w.pairs && e > -__builtin_inff() ? seen_bits(a, w.s, h, t0, end) : 0u;
    const uint32_t nan = r < w.pairs && e != e ? 0xffu : 0u;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      kv_f4 sc{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < D / 32; ++j) sc = mfma<BF16>(y[kt][j], q[j], sc);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sum[4 * kt + i] += ((in | nan) >> (4 * kt + i)) & 1u ? __builtin_amdgcn_exp2f(sc[i] * a.scale2 - e) : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) sum[i] += __shfl_xor(sum[i], d);
    const int t = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
    if (c == 0 && t < w.len && t < a.weights.cols)
      static_cast<float*>(a.weights.p_dev)[w.s * a.weights.seq_stride + h * a.weights.head_stride + t] += sum[i];
  }
}

}  // namespace

#define LAM_KV_DISPATCH(v, LAUNCH)                                   \
  do {                                                               \
    const bool bf_ = (v).dtype == LAM_BF16;                          \
    if ((v).head_dim == 64) { if (bf_) LAUNCH(64, true); else LAUNCH(64, false); }           \
    else if ((v).head_dim == 128) { if (bf_) LAUNCH(128, true); else LAUNCH(128, false); }   \
    else { if (bf_) LAUNCH(256, true); else LAUNCH(256, false); }    \
  } while (0)

lam_status launch_kv_attend(lam_ctx* ctx, const lam_kv_view& v, const void* q, int64_t q_row, int64_t q_head,
                            int32_t q_heads, float scale, bool causal, int64_t max_length, const lam_kv_slots& mask,
                            const lam_kv_slots& weights, void* out, float* lse) {
  AttendArgs a{};
  a.c = KvArgs::of(v);
  a.q = static_cast<const uint16_t*>(q);
  a.q_row = q_row;
  a.q_head = q_head;
  a.q_wide = (reinterpret_cast<uintptr_t>(q) & 15) == 0 && q_row % 8 == 0 && q_head % 8 == 0;
  a.q_heads = q_heads;
  a.group = q_heads / v.kv_heads;
  a.causal = causal;
  a.scale2 = (float)((double)scale * 1.4426950408889634);
  a.cut = (int64_t)v.table_cols * v.page_size;
  if (max_length > 0) a.cut = std::min(a.cut, max_length);
  a.mask = mask;
  a.weights = weights;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;

  int64_t tiles;
  if (v.starts_dev) {
    tiles = v.rows * a.group / kAttRows + v.n_seqs;
  } else {
    a.tiles_per_seq = (int)((v.rows / v.n_seqs * a.group + kAttRows - 1) / kAttRows);
    tiles = (int64_t)a.tiles_per_seq * v.n_seqs;
  }
  // parts of the length: enough workgroups for four on every compute unit, none
  // with less than a strip for each wave
  const int64_t units = tiles * v.kv_heads;
  const int64_t strips = std::max<int64_t>(1, (a.cut + kKvStrip * kAttWaves - 1) / (kKvStrip * kAttWaves));
  const int64_t want = std::min<int64_t>(strips, std::max<int64_t>(1, 1024 / units));
  const int64_t per = (strips + want - 1) / want;
  a.part = (int)(per * kKvStrip * kAttWaves);
  a.splits = (int)((strips + per - 1) / per);

  const int64_t pairs = v.rows * q_heads;
  const int64_t parts = a.splits > 1 ? pairs * a.splits : 0;
  DevBuf& buf = ctx->scratch[kScratchKv];
  LAM_TRY(buf.ensure((size_t)(parts * (v.head_dim + 2) + (weights.p_dev ? pairs : 0)) * 4));
  a.part_o = buf.as<float>();
  a.part_m = a.part_o + parts * v.head_dim;
  a.part_l = a.part_m + parts;
  if (weights.p_dev) a.lse2 = a.part_l + parts;

  const int64_t blocks = units * a.splits;
  LAM_CHECK(blocks < (1LL << 31), LAM_EINVAL, "too many rows for one launch");
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_attend", &e0, &e1));
#define LAM_GO(D, BF) \
  hipExtLaunchKernelGGL((k_kv_attend<D, BF>), dim3((unsigned)blocks), dim3(kAttThreads), 0, ctx->stream, e0, e1, 0, a)
  LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  if (a.splits > 1) {
    const int64_t per_block = kAttThreads / (v.head_dim / 4);
    const int64_t jb = (pairs + per_block - 1) / per_block;
    LAM_TRY(prof_launch_events(ctx, "kv_join", &e0, &e1));
#define LAM_GO(D, BF) \
  hipExtLaunchKernelGGL((k_kv_join<D, BF>), dim3((unsigned)jb), dim3(kAttThreads), 0, ctx->stream, e0, e1, 0, a)
    LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
    LAM_HIP(hipGetLastError());
  }
  if (weights.p_dev && a.cut > 0) {
    const int64_t wb = strips * v.kv_heads * v.n_seqs;
    LAM_CHECK(wb < (1LL << 31), LAM_EINVAL, "too many sequences for one launch");
    LAM_TRY(prof_launch_events(ctx, "kv_weights", &e0, &e1));
#define LAM_GO(D, BF) \
  hipExtLaunchKernelGGL((k_kv_weights<D, BF>), dim3((unsigned)wb), dim3(kAttThreads), 0, ctx->stream, e0, e1, 0, a)
    LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
    LAM_HIP(hipGetLastError());
  }
  return LAM_OK;
}

}  // namespace lam
