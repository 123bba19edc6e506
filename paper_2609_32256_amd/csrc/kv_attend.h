// What the kernels of attention over the 4-bit cache share: the call's arguments,
// how it is cut into workgroups, a strip's codes on their way from memory, and the
// matrix operands made of them.
#pragma once

#include <hip/hip_runtime.h>

#include "kv.h"
#include "lam_internal.h"
#include "wave.h"

namespace lam {

constexpr int kAttThreads = 256;
constexpr int kAttWaves = kAttThreads / 64;
constexpr int kAttRows = 16;        // rows of a tile of the kernel for single tokens

// The reference of a row's exponentials is at least its maximum so far less
// 2^kSpan and at most 2^-kLift of it when it was set: the weights reach 2^15,
// within float16, and those 2^-21 below the maximum are still normal numbers.
constexpr float kLift = 7.0f, kSpan = 15.0f;
constexpr float kNoMax = -3.0e38f;   // no token seen yet
// Workgroups (of four waves) that run at once: three a compute unit for single tokens,
// two for chunks, one where heads have 256 channels (by registers).  Lengths are split
// over as many where the tiles are fewer.  (Over twice as many: chunks of 2,400 to 8,192
// pairs 8 to 30 % slower, since the sums written for the join outweigh the evener
// parts; 800 to 1,500 tiles of single tokens split as well: 5 to 35 % slower but
// for a gain of 3 % at 800; 256 channels over 768 workgroups: 6 to 30 % slower than 256.)
constexpr int kFillDecode = 768, kFillChunk = 512, kFillWide = 256;
// No length up to these is split, since the launch that joins the parts takes as long as
// their walk: 1,400 tokens of single tokens of 1 to 64 sequences take 11 to 20 us whole
// and 18 to 25 split, 3,000 tokens 18 to 19 whole and 14 to 18 split; chunks at 600
// tokens 15 to 19 whole and 19 to 41 split, at 1,500 27 whole and 23 split.
constexpr int kWholeDecode = 2048, kWholeChunk = 1024;
// Least tokens of a part, whose results are written and read again: with 128 for single
// tokens 24,066 tokens of one head and 8 rows took 17.6 us for 12.5, 20,000 of four heads 20.9 for
// 14.2.  A chunk's part is of as many tokens or a multiple (its sums are 64 rows).
constexpr int kLeastDecode = 512, kLeastChunk = 512;
// The kernel for chunks is taken where sequences have more (row, head) pairs than
// this on average.  64 pairs over 10,000 tokens of 4 sequences and 8 heads of 128
// channels: 34 us by 16 rows, 37 by 64; 96 pairs over 4,096 tokens of 20: 66 and 87 without
// weights, but 109 and 96 with weights over 10,000 tokens of 4.
constexpr int kChunkPairs = 64;
constexpr int64_t kKeptBytes = 1LL << 30;   // most scratch for kept scores

struct AttendArgs {
  KvArgs c;
  const uint16_t* q;
  int64_t q_row, q_head;
  int q_wide;             // every eight channels of q are a 16-byte load
  int q_heads, group;
  int causal;
  float scale2;           // |scale| * log2(e), above 0
  int flip;               // the scale is negative
  int64_t cut;            // lengths are cut to it: the table's columns and the caller's bound
  int tiles_per_seq;      // where every sequence has the same number of rows
  int join_rows;          // rows a wave joins, 1 or 4
  int kept_waves;         // waves that share a token's kept scores, 1 or 4
  int split_to;           // workgroups to split the lengths over, 0: none is split
  int64_t blocks;         // workgroups of the attention: places for partial results
  lam_kv_slots mask, weights;
  uint16_t* out;
  float* lse;             // natural logarithm, the caller's
  float* lse2;            // base 2, for the weights
  float* kept;            // scores of every row's tokens, base 2: [row * q_heads + head][kept_cols], or null
  int64_t kept_cols;
  float* part_m;          // of workgroup b's row r of its tile: [b][rows of a tile]
  float* part_l;
  float* part_o;          // [b][rows of a tile][D]
};

// What a workgroup does: a part of the length for a tile of R (row, head of the
// group) pairs of a sequence and a key/value head.
struct Work {
  int s;               // sequence, -1: nothing to do
  int64_t first;       // its first row of the call
  int n;               // its rows
  int pairs;           // its pairs, row-major
  int len, end_full;   // cached tokens: those with a column of the table, cut to the bound; and all
  int parts, tokens;   // parts of its length, and the tokens of one
  uint32_t base;       // its first workgroup
  int h, r0, part;     // head, first pair of the tile, part
};

__device__ __forceinline__ int tiles_of(int pairs, int R) { return (pairs + R - 1) / R; }

// A lane's sequence: its rows, tiles and length.
struct LaneSeq {
  int64_t first;
  int n, tiles, full, len;
  __device__ __forceinline__ LaneSeq(const AttendArgs& a, int s, int R) {
    const bool in = s < a.c.n_seqs;
    const int q = min(s, a.c.n_seqs - 1);
    first = a.c.start(q);
    n = in ? (int)max((int64_t)0, a.c.start(q + 1) - first) : 0;
    full = a.c.tokens(q);
    len = (int)min((int64_t)full, a.cut);
    tiles = tiles_of(n * a.group, R);
  }
};

// The workgroups of a call whose lengths are split: every sequence's length is cut
// into parts of the same number of tokens, chosen from the lengths on the
// device so that about split_to workgroups with equal parts cover them all
// (equal parts of the longest length had left a ragged batch's short sequences
// with empty ones).  The last part of a tile is half full on average, so the parts are for
// split_to less half the tiles.  All lanes of a wave look at a sequence each.
// id: a workgroup; or a sequence, or a unit (a tile of a head), whose plan is wanted.
enum class PlanOf { kWorkgroup, kSequence, kUnit };

template <int R, PlanOf OF>
__device__ __forceinline__ Work plan(const AttendArgs& a, uint32_t id) {
  const int lane = threadIdx.x & 63;
  double tokens = 0.0, units = 0.0;
  LaneSeq q(a, lane, R);
  for (int b = 0;;) {
    tokens += (double)q.tiles * q.len;
    units += (double)q.tiles;
    b += 64;
    if (b >= a.c.n_seqs) break;
    q = LaneSeq(a, b + lane, R);
  }
  if (a.c.n_seqs > 64) q = LaneSeq(a, lane, R);
  const float all = (float)wave_sum_f64(tokens) * a.c.heads, half = 0.5f * (float)wave_sum_f64(units) * a.c.heads;
  constexpr int kStrips = kKvStrip * kAttWaves, kGrain = R == kAttRows ? kStrips : kLeastChunk;
  constexpr int kLeast = R == kAttRows ? kLeastDecode : kLeastChunk;
  const float want = all / fmaxf((float)a.split_to - half, 0.5f * a.split_to) * 1.0001f;
  Work w;
  w.s = -1;
  w.tokens = (int)fminf(fmaxf(floorf(want / kGrain) * kGrain + kGrain, (float)kLeast), 2147483520.0f);
  uint32_t before = 0, units_before = 0;
  for (int b = 0; b < a.c.n_seqs; b += 64) {
    if (b > 0) q = LaneSeq(a, b + lane, R);
    const int parts = max(1, (q.len + w.tokens - 1) / w.tokens);
    const int even = ((q.len + parts - 1) / parts + kStrips - 1) / kStrips * kStrips;   // its parts made equal
    const uint32_t my_units = (uint32_t)(q.tiles * a.c.heads), mine = my_units * parts;
    const uint32_t upto = wave_scan_u32(mine) + before;
    unsigned long long hit;
    uint32_t units_upto = 0;
    if constexpr (OF == PlanOf::kWorkgroup) {
      hit = __ballot(upto > id);
    } else if constexpr (OF == PlanOf::kSequence) {
      hit = (uint32_t)b <= id && id < (uint32_t)b + 64u ? 1ull << (id - b) : 0ull;
    } else {
      units_upto = wave_scan_u32(my_units) + units_before;
      hit = __ballot(units_upto > id);
    }
    if (hit) {
      const int l = (int)__builtin_ctzll(hit);
      w.s = b + l;
      w.first = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)q.first, l);
      w.n = __builtin_amdgcn_readlane(q.n, l);
      w.len = __builtin_amdgcn_readlane(q.len, l);
      w.end_full = __builtin_amdgcn_readlane(q.full, l);
      w.parts = __builtin_amdgcn_readlane(parts, l);
      w.tokens = __builtin_amdgcn_readlane(even, l);
      w.base = (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), l);
      w.pairs = w.n * a.group;
      if constexpr (OF != PlanOf::kSequence) {
        uint32_t unit = id - (uint32_t)__builtin_amdgcn_readlane((int)(units_upto - my_units), l);
        w.part = 0;
        if constexpr (OF == PlanOf::kWorkgroup) {
          const uint32_t in = id - w.base;
          unit = in / (uint32_t)w.parts;
          w.part = (int)(in % (uint32_t)w.parts);
        } else {
          w.base += unit * w.parts;   // the unit's own first workgroup
        }
        w.h = (int)(unit % (uint32_t)a.c.heads);
        w.r0 = (int)(unit / (uint32_t)a.c.heads) * R;
      }
      break;
    }
    before = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    if constexpr (OF == PlanOf::kUnit) units_before = (uint32_t)__builtin_amdgcn_readlane((int)units_upto, 63);
  }
  return w;
}

// The workgroup's work where no length is split: heads innermost, then tiles.
template <int R>
__device__ __forceinline__ Work tile_work(const AttendArgs& a, uint32_t id) {
  Work w;
  w.h = (int)(id % (uint32_t)a.c.heads);
  w.part = 0;
  w.parts = 1;
  w.tokens = 0x7fffffff;
  w.base = 0;
  const uint32_t t = id / (uint32_t)a.c.heads;
  int64_t next;
  if (!a.c.starts) {
    const uint32_t per = (uint32_t)a.tiles_per_seq;
    w.s = (int)(t / per);
    w.r0 = (int)(t % per) * R;
    w.first = (int64_t)w.s * a.c.per_seq;
    next = w.first + a.c.per_seq;
    w.end_full = a.c.tokens(w.s);
  } else {
    // Sequence s has its tiles from floor(start(s) * group / R) + s on, a bound that
    // leaves room for every partial tile and rises with s: the last s whose bound
    // is at most t is found by all lanes at once, 64 sequences a step, each lane
    // with its sequence's rows and length in hand (a search by halves had cost a
    // round trip to memory for each step).
    const int lane = threadIdx.x & 63;
    w.s = 0;
    w.r0 = -1;
    w.first = next = 0;
    w.end_full = 0;
    for (int b = 0; b < a.c.n_seqs; b += 64) {
      const int s = min(b + lane, a.c.n_seqs - 1);
      const int64_t s0 = a.c.start(s), s1 = a.c.start(s + 1);
      const int l = a.c.tokens(s);
      const uint32_t at = (uint32_t)(s0 * a.group / R) + (uint32_t)s;
      const unsigned long long in = __ballot(b + lane < a.c.n_seqs && at <= t);
      if (in == 0) break;
      const int last = (int)__popcll(in) - 1;
      w.s = b + last;
      w.first = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)s0, last);
      next = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)s1, last);
      w.end_full = __builtin_amdgcn_readlane(l, last);
      w.r0 = (int)min((t - (uint32_t)__builtin_amdgcn_readlane((int)at, last)) * (uint32_t)R, 0x7fffff00u);
      if (last < 63) break;
    }
  }
  w.n = (int)max((int64_t)0, next - w.first);
  w.pairs = w.n * a.group;
  w.len = (int)min((int64_t)w.end_full, a.cut);
  if (w.r0 < 0 || w.r0 >= w.pairs) w.s = -1;
  return w;
}

template <int R>
__device__ __forceinline__ Work work_of(const AttendArgs& a, uint32_t id) {
  return a.split_to ? plan<R, PlanOf::kWorkgroup>(a, id) : tile_work<R>(a, id);
}

// Rows of no sequence see no token: 0, and a log sum of -inf.  (A workgroup's last work:
// as its first it cost 0.2 us of 26 and registers.)
template <int D>
__device__ __forceinline__ void clear_rows(const AttendArgs& a) {
  if (!a.c.starts) return;
  const int64_t rows = a.c.rows;
  auto clipped = [&](int s) { return min(max((int64_t)kv_const(a.c.starts)[s], (int64_t)0), rows); };
  const int64_t before = clipped(0), after = clipped(a.c.n_seqs), row_size = (int64_t)a.q_heads * (D / 8);
  for (int64_t r = blockIdx.x; r < before + rows - after; r += gridDim.x) {
    const int64_t row = r < before ? r : after + r - before;
    for (int64_t i = threadIdx.x; i < row_size; i += kAttThreads)
      *reinterpret_cast<uint4*>(a.out + (row * row_size + i) * 8) = uint4{0, 0, 0, 0};
    if (a.lse)
      for (int j = threadIdx.x; j < a.q_heads; j += kAttThreads) a.lse[row * a.q_heads + j] = -__builtin_inff();
  }
}

// Tokens that pair r of the sequence sees: those below this.
__device__ __forceinline__ int pair_end(const AttendArgs& a, const Work& w, int r) {
  if (!a.causal) return w.len;
  return max(0, min(w.len, w.end_full - w.n + r / a.group + 1));
}

// B operand of a query row and head: lane (c, g) holds channels g D/4 + 8 j + 0..7
// of column c as step j.  p: where its channels begin.
template <int D>
__device__ __forceinline__ void load_row(const uint16_t* p, bool wide, uint4 q[D / 32]) {
  if (wide) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) q[j] = *reinterpret_cast<const uint4*>(p + 8 * j);
  } else {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (uint32_t)p[8 * j + 2 * i] | ((uint32_t)p[8 * j + 2 * i + 1] << 16);
      q[j] = uint4{x[0], x[1], x[2], x[3]};
    }
  }
}

// A negative scale: scale2 is its size, the queries (or the keys) take its sign.
template <int N>
__device__ __forceinline__ void flip_signs(uint4 x[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j)
    x[j] = uint4{x[j].x ^ 0x80008000u, x[j].y ^ 0x80008000u, x[j].z ^ 0x80008000u, x[j].w ^ 0x80008000u};
}

// The 16 pairs from r0 on.  Columns past the last pair repeat it; nothing of theirs
// is written.
template <int D>
__device__ __forceinline__ void load_q(const AttendArgs& a, const Work& w, int h, int r0, uint4 q[D / 32]) {
  const int r = min(r0 + (int)(threadIdx.x & 15), w.pairs - 1);
  const int g = (threadIdx.x & 63) >> 4;
  load_row<D>(a.q + (w.first + r / a.group) * a.q_row + (int64_t)(h * a.group + r % a.group) * a.q_head + g * (D / 4),
              a.q_wide, q);
  if (a.flip) flip_signs<D / 32>(q);
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

// Loads of a strip go through a buffer resource over its head's part of the page:
// one of no bytes stands for a strip past the end or a page outside the pool and
// reads as zeros without touching memory, so no load hangs on a branch and the
// compiler can count those in flight.  Codes are read once and marked so
// (non-temporal: 199 -> 173 us for eight sequences of 131,072 tokens, 6.6 TB/s).
constexpr int kNonTemporal = 2;

// The codes and the scales of a strip at token t of a page: resources whose base
// is the strip's, so that what a lane adds is constant.
struct StripRsrc {
  __amdgpu_buffer_rsrc_t codes, scales;
};

template <int D>
__device__ __forceinline__ StripRsrc strip_rsrc(uint8_t* head, int T, int t, bool ok) {
  const int bytes = ok ? (int)KvLayout<D>::head_bytes(T) : 0;
  return StripRsrc{__builtin_amdgcn_make_buffer_rsrc(head + t * (D / 2), (short)0, bytes, 0x00020000),
                   __builtin_amdgcn_make_buffer_rsrc(head + T * D + t * (D / 32), (short)0, bytes, 0x00020000)};
}

template <int D>
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t rs, uint32_t at, uint32_t w[D / 32]) {
  if constexpr (D == 64) {
    const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, kNonTemporal));
    w[0] = u.x, w[1] = u.y;
  } else {
#pragma unroll
    for (int j = 0; j < D / 128; ++j) {
      const uint4 u = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, at + 16 * j, 0, kNonTemporal));
      w[4 * j] = u.x, w[4 * j + 1] = u.y, w[4 * j + 2] = u.z, w[4 * j + 3] = u.w;
    }
  }
}

// Where a lane's codes and scales lie from a strip's bases on.
template <int D>
struct LaneAt {
  uint32_t k, ks, shift, v, vs;
  __device__ __forceinline__ explicit LaneAt(int T) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    k = c * (D / 2) + g * (D / 8);
    // the word that holds the lane's scale bytes, and their place in it
    const int b = c * (D / 32) + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g);
    ks = b & ~3;
    shift = (b & 3) * 8;
    v = T * (D / 2) + (g * 16 + c) * (D / 8);
    vs = T * (D / 32) + (g * (D / 32) + c * (D / 16) / kKvBlock) * 4;
  }
};

// Keys: tile kt of a strip, token 16 kt + c, the lane's quarter of the channels.
template <int D>
__device__ __forceinline__ void load_keys(const StripRsrc& rs, const LaneAt<D>& at, Codes<D>& k) {
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    load_words<D>(rs.codes, at.k + 16 * kt * (D / 2), k.w[kt]);
    k.s[kt] = __builtin_amdgcn_raw_buffer_load_b32(rs.scales, at.ks + 16 * kt * (D / 32), 0, 0);
  }
}

// Values: half `half` of a strip, tokens 16 half + 4 g + 0..3, run c of the channels.
template <int D>
__device__ __forceinline__ void load_vals(const StripRsrc& rs, const LaneAt<D>& at, Codes<D>& v) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    load_words<D>(rs.codes, at.v + 16 * half * (D / 2), v.w[half]);
    v.s[half] = __builtin_amdgcn_raw_buffer_load_b32(rs.scales, at.vs + 16 * half * (D / 32), 0, 0);
  }
}

// A operands of a strip's keys times the queries: scores of tokens 16 kt + 4 g + i.
template <int D, bool BF16>
__device__ __forceinline__ void key_operand(const Codes<D>& k, uint32_t shift, int kt, uint4 x[D / 32]) {
  const uint32_t bytes = k.s[kt] >> shift;
#pragma unroll
  for (int j = 0; j < D / 32; ++j)
    x[j] = kv_values8<BF16>(k.w[kt][j], kv_scale((D == 256 && j >= 4 ? bytes >> 8 : bytes) & 0xffu));
}

// Two values of token TOK (of four) of a half's codes: channels 2 JP and 2 JP + 1 of the run.
template <int D, int TOK, int JP>
__device__ __forceinline__ uint32_t val_pair(const uint32_t w[D / 32], float s) {
  constexpr int byte = TOK * (D / 32) + JP;
  return kv_values<false, byte % 4>(w[byte / 4], s);
}

// O^T += V^T P^T of a strip for TILES tiles of queries: one product per channel of
// the lane's run and tile.
template <int D, int TILES, int JP>
__device__ __forceinline__ void add_values(const Codes<D>& v, const float s[2][4], const uint4 p[TILES],
                                           kv_f4 o[TILES][D / 16]) {
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
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      o[t][2 * JP] = mfma<false>(even, p[t], o[t][2 * JP]);
      o[t][2 * JP + 1] = mfma<false>(odd, p[t], o[t][2 * JP + 1]);
    }
    add_values<D, TILES, JP + 1>(v, s, p, o);
  }
}

// Mask of a strip's tokens: lane l reads token t0 + l % 32's byte.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mask_rsrc(const AttendArgs& a, int s, int h) {
  const uint8_t* p = static_cast<const uint8_t*>(a.mask.p_dev) + s * a.mask.seq_stride + h * a.mask.head_stride;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, a.mask.cols, 0x00020000);
}

__device__ __forceinline__ uint32_t load_mask(__amdgpu_buffer_rsrc_t rs, int t0) {
  return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rs, t0 + (threadIdx.x & 31), 0, 0);
}

// A strip's tokens as bits, from the lanes' mask bytes.  Strips of which the mask leaves
// nothing are passed over, and where it leaves all, the scores are not looked through
// (a chunk of 239 rows of 64 heads over 7,392 tokens, a quarter of the records of 16 tokens
// masked: 177 us for 119).
constexpr uint32_t kAllTokens = 0xffffffffu;
template <bool MASK>
__device__ __forceinline__ uint32_t mask_bits(uint32_t mask_byte) {
  return MASK ? (uint32_t)__ballot(mask_byte != 0) : kAllTokens;
}

// Which of a strip's tokens the lane's query sees: bit 4 half + i for token t0 + 16 half + 4 g + i.
__device__ __forceinline__ uint32_t seen_bits(uint32_t all, int t0, int end) {
  const int g = (threadIdx.x & 63) >> 4;
  const int n = min(max(end - t0, 0), 32);
  const uint32_t in = (all & (n == 32 ? 0xffffffffu : (1u << n) - 1u)) >> (4 * g);
  return (in & 0xfu) | ((in >> 12) & 0xf0u);
}

// The scales of the lane's eight tokens of a strip at t0.  Memory past the last
// token, or of a token that the mask takes out (bits), may hold anything, and 0 times it
// must be 0: its codes become 0.
template <int D>
__device__ __forceinline__ void value_scales(Codes<D>& v, int t0, int len, uint32_t bits, float s[2][4]) {
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[half][i] = kv_scale((v.s[half] >> (8 * i)) & 0xffu);
  if (t0 + kKvStrip > len || bits != kAllTokens) {
    const uint32_t in = seen_bits(bits, t0, len);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!((in >> (4 * half + i)) & 1u)) {
          s[half][i] = 1.0f;
#pragma unroll
          for (int b = i * (D / 32); b < (i + 1) * (D / 32); ++b) v.w[half][b >> 2] &= ~(0xffu << (8 * (b & 3)));
        }
  }
}

// The softmax of a lane's query over the strips so far.  Four lanes (g) share a
// query: m and seen are the same in them, l counts each lane's own tokens.
struct Row {
  float m = 0.0f;      // reference of the exponentials, base 2
  float l = 0.0f;
  bool seen = false;   // m is a score's

  // top: the largest score of a strip less m
  __device__ __forceinline__ bool rises(float top) const { return top > kSpan || (!seen && top > -__builtin_inff()); }

  // A new reference for the rows that need one; x becomes relative to it.  The
  // factor for what was summed relative to the old one.
  __device__ __forceinline__ float raise(float top, kv_f4 x[2]) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float by = rises(top) ? top - kLift : 0.0f;
    x[0] -= by;
    x[1] -= by;
    m += by;
    const float f = seen ? __builtin_amdgcn_exp2f(-by) : 0.0f;   // (nothing summed yet: by may be anything)
    seen = seen || top > -__builtin_inff();
    l *= f;
    return f;
  }

  // 2^x of the strip as the B operand of the values' product.  There they are
  // float16: 11 bits of each, an error that averages out below the result's own
  // rounding (bfloat16) or about at it (float16).  Their sum keeps them in float32,
  // since the log sums and the accumulated weights come from it.
  __device__ __forceinline__ uint4 weights(const kv_f4 x[2]) {
    uint32_t p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = __builtin_amdgcn_exp2f(x[i >> 1][2 * (i & 1)]), b = __builtin_amdgcn_exp2f(x[i >> 1][2 * (i & 1) + 1]);
      const kv_h2 h{(_Float16)a, (_Float16)b};
      l += a;
      l += b;
      p[i] = __builtin_bit_cast(uint32_t, h);
    }
    return uint4{p[0], p[1], p[2], p[3]};
  }

  __device__ __forceinline__ float sum() const {
    const float s = l + __shfl_xor(l, 16);
    return s + __shfl_xor(s, 32);
  }
  __device__ __forceinline__ float reference() const { return seen ? m : kNoMax; }
};

__device__ __forceinline__ void less_reference(kv_f4 x[2], float scale2, const Row& r) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i >> 2][i & 3] = __builtin_fmaf(x[i >> 2][i & 3], scale2, -r.m);
}

__device__ __forceinline__ void hide(kv_f4 x[2], uint32_t seen) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i >> 2][i & 3] = (seen >> i) & 1u ? x[i >> 2][i & 3] : -__builtin_inff();
}

__device__ __forceinline__ float top_of(const kv_f4 x[2]) {
  float z = fmaxf(x[0][0], x[1][0]);
#pragma unroll
  for (int i = 1; i < 4; ++i) z = fmaxf(fmaxf(z, x[0][i]), x[1][i]);
  return z;
}

__device__ __forceinline__ uint16_t to_out(float x, bool bf16) {
  if (bf16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  return __builtin_bit_cast(uint16_t, (_Float16)x);
}

__device__ __forceinline__ float log_sum(float M, float sum) {
  return sum == 0.0f ? -__builtin_inff() : M + __builtin_amdgcn_logf(sum);
}

// A lane's channels of a finished row, and the row's log sums.
template <int D, bool BF16>
__device__ __forceinline__ void write_row(const AttendArgs& a, int64_t row, int run, const float acc[D / 16], float M,
                                          float sum) {
  constexpr int kRun = D / 16;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t* d = a.out + row * D + run * kRun;
#pragma unroll
  for (int j = 0; j < kRun; j += 4) {
    uint2 u;
    u.x = (uint32_t)to_out(acc[j] * inv, BF16) | ((uint32_t)to_out(acc[j + 1] * inv, BF16) << 16);
    u.y = (uint32_t)to_out(acc[j + 2] * inv, BF16) | ((uint32_t)to_out(acc[j + 3] * inv, BF16) << 16);
    *reinterpret_cast<uint2*>(d + j) = u;
  }
  if (run == 0) {
    const float e = log_sum(M, sum);
    if (a.lse2) a.lse2[row] = e;
    if (a.lse) a.lse[row] = e * 0.6931471805599453f;
  }
}

// Where the waves of a workgroup put their sums of 16 rows to be joined.
template <int D>
struct JoinSpace {
  float m[kAttWaves][kAttRows], l[kAttWaves][kAttRows];
  __align__(16) float o[kAttWaves][kAttRows][D + 4];
};

// Joins the waves' sums of the 16 rows from r0 on, relative to the largest
// maximum; 16 lanes a row write them out, or as the part's.  slot: where the
// first row's partial results go.
template <int D, bool BF16>
__device__ __forceinline__ void join_waves(const AttendArgs& a, const Work& w, int r0, int64_t slot, const Row& row,
                                           const kv_f4 o[D / 16], JoinSpace<D>& js) {
  constexpr int kRun = D / 16;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
  const float m = row.reference(), l = row.sum();
  if (g == 0) {
    js.m[wave][c] = m;
    js.l[wave][c] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < kRun; j += 4)
      *reinterpret_cast<kv_f4*>(&js.o[wave][c][(4 * g + i) * kRun + j]) =
          kv_f4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
  __syncthreads();
  const int col = threadIdx.x >> 4, run = threadIdx.x & 15;
  const int pair = r0 + col;
  if (pair >= w.pairs) return;
  float M = js.m[0][col];
#pragma unroll
  for (int i = 1; i < kAttWaves; ++i) M = fmaxf(M, js.m[i][col]);
  float f[kAttWaves], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kAttWaves; ++i) {
    f[i] = __builtin_amdgcn_exp2f(js.m[i][col] - M);
    sum += f[i] * js.l[i][col];
  }
  float acc[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    acc[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < kAttWaves; ++i) acc[j] += f[i] * js.o[i][col][run * kRun + j];
  }
  if (w.parts > 1) {
    if (run == 0) {
      a.part_m[slot + col] = M;
      a.part_l[slot + col] = sum;
    }
    float* d = a.part_o + (slot + col) * D + run * kRun;
#pragma unroll
    for (int j = 0; j < kRun; j += 4) *reinterpret_cast<kv_f4*>(d + j) = kv_f4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
  } else {
    const int64_t at = (w.first + pair / a.group) * a.q_heads + w.h * a.group + pair % a.group;
    write_row<D, BF16>(a, at, run, acc, M, sum);
  }
}

// Rows of a tile of the kernel for chunks (kv_chunk.hip): 64, or 32 and 48 of 256
// channels, and its launch.
constexpr int kChunkRows = 64, kChunkRowsWide = 32, kChunkRowsWider = 48;
lam_status launch_kv_chunk(lam_ctx* ctx, const lam_kv_view& v, const AttendArgs& a, int rows, int64_t blocks, bool masked);

}  // namespace lam
