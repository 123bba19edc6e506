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
//
// Bound by reading the cache once: 8 sequences of 131,072 tokens, 32 query heads over 8
// key/value heads of 128 channels, bfloat16, take 172 us, 6.6 TB/s; 37 sequences of 3,000
// to 6,000 and 28 over 4 heads 20 to 22 us, 4.3 TB/s, of which 5 are the start and the plan.
// Sixteen rows fill the products' columns where four or seven are there: the matrix
// units have the time.  Lengths are split where the tiles are fewer than the workgroups
// that run at once, and joined by a second launch (5 us; a join by the last workgroup of each
// unit took 2 to 30 us more, since its parts have to leave the caches of the XCDs).
#include <algorithm>
#include <cmath>

#include "kv_attend.h"

namespace lam {
namespace {

// A strip of a page outside the pool, or all masked: no scores.
__device__ __forceinline__ void keep_nothing(float* scores) {
  const int g = (threadIdx.x & 63) >> 4;
  const float no = -__builtin_inff();
  *reinterpret_cast<kv_f4*>(scores + 4 * g) = kv_f4{no, no, no, no};
  *reinterpret_cast<kv_f4*>(scores + 4 * g + 16) = kv_f4{no, no, no, no};
}

// The running softmax of 16 query rows over the strips a wave takes.
template <int D, bool BF16, bool MASK>
struct Running {
  static constexpr int kRun = D / 16;
  kv_f4 o[kRun];
  Row row;

  __device__ __forceinline__ Running() {
#pragma unroll
    for (int j = 0; j < kRun; ++j) o[j] = kv_f4{0, 0, 0, 0};
  }

  // One strip at t0; whole: every query sees all of its tokens.  scores: where
  // the query's scores are kept (null: nowhere), slot by slot.
  __device__ __forceinline__ void add(const AttendArgs& a, int len, int t0, bool whole, int end, uint32_t bits,
                                      float* scores, uint32_t shift, const uint4 q[D / 32], const Codes<D>& k,
                                      Codes<D>& v) {
    kv_f4 x[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      uint4 y[D / 32];
      key_operand<D, BF16>(k, shift, kt, y);
      x[kt] = kv_f4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < D / 32; ++j) x[kt] = mfma<BF16>(y[j], q[j], x[kt]);
    }
    less_reference(x, a.scale2, row);
    if (!whole) hide(x, seen_bits(bits, t0, end));
    if (scores) {
      const int g = (threadIdx.x & 63) >> 4;
      *reinterpret_cast<kv_f4*>(scores + t0 + 4 * g) = x[0] + row.m;
      *reinterpret_cast<kv_f4*>(scores + t0 + 4 * g + 16) = x[1] + row.m;
    }
    const float top = top_of(x);
    if (__any(row.rises(top))) {
      const float f = row.raise(top, x);
#pragma unroll
      for (int j = 0; j < kRun; ++j) o[j] *= f;
    }
    const uint4 p = row.weights(x);
    float s[2][4];
    value_scales<D>(v, t0, len, bits, s);
    add_values<D, 1, 0>(v, s, &p, &o);
  }
};

template <int D, bool BF16, bool MASK>
__global__ __launch_bounds__(kAttThreads, D == 256 ? 1 : 3) void k_kv_attend(AttendArgs a) {
  constexpr int kRun = D / 16;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work_of<kAttRows>(a, blockIdx.x);
  if (w.s < 0) {
    clear_rows<D>(a);
    return;
  }
  const int h = w.h;
  const int T = 1 << a.c.page_shift;
  const int64_t head_bytes = KvLayout<D>::head_bytes(T);

  const int end = pair_end(a, w, min(w.r0 + c, w.pairs - 1));
  const int end_first = pair_end(a, w, w.r0), end_last = pair_end(a, w, min(w.r0 + kAttRows, w.pairs) - 1);
  const int64_t part_at = (int64_t)w.part * w.tokens;
  const int from = (int)min(part_at, (int64_t)w.len), to = (int)min(part_at + w.tokens, (int64_t)end_last);
  const int whole_to = end_first - kKvStrip;   // strips up to here are seen whole

  // Strips at t0, t0 + 128, ...: kAhead strips' codes are on their way while one
  // is taken in, and the page of the next to load is read from the table before.
  constexpr int kStep = kKvStrip * kAttWaves, kAhead = D == 256 ? 1 : 2, kBufs = kAhead + 1;
  const LaneAt<D> at(T);
  Codes<D> k[kBufs], v[kBufs];
  uint32_t mb[kBufs] = {};
  bool ok[kBufs];
  const __amdgpu_buffer_rsrc_t mrs = mask_rsrc(a, w.s, h);
  // Entries of the table are scalar loads, held as they come until they are
  // needed: a vector load, or a test of one at once, would wait for every strip
  // that is on its way.
  const kv_const_i32 entries = kv_const(a.c.table + (int64_t)w.s * a.c.table_stride);
  const int last_col = max(a.c.table_cols - 1, 0);
  auto entry = [&](int t) { return entries[min(t >> a.c.page_shift, last_col)]; };
  auto load = [&](int b, int32_t page, int t) {
    ok[b] = t < to && page >= 0 && page < a.c.n_pages;
    const StripRsrc rs = strip_rsrc<D>(a.c.head_page(ok[b] ? page : 0, h, head_bytes), T, t & (T - 1), ok[b]);
    load_keys<D>(rs, at, k[b]);
    load_vals<D>(rs, at, v[b]);
    if constexpr (MASK) mb[b] = load_mask(mrs, t);   // (a byte load's result is moved, so waited for, each round)
  };
  uint4 q[D / 32];
  load_q<D>(a, w, h, w.r0, q);
  int t0 = from + wave * kKvStrip;
  int32_t pages[kAhead + 1];
#pragma unroll
  for (int i = 0; i <= kAhead; ++i) pages[i] = entry(t0 + i * kStep);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load(i, pages[i], t0 + i * kStep);
  int32_t next = pages[kAhead];
  float* scores = nullptr;
  if (a.kept && w.r0 + c < w.pairs) {
    const int r = w.r0 + c;
    scores = a.kept + ((w.first + r / a.group) * a.q_heads + h * a.group + r % a.group) * a.kept_cols;
  }
  Running<D, BF16, MASK> r;
  while (t0 < to) {
#pragma unroll
    for (int i = 0; i < kBufs; ++i) {
      if (t0 >= to) break;
      const int32_t page = next;
      next = entry(t0 + (kAhead + 1) * kStep);
      load((i + kAhead) % kBufs, page, t0 + kAhead * kStep);
      const uint32_t bits = mask_bits<MASK>(mb[i]);
      if (ok[i] && bits != 0)
        r.add(a, w.len, t0, t0 <= whole_to && bits == kAllTokens, end, bits, scores, at.shift, q, k[i], v[i]);
      else if (scores) keep_nothing(scores + t0);
      t0 += kStep;
    }
  }
  kv_f4(&o)[kRun] = r.o;
  __shared__ JoinSpace<D> js;
  join_waves<D, BF16>(a, w, w.r0, (int64_t)blockIdx.x * kAttRows, r.row, r.o, js);
  clear_rows<D>(a);
}

// Maxima and sums of N rows over their parts, by a wave: lane i reads part i's (a lane
// that read them all in turn took 17 us for 96 parts).  slot: where a row's first part is.
template <int R, int N>
__device__ __forceinline__ void joined(const AttendArgs& a, const int64_t slot[N], int parts, float M[N], float sum[N]) {
  float m[N], l[N];
#pragma unroll
  for (int n = 0; n < N; ++n) m[n] = kNoMax, l[n] = 0.0f;
  for (int i = threadIdx.x & 63; i < parts; i += 64)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float pm = a.part_m[slot[n] + (int64_t)i * R], pl = a.part_l[slot[n] + (int64_t)i * R];
      const float top = fmaxf(m[n], pm);
      l[n] = l[n] * __builtin_amdgcn_exp2f(m[n] - top) + pl * __builtin_amdgcn_exp2f(pm - top);
      m[n] = top;
    }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    M[n] = wave_max_f32(m[n]);
    sum[n] = (float)wave_sum_f64(l[n] * __builtin_amdgcn_exp2f(m[n] - M[n]));
  }
}

// Joins N rows by a wave: D/4 lanes hold a part's channels, the wave's groups of them
// every other (or fourth) part.  Rows at or past n_rows repeat the first and are not
// written.
template <int D, bool BF16, int R, int N>
__device__ __forceinline__ void join_some(const AttendArgs& a, const Work& w, int col, int n_rows) {
  constexpr int kLanes = D / 4, kGroups = 64 / kLanes;
  const int lane = threadIdx.x & 63, sub = lane % kLanes, group = lane / kLanes;
  int64_t slot[N];
#pragma unroll
  for (int n = 0; n < N; ++n) slot[n] = (int64_t)w.base * R + col + (n < n_rows ? n * kAttWaves : 0);
  float M[N], sum[N];
  joined<R, N>(a, slot, w.parts, M, sum);
  kv_f4 acc[N] = {};
#pragma unroll N == 1 ? 8 : 4
  for (int i = group; i < w.parts; i += kGroups)
#pragma unroll
    for (int n = 0; n < N; ++n)
      acc[n] += __builtin_amdgcn_exp2f(a.part_m[slot[n] + (int64_t)i * R] - M[n]) *
                *reinterpret_cast<const kv_f4*>(a.part_o + (slot[n] + (int64_t)i * R) * D + 4 * sub);
#pragma unroll
  for (int n = 0; n < N; ++n) {
#pragma unroll
    for (int d = kLanes; d < 64; d <<= 1)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[n][j] += __shfl_xor(acc[n][j], d);
    if (group != 0 || n >= n_rows) continue;
    const int pair = w.r0 + col + n * kAttWaves;
    const int64_t at = (w.first + pair / a.group) * a.q_heads + w.h * a.group + pair % a.group;
    const float inv = sum[n] == 0.0f ? 0.0f : 1.0f / sum[n];
    uint2 u;
    u.x = (uint32_t)to_out(acc[n][0] * inv, BF16) | ((uint32_t)to_out(acc[n][1] * inv, BF16) << 16);
    u.y = (uint32_t)to_out(acc[n][2] * inv, BF16) | ((uint32_t)to_out(acc[n][3] * inv, BF16) << 16);
    *reinterpret_cast<uint2*>(a.out + at * D + 4 * sub) = u;
    if (sub == 0) {
      const float e = log_sum(M[n], sum[n]);
      if (a.lse2) a.lse2[at] = e;
      if (a.lse) a.lse[at] = e * 0.6931471805599453f;
    }
  }
}

// Joins the parts of 16 rows of a unit, four a wave with their loads on their way together
// (one after the other: 13 us for 20 parts, 8 so), or, where the units' rows are up to
// kJoinFew, one: 24,066 tokens of a head and 8 rows take 18 us for 33, 4 sequences of 8,000 with 8
// heads and 16 rows 19 for 22; with 5,120 rows the plans of four times the workgroups cost
// 45 us for 43.6.
constexpr int kJoinRows = 4;
constexpr int kJoinFew = 2048;

template <int D, bool BF16, int R>
__device__ __forceinline__ void join_rows(const AttendArgs& a, uint32_t block) {
  const uint32_t per = kAttWaves * (uint32_t)a.join_rows, blocks = R / per;   // rows of a workgroup, workgroups of a unit
  const Work w = plan<R, PlanOf::kUnit>(a, block / blocks);
  if (w.s < 0 || w.parts == 1 || (int64_t)w.base + w.parts > a.blocks) return;   // (the last: starts that do not rise)
  const int col = (int)(block % blocks * per) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_rows = min((w.pairs - w.r0 - col + kAttWaves - 1) / kAttWaves, a.join_rows);
  if (n_rows <= 0) return;
  if (n_rows == 1) join_some<D, BF16, R, 1>(a, w, col, 1);
  else join_some<D, BF16, R, kJoinRows>(a, w, col, n_rows);
}

// Weights from the scores that the attention kept: p = 2^(s - lse) summed over the
// sequence's rows.  A thread takes four tokens of one head; a workgroup 1,024 with all
// rows to each thread, or, where those workgroups are few, 256 with a quarter of every
// 16 rows to each wave.
constexpr int kKeptTokens = 4 * kAttThreads;

__device__ __forceinline__ void add_kept(const AttendArgs& a, uint32_t block) {
  const int tokens = kKeptTokens / a.kept_waves, wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
  const uint32_t chunks = (uint32_t)(a.kept_cols / tokens);
  const bool share = a.kept_waves > 1;
  const int t = (int)(block % chunks) * tokens + 4 * (share ? lane : (int)threadIdx.x);
  const int h = (int)(block / chunks % (uint32_t)a.c.heads), s = (int)(block / chunks / (uint32_t)a.c.heads);
  const int64_t first = a.c.start(s);
  const int n = (int)max((int64_t)0, a.c.start(s + 1) - first), full = a.c.tokens(s);
  const int len = (int)min((int64_t)full, a.cut), pairs = n * a.group;
  if ((int)(block % chunks) * tokens >= len) return;
  // Four rows' scores at a time, the first four on their way before the plan and the
  // sums are known.
  kv_f4 x[4];
  auto load = [&](int r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // whole strips up to the row's last token were kept, others not
      const int i = (r + j) / a.group, last = a.causal ? min(len, full - n + i + 1) : len;
      const int64_t at = (first + i) * a.q_heads + h * a.group + (r + j) % a.group;
      const float no = -__builtin_inff();
      x[j] = r + j < pairs && t < last ? *reinterpret_cast<const kv_f4*>(a.kept + at * a.kept_cols + t)
                                       : kv_f4{no, no, no, no};
    }
  };
  const int r_first = share ? 4 * wave : 0, r_step = share ? kAttRows : 4;
  load(r_first);
  float* d = static_cast<float*>(a.weights.p_dev) + s * a.weights.seq_stride + h * a.weights.head_stride + t;
  // The call's sum starts at 0 and is added to what was there once: added one by one, each
  // small p would be rounded at the size of the running total.
  float w[4] = {}, had[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) had[j] = (!share || wave == 0) && t + j < min(len, a.weights.cols) ? d[j] : 0.0f;
  Work q;
  q.parts = 1;
  if (a.split_to) q = plan<kAttRows, PlanOf::kSequence>(a, (uint32_t)s);
  __shared__ float lse[kAttRows];
  for (int r0 = 0; r0 < pairs; r0 += kAttRows) {
    __syncthreads();
    if (q.parts > 1) {
      const int64_t first_part = q.base + (int64_t)(r0 / kAttRows * a.c.heads + h) * q.parts;
      float M[kJoinRows] = {}, sum[kJoinRows] = {};
      int64_t slot[kJoinRows];
      const int last = min(pairs - r0, kAttRows) - 1;
#pragma unroll
      for (int n = 0; n < kJoinRows; ++n) slot[n] = first_part * kAttRows + min(wave + n * kAttWaves, last);
      if (first_part + q.parts > a.blocks) q.parts = 0;   // (starts that do not rise)
      if (last < kAttWaves) joined<kAttRows, 1>(a, slot, q.parts, M, sum);
      else joined<kAttRows, kJoinRows>(a, slot, q.parts, M, sum);
#pragma unroll
      for (int n = 0; n < kJoinRows; ++n)
        if (lane == 0 && wave + n * kAttWaves <= last) lse[wave + n * kAttWaves] = log_sum(M[n], sum[n]);
    } else if ((int)threadIdx.x < min(pairs - r0, kAttRows)) {
      const int r = r0 + (int)threadIdx.x;
      lse[threadIdx.x] = a.lse2[(first + r / a.group) * a.q_heads + h * a.group + r % a.group];
    }
    __syncthreads();
    for (int r = r0 + r_first; r < min(pairs, r0 + kAttRows); r += r_step) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float e = r + j < pairs ? lse[r + j - r0] : 0.0f;
        e = e == -__builtin_inff() ? __builtin_inff() : e;   // no token: 2^(-inf) each
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] += __builtin_amdgcn_exp2f(x[j][i] - e);
      }
      load(r + r_step);
    }
  }
  if (share) {   // the waves' sums, in their order
    __shared__ float sums[kAttWaves][256];
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[wave][4 * lane + j] = w[j];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int i = 1; i < kAttWaves; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] += sums[i][4 * lane + j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (t + j < min(len, a.weights.cols)) d[j] = had[j] + w[j];
}

// What follows the attention, in one launch: the parts joined, the kept scores made weights.
// Bound by latency (two dependent loads for the plan, two for a row): 5 to 7 us for parts
// alone; with the scores of 16 sequences of 8,192 to 16,383 tokens and 32 heads 17 us.
template <int D, bool BF16, int R>
__global__ __launch_bounds__(kAttThreads) void k_kv_finish(AttendArgs a, uint32_t join_blocks) {
  const uint32_t b = blockIdx.x;
  if (b < join_blocks) join_rows<D, BF16, R>(a, b);
  else add_kept(a, b - join_blocks);
}

// Accumulated weights: a workgroup owns 128 tokens of one head (64 of 256 channels),
// whose keys each wave converts once; its waves share the call's rows, 16 at a time, the
// next 16 on their way; p = 2^(s - lse).  The waves' sums are added in their order, so the
// result does not depend on timing.  Bound by issue: an exponential, two additions or
// multiplications a score beside the products (64 channels: vector instructions active in 62 % of
// a SIMD's cycles, the matrix unit busy in 20), and the queries from the L2 for every
// workgroup.  2,048 rows of 32 heads over 16,384 tokens, 8 key/value heads of 128 channels:
// 267 us (64 tokens a workgroup 490, and 32 with all rows to each wave more).
template <int D>
constexpr int weight_strips() { return D == 256 ? 2 : 4; }
// Where workgroups of 128 tokens are fewer than this, they take 64: 100 rows over 3,000
// tokens of one sequence and 4 heads of 64 channels 11 us for 15, 512 rows over 8,192 24 for 31
// (with 8 heads of 128, 512 workgroups, 75 for 45).
constexpr int64_t kWeightBlocks = 512;

template <int D, bool BF16, int kStrips>
__global__ __launch_bounds__(kAttThreads, D == 256 ? 2 : D == 64 && kStrips == 2 ? 4 : D == 64 || kStrips == 2 ? 3 : 2)
void k_kv_weights(AttendArgs a) {
  constexpr int kSteps = D / 32, kTokens = kStrips * kKvStrip;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t chunks = (uint32_t)((a.cut + kTokens - 1) / kTokens);
  // Workgroups of a head read the same queries.  They are dealt out in turn to eight XCDs:
  // where each can have as many heads of every sequence, all of a head go to one and find
  // them in its L2 (2,048 rows of 32 heads over 16,384 tokens and 8 heads: of 64 channels 212
  // us for 197, of 128 265 both, of 256 956 for 923; with 4 heads of sequences of unequal
  // lengths 106 for 147, so not there).
  const bool by_xcd = a.c.heads % 8 == 0;
  const uint32_t turn = blockIdx.x / 8;
  const int t0 = (int)((by_xcd ? turn : blockIdx.x) % chunks) * kTokens;
  const uint32_t id = by_xcd ? turn / chunks * 8 + blockIdx.x % 8 : blockIdx.x / chunks;
  const int h = (int)(id % (uint32_t)a.c.heads);
  Work w;
  w.s = (int)(id / (uint32_t)a.c.heads);
  w.first = a.c.start(w.s);
  w.n = (int)max((int64_t)0, a.c.start(w.s + 1) - w.first);
  w.pairs = w.n * a.group;
  w.end_full = a.c.tokens(w.s);
  w.len = (int)min((int64_t)w.end_full, a.cut);
  if (t0 >= w.len || w.pairs == 0) return;
  const int T = 1 << a.c.page_shift;
  const LaneAt<D> at(T);
  uint4 y[2 * kStrips][kSteps];
  uint32_t bits[kStrips], any = 0, all = kAllTokens;
  bool ok[kStrips];   // the strip's page is there
#pragma unroll
  for (int n = 0; n < kStrips; ++n) {
    const int t = t0 + n * kKvStrip;
    const int64_t page = t < w.len ? a.c.page(w.s, t >> a.c.page_shift) : -1;
    ok[n] = page >= 0;
    Codes<D> k;
    load_keys<D>(strip_rsrc<D>(a.c.head_page(ok[n] ? page : 0, h, KvLayout<D>::head_bytes(T)), T, t & (T - 1), ok[n]), at, k);
    bits[n] = a.mask.p_dev ? mask_bits<true>(load_mask(mask_rsrc(a, w.s, h), t)) : kAllTokens;
    any |= ok[n] ? bits[n] : 0u;
    all &= bits[n];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      key_operand<D, BF16>(k, at.shift, kt, y[2 * n + kt]);
      if (a.flip) flip_signs<kSteps>(y[2 * n + kt]);
    }
  }
  if (any == 0) return;   // no token gets anything
  float sum[kStrips][8] = {};

  // with a causal limit the first row that sees token t0 is row t0 - (end_full - n)
  const int hidden = w.end_full - w.n;
  const int first = a.causal ? (int)min(max((int64_t)0, (int64_t)t0 - hidden) * a.group, (int64_t)w.pairs) / 16 * 16 : 0;
  int r0 = first + 16 * wave;
  // The lane's pair of the next tile: row i of the sequence, head j of the group, and
  // where its query and its log sum lie; the last pair's stand in past the end.
  constexpr int kStep = 16 * kAttWaves;
  int i = (r0 + c) / a.group, j = (r0 + c) % a.group;
  const int di = kStep / a.group, dj = kStep % a.group;
  const int64_t q_step = di * a.q_row + dj * a.q_head, q_turn = a.q_row - a.group * a.q_head;
  const int l_step = di * a.q_heads + dj, l_turn = a.q_heads - a.group;
  auto q_of = [&](int i, int j) { return a.q + (w.first + i) * a.q_row + (int64_t)(h * a.group + j) * a.q_head + g * (D / 4); };
  auto l_of = [&](int i, int j) { return a.lse2 + (w.first + i) * a.q_heads + h * a.group + j; };
  const uint16_t* qp = q_of(i, j);
  const float* lp = l_of(i, j);
  const uint16_t* const q_end = q_of(w.n - 1, a.group - 1);
  const float* const l_end = l_of(w.n - 1, a.group - 1);
  uint4 q[2][kSteps];
  float e[2];
  int row[2];
  auto load = [&](int b, int r) {
    const bool in = r + c < w.pairs;
    row[b] = i;
    load_row<D>(in ? qp : q_end, a.q_wide, q[b]);
    e[b] = *(in ? lp : l_end);   // (as it comes: a test here would wait for all that is on its way)
    i += di;
    j += dj;
    qp += q_step;
    lp += l_step;
    const bool turn = j >= a.group;
    j -= turn ? a.group : 0;
    i += turn ? 1 : 0;
    qp += turn ? q_turn : 0;
    lp += turn ? l_turn : 0;
  };
  auto add = [&](int b, int r) {
    const bool whole = all == kAllTokens && t0 + kTokens <= (a.causal ? min(w.len, hidden + r / a.group + 1) : w.len);
    const bool out = r + c >= w.pairs || e[b] == -__builtin_inff();
    const float less = out ? __builtin_inff() : e[b];   // no row, or one that sees no token: 2^(-inf) each
#pragma unroll
    for (int n = 0; n < kStrips; ++n) {
      kv_f4 x[2];
      x[0] = x[1] = kv_f4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        x[0] = mfma<BF16>(y[2 * n][s], q[b][s], x[0]);
        x[1] = mfma<BF16>(y[2 * n + 1][s], q[b][s], x[1]);
      }
#pragma unroll
      for (int v = 0; v < 8; ++v) x[v >> 2][v & 3] = __builtin_fmaf(x[v >> 2][v & 3], a.scale2, -less);
      if (!whole) {
        const int end = a.causal ? min(w.len, hidden + row[b] + 1) : w.len;
        hide(x, seen_bits(bits[n], t0 + n * kKvStrip, end));
      }
#pragma unroll
      for (int v = 0; v < 8; ++v) sum[n][v] += __builtin_amdgcn_exp2f(x[v >> 2][v & 3]);
    }
  };
  load(0, r0);
  while (r0 < w.pairs) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if (r0 >= w.pairs) break;
      load(1 - b, r0 + kStep);
      add(b, r0);
      r0 += kStep;
    }
  }
  __shared__ float total[kAttWaves][kTokens];
#pragma unroll
  for (int n = 0; n < kStrips; ++n)
#pragma unroll
    for (int v = 0; v < 8; ++v) {
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) sum[n][v] += __shfl_xor(sum[n][v], d);
      if (c == 0) total[wave][n * kKvStrip + 16 * (v >> 2) + 4 * g + (v & 3)] = ok[n] ? sum[n][v] : 0.0f;
    }
  __syncthreads();
  const int t = t0 + (int)threadIdx.x;
  if ((int)threadIdx.x < kTokens && t < w.len && t < a.weights.cols) {
    float all = 0.0f;
#pragma unroll
    for (int n = 0; n < kAttWaves; ++n) all += total[n][threadIdx.x];
    static_cast<float*>(a.weights.p_dev)[w.s * a.weights.seq_stride + h * a.weights.head_stride + t] += all;
  }
}

}  // namespace

lam_status launch_kv_attend(lam_ctx* ctx, const lam_kv_view& v, const void* q, int64_t q_row, int64_t q_head,
                            int32_t q_heads, float scale, bool causal, int64_t max_length, const lam_kv_slots& mask,
                            const lam_kv_slots& weights, void* out, float* lse) {
  AttendArgs a{};
  a.c = KvArgs::of(v);
  if (v.table_cols == 0) a.c.table = v.lengths_dev, a.c.table_stride = 0;   // never used, but read ahead of the length
  a.q = static_cast<const uint16_t*>(q);
  a.q_row = q_row;
  a.q_head = q_head;
  a.q_wide = (reinterpret_cast<uintptr_t>(q) & 15) == 0 && q_row % 8 == 0 && q_head % 8 == 0;
  a.q_heads = q_heads;
  a.group = q_heads / v.kv_heads;
  a.causal = causal;
  // a scale of 0 becomes one that no score survives, and masked ones (-inf) stay what they are
  a.scale2 = std::max((float)(std::fabs((double)scale) * 1.4426950408889634), 1e-37f);
  a.flip = scale < 0.0f;
  a.cut = (int64_t)v.table_cols * v.page_size;
  if (max_length > 0) a.cut = std::min(a.cut, max_length);
  if (v.n_pages == 0) a.cut = 0;

  a.mask = mask;
  a.weights = weights;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;

  const bool chunk = v.rows * a.group > kChunkPairs * (int64_t)v.n_seqs;
  const int fill = v.head_dim == 256 ? kFillWide : chunk ? kFillChunk : kFillDecode;
  auto units_of = [&](int rows) {   // tiles of every head
    const int64_t tiles = v.starts_dev ? v.rows * a.group / rows + v.n_seqs
                                       : (v.rows / v.n_seqs * a.group + rows - 1) / rows * v.n_seqs;
    return tiles * v.kv_heads;
  };
  int rows = chunk ? kChunkRows : kAttRows;
  if (chunk && v.head_dim == 256) {
    // A round of 48 rows takes 1.2 times one of 32: 48 where the rounds that the chip takes
    // are fewer by as much.  (405 rows of 32 heads, 4 key/value heads, 17,034 tokens: two
    // rounds of either, 514 us by 32 and 599 by 48; 100 rows of 32 and 8 heads of 3
    // sequences of 8,000: 247 and 160; 2,048 rows over 8,192: 893 and 808.)
    const int64_t wide = (units_of(kChunkRowsWide) + fill - 1) / fill, wider = (units_of(kChunkRowsWider) + fill - 1) / fill;
    rows = 6 * wider <= 5 * wide ? kChunkRowsWider : kChunkRowsWide;
  }
  if (!v.starts_dev) a.tiles_per_seq = (int)((v.rows / v.n_seqs * a.group + rows - 1) / rows);
  // Lengths are split where the tiles do not fill the chip; of 256 channels, whose
  // workgroups have a compute unit each, over two rounds where the tiles fill a little more
  // than one (1.06 to 1.31 times: 10 to 19 % less, 36 sequences of 30,000 tokens 598 us to
  // 487; 1.4 times: 2 % more; of 128 channels 1.04 times: 3 % less to 14 % more).
  const int64_t units = units_of(rows);
  const int split_to = v.head_dim == 256 && units >= fill && 8 * units < 11 * fill ? 2 * fill : fill;
  int64_t blocks = units;
  if (units < split_to && a.cut > (chunk ? kWholeChunk : kWholeDecode)) {
    a.split_to = split_to;
    blocks = split_to + units;   // see plan(): at most split_to - units / 2 (or split_to / 2) full parts, and one more a tile
  }
  a.blocks = blocks;

  // Weights: from scores that the attention keeps (8 bytes a row and token, written
  // and read) where it is not the kernel for chunks, else from a second pass over the
  // keys.  (16 sequences of 8,192 tokens, 8 heads of 128 channels: 44 and 158 us for 4 pairs
  // a head, 60 and 161 for 16.)
  const int64_t pairs = v.rows * q_heads;
  const int64_t parts = a.split_to ? blocks * rows : 0;
  a.kept_cols = (a.cut + kKeptTokens - 1) / kKeptTokens * kKeptTokens;
  const bool keep = weights.p_dev && !chunk && pairs <= kKeptBytes / 4 / std::max<int64_t>(a.kept_cols, 1);
  // every refusal, before the first launch is queued: a call that is refused has written nothing
  a.join_rows = units * rows <= kJoinFew ? 1 : kJoinRows;
  const int64_t join_blocks = a.split_to ? units * (rows / (kAttWaves * a.join_rows)) : 0;
  int64_t kept_blocks = keep ? a.kept_cols / kKeptTokens * v.kv_heads * v.n_seqs : 0;
  // (4 sequences of 4,000 tokens, 64 pairs: 51 us with one wave a token, 46 with four;
  // 4 of 8,192 and 4 pairs: 21 and 22)
  a.kept_waves = kept_blocks < 1024 && v.rows * a.group > kAttRows * (int64_t)v.n_seqs ? 4 : 1;
  kept_blocks *= a.kept_waves;
  const int64_t heads = (int64_t)v.kv_heads * v.n_seqs;
  auto weight_blocks_of = [&](int strips) { return (a.cut + strips * kKvStrip - 1) / (strips * kKvStrip) * heads; };
  const bool few = v.head_dim == 256 || weight_blocks_of(4) < kWeightBlocks;
  const int64_t weight_blocks = weights.p_dev && !keep ? weight_blocks_of(few ? 2 : 4) : 0;   // (a cut of 0: none)
  LAM_CHECK(std::max({blocks, join_blocks + kept_blocks, weight_blocks}) <= most_blocks(kAttThreads), LAM_EINVAL,
            "too many rows, or sequences times the bound of lengths, for one launch (%lld tokens: give max_length)",
            (long long)a.cut);
  LAM_CHECK(weight_blocks == 0 || q != out, LAM_EINVAL, "out is q, which the weights take a second pass over");
  const int64_t floats = (keep ? pairs * a.kept_cols : 0) + parts * (v.head_dim + 2) + (weights.p_dev ? pairs : 0);
  void* scratch = nullptr;
  if (floats > 0) LAM_TRY(kv_scratch(ctx, (size_t)floats * 4, &scratch));
  float* at = static_cast<float*>(scratch);
  if (keep) {
    a.kept = at;
    at += pairs * a.kept_cols;
  }
  a.part_o = at;
  a.part_m = a.part_o + parts * v.head_dim;
  a.part_l = a.part_m + parts;
  if (weights.p_dev) a.lse2 = a.part_l + parts;

  hipEvent_t e0, e1;
  if (chunk) {
    LAM_TRY(launch_kv_chunk(ctx, v, a, rows, blocks, mask.p_dev != nullptr));
  } else {
    LAM_TRY(prof_launch_events(ctx, "kv_attend", &e0, &e1));
#define LAM_GO(D, BF)                                                                                          \
  do {                                                                                                         \
    if (mask.p_dev) launch(k_kv_attend<D, BF, true>, dim3((unsigned)blocks), kAttThreads, ctx->stream, e0, e1, a); \
    else launch(k_kv_attend<D, BF, false>, dim3((unsigned)blocks), kAttThreads, ctx->stream, e0, e1, a);       \
  } while (0)
    LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
    LAM_HIP(hipGetLastError());
  }
  if (join_blocks + kept_blocks > 0) {
    LAM_TRY(prof_launch_events(ctx, "kv_finish", &e0, &e1));
    const dim3 grid((unsigned)(join_blocks + kept_blocks));
    const uint32_t jb = (uint32_t)join_blocks;
#define LAM_GO(D, BF)                                                                                 \
  do {                                                                                                \
    constexpr int kMost = D == 256 ? kChunkRowsWider : kChunkRows;                                    \
    constexpr int kLess = D == 256 ? kChunkRowsWide : kChunkRows;                                     \
    if (!chunk) launch(k_kv_finish<D, BF, kAttRows>, grid, kAttThreads, ctx->stream, e0, e1, a, jb);  \
    else if (rows == kMost) launch(k_kv_finish<D, BF, kMost>, grid, kAttThreads, ctx->stream, e0, e1, a, jb); \
    else launch(k_kv_finish<D, BF, kLess>, grid, kAttThreads, ctx->stream, e0, e1, a, jb);            \
  } while (0)
    LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
    LAM_HIP(hipGetLastError());
  }
  if (weight_blocks > 0) {
    LAM_TRY(prof_launch_events(ctx, "kv_weights", &e0, &e1));
    const dim3 grid((unsigned)weight_blocks);
#define LAM_GO(D, BF)                                                                                       \
  do {                                                                                                      \
    if (few) launch(k_kv_weights<D, BF, 2>, grid, kAttThreads, ctx->stream, e0, e1, a);                     \
    else launch(k_kv_weights<D, BF, weight_strips<D>()>, grid, kAttThreads, ctx->stream, e0, e1, a);        \
  } while (0)
    LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
    LAM_HIP(hipGetLastError());
  }
  return LAM_OK;
}

}  // namespace lam
