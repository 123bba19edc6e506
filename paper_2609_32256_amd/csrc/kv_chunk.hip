// Attention of chunks of queries over the 4-bit cache (lam_kv_attend where a
// sequence has more than a few rows).
//
// As in kv_attend.hip the waves of a workgroup walk strips of 32 tokens and keep
// everything but the queries in registers; here they take 64 query rows (32 or 48 for
// heads of 256 channels), so that a strip's conversions serve four products instead of
// one.  The queries lie in LDS for all of them; they meet only at the end, when
// their sums are joined.
//
// Bound by instructions that share their issue with the products: a strip's conversions, and
// for every score an exponential, a fused multiply and add, a comparison, a sum and half a
// conversion.  2,048 rows of 32 heads over 32,768 tokens (8 key/value heads of 128 channels,
// bfloat16): 1,045 us, 1,020 TFLOP/s; a library product of 8,192^3 reaches 1,200.  By the
// counters vector instructions are active in 62 % of a SIMD's cycles there and the matrix unit
// is busy in 42; with heads of 64 channels in 67 and 26.  4,096 rows over 32,768 tokens with a window of
// 4,096: 298 us, 923 TFLOP/s, in four rounds of tiles that each begin and end with a wait.  Of 256 channels, 2,048
// rows of 16 heads over 4: with that window 284 us, 484 TFLOP/s, without one 1,900 us, 560.
#include "kv_attend.h"

namespace lam {
namespace {

template <int D, bool BF16, bool MASK, bool WINDOW, int kRows>
__global__ __launch_bounds__(kAttThreads, D == 256 ? 1 : D == 64 ? 3 : 2) void k_kv_chunk(AttendArgs a) {
  constexpr int kRun = D / 16, kTiles = kRows / 16, kSteps = D / 32;
  const int lane = threadIdx.x & 63, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work_of<kRows>(a, blockIdx.x);
  if (w.s < 0) {
    clear_rows<D>(a);
    return;
  }
  const int T = 1 << a.c.page_shift;
  const int64_t head_bytes = KvLayout<D>::head_bytes(T);

  // the queries, as B operands, for the whole walk
  __shared__ uint4 sq[kTiles][kSteps][64];
  for (int t = wave; t < kTiles; t += kAttWaves) {
    uint4 q[kSteps];
    load_q<D>(a, w, w.h, w.r0 + 16 * t, q);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) sq[t][j][lane] = q[j];
  }

  __syncthreads();

  const int last = min(w.r0 + kRows, w.pairs) - 1, end_first = pair_end(a, w, w.r0);
  int begin_first = 0, begin_last = 0;
  Walk walk;
  if constexpr (WINDOW) {
    begin_first = pair_begin(a, w, w.r0);
    begin_last = pair_begin(a, w, last);
    walk = Walk(a, w.len, begin_first);
  }
  // places from `from` to `to`, which are tokens where there is no window
  const int64_t part_at = (int64_t)w.part * w.tokens;
  const int from = (int)min(part_at, (int64_t)walk.places(w.len));
  const int to = (int)min(part_at + w.tokens, (int64_t)walk.places(pair_end(a, w, last)));
  const int whole_to = end_first - kKvStrip;

  kv_f4 o[kTiles][kRun];
  Row row[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int j = 0; j < kRun; ++j) o[t][j] = kv_f4{0, 0, 0, 0};

  // One strip's codes in registers: the next one's keys are loaded as soon as the
  // keys are converted, its values when the values are.
  const LaneAt<D> at(T);
  Codes<D> k, v;
  uint32_t mb = 0;
  const __amdgpu_buffer_rsrc_t mrs = mask_rsrc(a, w.s, w.h);
  const kv_const_i32 entries = kv_const(a.c.table + (int64_t)w.s * a.c.table_stride);
  const int last_col = max(a.c.table_cols - 1, 0);
  auto entry = [&](int place) { return entries[min(walk.token(place) >> a.c.page_shift, last_col)]; };
  const uint32_t n_pages = (uint32_t)a.c.n_pages;
  // the page of the strip to load next
  uint8_t* head;
  bool ok_page;
  auto turn = [&](int32_t page) {
    ok_page = (uint32_t)page < n_pages;
    head = a.c.head_page(ok_page ? page : 0, w.h, head_bytes);
  };
  constexpr int kStep = kKvStrip * kAttWaves;
  int place = from + wave * kKvStrip;
  int32_t next = entry(place + kStep);
  turn(entry(place));
  bool ok = place < to && ok_page;
  {
    const int t0 = walk.token(place);
    const StripRsrc rs = strip_rsrc<D>(head, T, t0 & (T - 1), ok);
    load_keys<D>(rs, at, k);
    load_vals<D>(rs, at, v);
    if constexpr (MASK) mb = load_mask(mrs, t0);
  }
  for (; place < to; place += kStep) {
    const int t0 = walk.token(place);
    uint4 y[2][kSteps];
    key_operand<D, BF16>(k, at.shift, 0, y[0]);
    key_operand<D, BF16>(k, at.shift, 1, y[1]);
    const int t1 = walk.token(place + kStep);
    turn(next);
    next = entry(place + 2 * kStep);
    const bool ok_next = place + kStep < to && ok_page;
    const StripRsrc rs = strip_rsrc<D>(head, T, t1 & (T - 1), ok_next);
    load_keys<D>(rs, at, k);
    uint32_t bits = mask_bits<MASK>(mb);
    bool whole = t0 <= whole_to;
    if constexpr (WINDOW) {
      bits &= window_bits(a, t0, begin_first);   // (what no row sees may hold anything)
      whole = whole && (t0 >= begin_last || t0 + kKvStrip <= a.sinks);
    }
    if (ok && bits != 0) {
      // scores of 32 tokens for every tile of queries, less the row's reference
      kv_f4 x[kTiles][2];
      uint4 q = sq[0][0][lane];
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        x[t][0] = x[t][1] = kv_f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const int n = t * kSteps + j + 1;
          uint4 q_next = q;
          if (n < kTiles * kSteps) q_next = sq[n / kSteps][n % kSteps][lane];
          x[t][0] = mfma<BF16>(y[0][j], q, x[t][0]);
          x[t][1] = mfma<BF16>(y[1][j], q, x[t][1]);
          q = q_next;
        }
      }
      float s[2][4];
      value_scales<D>(v, t0, w.len, bits, s);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) less_reference(x[t], a.scale2, row[t]);
      // with a window what the mask takes out of whole strips is taken out of all rows alike (not at 64
      // channels, where it spills)
      constexpr bool kAlike = MASK && WINDOW && D != 64;
      if (!whole || (!kAlike && bits != kAllTokens)) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          const int r = min(w.r0 + 16 * t + c, w.pairs - 1);
          uint32_t in = bits;
          if constexpr (WINDOW) in &= window_bits(a, t0, pair_begin(a, w, r));
          hide(x[t], seen_bits(in, t0, pair_end(a, w, r)));
        }
      } else if (kAlike && bits != kAllTokens) {
        const uint32_t in = seen_bits(bits, t0, t0 + kKvStrip);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) hide(x[t], in);
      }
      bool up = false;
      float top[kTiles];
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        top[t] = top_of(x[t]);
        up |= row[t].rises(top[t]);
      }
      if (__any(up)) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          const float f = row[t].raise(top[t], x[t]);
#pragma unroll
          for (int j = 0; j < kRun; ++j) o[t][j] *= f;
        }
      }
      uint4 p[kTiles];
#pragma unroll
      for (int t = 0; t < kTiles; ++t) p[t] = row[t].weights(x[t]);
      add_values<D, kTiles, 0>(v, s, p, o);
    }
    load_vals<D>(rs, at, v);
    if constexpr (MASK) mb = load_mask(mrs, t1);
    ok = ok_next;
  }

  __shared__ JoinSpace<D> js;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    if (t > 0) __syncthreads();   // (all 256 threads get here for every tile)
    join_waves<D, BF16>(a, w, w.r0 + 16 * t, (int64_t)blockIdx.x * kRows + 16 * t, row[t], o[t], js);
  }
  clear_rows<D>(a);
}

}  // namespace

lam_status launch_kv_chunk(lam_ctx* ctx, const lam_kv_view& v, const AttendArgs& a, int rows, int64_t blocks,
                           bool masked, bool windowed) {
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_chunk", &e0, &e1));
  const dim3 grid((unsigned)blocks);
#define LAM_VIEW(D, BF, M, W, R) launch(k_kv_chunk<D, BF, M, W, R>, grid, kAttThreads, ctx->stream, e0, e1, a)
#define LAM_ROWS(D, BF, R)                                                                                 \
  do {                                                                                                     \
    if (windowed) { if (masked) LAM_VIEW(D, BF, true, true, R); else LAM_VIEW(D, BF, false, true, R); }    \
    else { if (masked) LAM_VIEW(D, BF, true, false, R); else LAM_VIEW(D, BF, false, false, R); }           \
  } while (0)
#define LAM_GO(D, BF)                                                                             \
  do {                                                                                            \
    if constexpr (D != 256) LAM_ROWS(D, BF, kChunkRows);                                          \
    else if (rows == kChunkRowsWider) LAM_ROWS(D, BF, kChunkRowsWider);                           \
    else LAM_ROWS(D, BF, kChunkRowsWide);                                                         \
  } while (0)
  LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
#undef LAM_ROWS
#undef LAM_VIEW
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

}  // namespace lam
