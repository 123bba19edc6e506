// Attention of chunks of queries over the 4-bit cache (lam_kv_attend where a
// sequence has more than a few rows).
//
// As in kv_attend.hip a wave walks strips of 32 tokens and keeps everything but
// the queries in registers; here it takes 64 query rows (32 for heads of 256
// channels), so that a strip's conversions serve four products instead of one.
// One wave is a workgroup: nothing is shared, nothing waits at a barrier.
#include <hip/hip_ext.h>

#include "kv_attend.h"

namespace lam {
namespace {

template <int D, bool BF16, bool MASK>
__global__ __launch_bounds__(64, D == 256 ? 1 : 2) void k_kv_chunk(AttendArgs a) {
  constexpr int kRun = D / 16, kRows = chunk_rows(D), kTiles = kRows / 16, kSteps = D / 32;
  const int lane = threadIdx.x, c = lane & 15, g = lane >> 4;
  const Work w = work_of<kRows>(a, blockIdx.x);
  if (w.s < 0) return;
  const int T = 1 << a.c.page_shift;
  const int64_t head_bytes = KvLayout<D>::head_bytes(T);

  // the queries, as B operands, for the whole walk
  __shared__ uint4 sq[kTiles][kSteps][64];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    uint4 q[kSteps];
    load_q<D>(a, w, w.h, w.r0 + 16 * t, q);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) sq[t][j][lane] = q[j];
  }

  const int end_first = pair_end(a, w, w.r0), end_last = pair_end(a, w, min(w.r0 + kRows, w.pairs) - 1);
  const int64_t part_at = (int64_t)w.part * w.tokens;
  const int from = (int)min(part_at, (int64_t)w.len), to = (int)min(part_at + w.tokens, (int64_t)end_last);
  const int whole_to = MASK ? -1 : end_first - kKvStrip;

  kv_f4 o[kTiles][kRun];
  float m[kTiles], l[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    m[t] = kNoMax;
    l[t] = 0.0f;
#pragma unroll
    for (int j = 0; j < kRun; ++j) o[t][j] = kv_f4{0, 0, 0, 0};
  }

  const LaneAt<D> at(T);
  Codes<D> k[2], v[2];
  uint32_t mb[2] = {};
  bool ok[2];
  const __amdgpu_buffer_rsrc_t mrs = mask_rsrc(a, w.s, w.h);
  const kv_const_i32 entries = kv_const(a.c.table + (int64_t)w.s * a.c.table_stride);
  const int last_col = max(a.c.table_cols - 1, 0);
  auto entry = [&](int t) { return entries[min(t >> a.c.page_shift, last_col)]; };
  auto load = [&](int b, int32_t page, int t) {
    ok[b] = t < to && page >= 0 && page < a.c.n_pages;
    const StripRsrc rs = strip_rsrc<D>(a.c.head_page(ok[b] ? page : 0, w.h, head_bytes), T, t & (T - 1), ok[b]);
    load_keys<D>(rs, at, k[b]);
    load_vals<D>(rs, at, v[b]);
    if constexpr (MASK) mb[b] = load_mask(mrs, t);
  };

  auto add = [&](int b, int t0) {
    // scores of 32 tokens for every tile of queries
    kv_f4 x[kTiles][2];
    {
      uint4 y[2][kSteps];
      key_operand<D, BF16>(k[b], at.shift, 0, y[0]);
      key_operand<D, BF16>(k[b], at.shift, 1, y[1]);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        x[t][0] = x[t][1] = kv_f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const uint4 q = sq[t][j][lane];
          x[t][0] = mfma<BF16>(y[0][j], q, x[t][0]);
          x[t][1] = mfma<BF16>(y[1][j], q, x[t][1]);
        }
      }
    }
    if (t0 > whole_to) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int end = pair_end(a, w, min(w.r0 + 16 * t + c, w.pairs - 1));
        const uint32_t in = seen_bits(MASK, mb[b], t0, end);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[t][i >> 2][i & 3] = (in >> i) & 1u ? x[t][i >> 2][i & 3] : -__builtin_inff();
      }
    }
    float top[kTiles];
    bool up = false;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      float z = fmaxf(x[t][0][0], x[t][1][0]);
#pragma unroll
      for (int i = 1; i < 4; ++i) z = fmaxf(z, fmaxf(x[t][0][i], x[t][1][i]));
      top[t] = z * a.scale2;
      up |= top[t] > m[t] + kSpan;
    }
    if (__any(up)) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        float z = fmaxf(top[t], __shfl_xor(top[t], 16));
        z = fmaxf(z, __shfl_xor(z, 32));
        const float next = z > m[t] + kSpan ? z - kLift : m[t];
        const float f = __builtin_amdgcn_exp2f(m[t] - next);
        m[t] = next;
        l[t] *= f;
#pragma unroll
        for (int j = 0; j < kRun; ++j) o[t][j] *= f;
      }
    }
    uint4 p[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][i >> 2][i & 3], a.scale2, -m[t]));
        l[t] += e[i];
      }
      p[t] = uint4{pack_half(e[0], e[1]), pack_half(e[2], e[3]), pack_half(e[4], e[5]), pack_half(e[6], e[7])};
    }
    float s[2][4];
    value_scales<D>(v[b], t0, w.len, s);
    add_values<D, kTiles, 0>(v[b], s, p, o);
  };

  int t0 = from;
  int32_t page = entry(t0), next = entry(t0 + kKvStrip);
  load(0, page, t0);
  while (t0 < to) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (t0 >= to) break;
      page = next;
      next = entry(t0 + 2 * kKvStrip);
      load(1 - i, page, t0 + kKvStrip);
      if (ok[i]) add(i, t0);
      t0 += kKvStrip;
    }
  }

#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    float sum = l[t];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const int pair = w.r0 + 16 * t + c;
    if (pair >= w.pairs) continue;
    if (w.parts > 1) {
      const int64_t p = (int64_t)blockIdx.x * kRows + 16 * t + c;
      if (g == 0) {
        a.part_m[p] = m[t];
        a.part_l[p] = sum;
      }
      float* d = a.part_o + p * D + 4 * g * kRun;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kRun; j += 4)
          *reinterpret_cast<kv_f4*>(d + i * kRun + j) = kv_f4{o[t][j][i], o[t][j + 1][i], o[t][j + 2][i], o[t][j + 3][i]};
    } else {
      const int64_t row = (w.first + pair / a.group) * a.q_heads + w.h * a.group + pair % a.group;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float acc[kRun];
#pragma unroll
        for (int j = 0; j < kRun; ++j) acc[j] = o[t][j][i];
        write_row<D, BF16>(a, row, 4 * g + i, acc, m[t], sum);
      }
    }
  }
}

}  // namespace

lam_status launch_kv_chunk(lam_ctx* ctx, const lam_kv_view& v, const AttendArgs& a, int64_t blocks, bool masked) {
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_chunk", &e0, &e1));
#define LAM_GO(D, BF)                                                                                            \
  do {                                                                                                           \
    if (masked)                                                                                                  \
      hipExtLaunchKernelGGL((k_kv_chunk<D, BF, true>), dim3((unsigned)blocks), dim3(64), 0, ctx->stream, e0, e1, \
                            0, a);                                                                               \
    else                                                                                                         \
      hipExtLaunchKernelGGL((k_kv_chunk<D, BF, false>), dim3((unsigned)blocks), dim3(64), 0, ctx->stream, e0,    \
                            e1, 0, a);                                                                           \
  } while (0)
  LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

}  // namespace lam
