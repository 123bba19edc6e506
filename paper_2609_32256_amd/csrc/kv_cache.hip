// The 4-bit key/value cache's own memory: rows quantized into it, values read
// back, and tokens evicted from it (include/lam.h, lam_kv_*).
#include <hip/hip_ext.h>

#include <algorithm>

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

// Eight channels of a row as float32.
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t at, bool wide, float x[8]) {
  const uint16_t* h = static_cast<const uint16_t*>(p) + at;
  uint32_t w[4];
  if (wide) {
    const uint4 u = *reinterpret_cast<const uint4*>(h);
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

// One lane per eight channels of a row's head.
template <int D, bool BF16>
__global__ __launch_bounds__(kKvThreads) void k_kv_append(KvArgs a, RowArgs k, RowArgs v, lam_kv_slots weights,
                                                          lam_kv_slots positions, const int32_t* first,
                                                          uint32_t* status) {
  using L = KvLayout<D>;
  constexpr int kLanes = D / 8;
  const int64_t item = (int64_t)blockIdx.x * kKvThreads + threadIdx.x;
  const int64_t unit = item / kLanes;
  const int sub = (int)(item % kLanes);
  const int64_t row = unit / a.heads;
  const int h = (int)(unit % a.heads);
  bool bad = false, over = false, lost = false;
  if (row < a.rows) {
    const int s = a.seq_of(row);
    const int T = 1 << a.page_shift;
    int64_t page = -1, slot = -1;
    int64_t i = 0;
    if (s >= 0) {
      const int64_t r0 = a.start(s), n = a.start(s + 1) - r0;
      i = row - r0;
      slot = (int64_t)a.lengths[s] - n + i;
      if (slot >= 0 && (slot >> a.page_shift) < a.table_cols) page = a.page(s, (int)(slot >> a.page_shift));
    }
    lost = page < 0 && sub == 0;
    if (page >= 0) {
      float x[8], y[8];
      load8<BF16>(k.p, row * k.row + h * k.head + 8 * sub, k.wide, x);
      load8<BF16>(v.p, row * v.row + h * v.head + 8 * sub, v.wide, y);
      uint32_t kb, vb;
      const uint32_t kw = quantize8(x, &kb, &bad, &over), vw = quantize8(y, &vb, &bad, &over);
      uint8_t* base = a.head_page(page, h, L::head_bytes(T));
      const int t = (int)(slot & (T - 1));
      *reinterpret_cast<uint32_t*>(base + L::k_codes(t) + 4 * sub) = kw;
      put_v_word<D>(base, T, t, sub, vw);
      if ((sub & 3) == 0) {
        base[L::k_scales(T, t) + (sub >> 2)] = (uint8_t)kb;
        base[L::v_scales(T, t, sub >> 2)] = (uint8_t)vb;
      }
      if (sub == 0) {
        if (weights.p_dev && slot < weights.cols)
          static_cast<float*>(weights.p_dev)[s * weights.seq_stride + h * weights.head_stride + slot] = 0.0f;
        if (positions.p_dev && slot < positions.cols)
          static_cast<int32_t*>(positions.p_dev)[s * positions.seq_stride + h * positions.head_stride + slot] =
              (int32_t)(first[s] + i);
      }
    }
  }
  if (status) {
    count_in(status, 0, bad);
    count_in(status, 1, over);
    count_in(status, 2, lost);
  }
}

template <int D, bool BF16>
__global__ __launch_bounds__(kKvThreads) void k_kv_read(KvArgs a, uint4* k, uint4* v) {
  using L = KvLayout<D>;
  constexpr int kLanes = D / 8;
  const int64_t item = (int64_t)blockIdx.x * kKvThreads + threadIdx.x;
  const int64_t unit = item / kLanes;
  const int sub = (int)(item % kLanes);
  const int64_t row = unit / a.heads;
  const int h = (int)(unit % a.heads);
  if (row >= a.rows) return;
  const int s = a.seq_of(row);
  const int T = 1 << a.page_shift;
  uint4 x{0, 0, 0, 0}, y{0, 0, 0, 0};
  if (s >= 0) {
    const int64_t r0 = a.start(s), n = a.start(s + 1) - r0;
    const int64_t slot = (int64_t)a.lengths[s] - n + (row - r0);
    if (slot >= 0 && (slot >> a.page_shift) < a.table_cols) {
      const int64_t page = a.page(s, (int)(slot >> a.page_shift));
      if (page >= 0) {
        const uint8_t* base = a.head_page(page, h, L::head_bytes(T));
        const int t = (int)(slot & (T - 1));
        x = kv_values8<BF16>(*reinterpret_cast<const uint32_t*>(base + L::k_codes(t) + 4 * sub),
                             kv_scale(base[L::k_scales(T, t) + (sub >> 2)]));
        y = kv_values8<BF16>(get_v_word<D>(base, T, t, sub), kv_scale(base[L::v_scales(T, t, sub >> 2)]));
      }
    }
  }
  k[item] = x;
  v[item] = y;
}

// ------------------------------------------------------------------ eviction
constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;

struct EvictArgs {
  lam_kv_slots scores, positions, scores_out, positions_out;
  int32_t budget, recent, sinks, bound;   // bound: most tokens of a sequence
  int32_t moves;                          // most moves of a sequence's head
  int32_t* kept;
  int32_t* lengths_out;
  int32_t* holes;    // [seq][head][moves]
  int32_t* extras;
  int32_t* n_moves;  // [seq][head]
};

// Order of the scores as unsigned integers: protected slots above all, NaN below all.
__device__ __forceinline__ uint32_t evict_key(float s, int pos, int newest, int recent, int sinks) {
  if (pos < sinks || (int64_t)pos > (int64_t)newest - recent) return 0xffffffffu;
  if (s != s) return 0u;
  const uint32_t b = __float_as_uint(s + 0.0f);   // -0 counts as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// One workgroup per sequence and head.  The budget-th largest key is found digit
// by digit (four histograms of 256 counts); then one pass over the slots in order
// marks those that stay (ties by slot) and lists the holes below budget and the
// kept slots beyond it.
__global__ __launch_bounds__(kSelThreads) void k_kv_select(KvArgs a, EvictArgs e) {
  const int bh = blockIdx.x;
  const int s = bh / a.heads, h = bh % a.heads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = min(a.length(s), e.bound);
  const float* sc = static_cast<const float*>(e.scores.p_dev) + s * e.scores.seq_stride + h * e.scores.head_stride;
  const int32_t* ps = e.positions.p_dev ? static_cast<const int32_t*>(e.positions.p_dev) + s * e.positions.seq_stride +
                                              h * e.positions.head_stride
                                        : nullptr;
  float* so = static_cast<float*>(e.scores_out.p_dev) + s * e.scores_out.seq_stride + h * e.scores_out.head_stride;
  int32_t* po = e.positions_out.p_dev ? static_cast<int32_t*>(e.positions_out.p_dev) +
                                            s * e.positions_out.seq_stride + h * e.positions_out.head_stride
                                      : nullptr;
  int32_t* kept = e.kept + (int64_t)bh * e.budget;
  int32_t* holes = e.holes + (int64_t)bh * e.moves;
  int32_t* extras = e.extras + (int64_t)bh * e.moves;
  if (len <= e.budget) {
    for (int t = tid; t < e.budget; t += kSelThreads) {
      const bool in = t < len;
      kept[t] = in ? t : -1;
      so[t] = in ? sc[t] : 0.0f;
      if (po) po[t] = in ? (ps ? ps[t] : t) : -1;
    }
    if (tid == 0) e.n_moves[bh] = 0;
    return;
  }
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];
  __shared__ int32_t cnt[2][3][kSelWaves];
  const int newest = ps ? ps[len - 1] : len - 1;
  auto key_of = [&](int t) { return evict_key(sc[t], ps ? ps[t] : t, newest, e.recent, e.sinks); };

  uint32_t prefix = 0, need = (uint32_t)e.budget;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    const uint32_t above = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int t = tid; t < len; t += kSelThreads) {
      const uint32_t k = key_of(t);
      if ((k & above) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      // lane l holds the digits 255 - 4 l down to 252 - 4 l; sums from the top
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j] = hist[255 - 4 * lane - j];
      uint32_t upto = sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
      }
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
  for (int t0 = 0; t0 < len; t0 += kSelThreads, buf ^= 1) {
    const int t = t0 + tid;
    const uint32_t k = t < len ? key_of(t) : 0u;
    const bool eq = t < len && k == prefix;
    const unsigned long long me = __ballot(eq), low = (1ull << lane) - 1;
    if (lane == 0) cnt[buf][0][wave] = (int)__popcll(me);
    __syncthreads();
    int rank = ties + (int)__popcll(me & low);
    for (int w = 0; w < kSelWaves; ++w) {
      if (w < wave) rank += cnt[buf][0][w];
      ties += cnt[buf][0][w];
    }
    const bool stays = t < len && (k > prefix || (eq && rank < (int)need));
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
    if (t < e.budget && stays) {
      kept[t] = t;
      so[t] = sc[t];
      if (po) po[t] = ps ? ps[t] : t;
    }
  }
  __syncthreads();
  for (int i = tid; i < n_holes; i += kSelThreads) {
    const int to = holes[i], from = extras[i];
    kept[to] = from;
    so[to] = sc[from];
    if (po) po[to] = ps ? ps[from] : from;
  }
  if (tid == 0) e.n_moves[bh] = n_holes;
}

// Moves the listed tokens' codes and scales: D/8 lanes a token.  Sources lie at
// or beyond budget and destinations below it, so no move reads what another wrote.
template <int D>
__global__ __launch_bounds__(kKvThreads) void k_kv_move(KvArgs a, EvictArgs e) {
  using L = KvLayout<D>;
  constexpr int kLanes = D / 8;
  const int bh = blockIdx.y;
  const int s = bh / a.heads, h = bh % a.heads;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0)
    e.lengths_out[s] = min(min(a.length(s), e.bound), e.budget);
  const int T = 1 << a.page_shift;
  const int i = blockIdx.x * (kKvThreads / kLanes) + threadIdx.x / kLanes;
  const int sub = threadIdx.x % kLanes;
  if (i >= e.n_moves[bh]) return;
  const int to = e.holes[(int64_t)bh * e.moves + i], from = e.extras[(int64_t)bh * e.moves + i];
  const int64_t pd = a.page(s, to >> a.page_shift), pf = a.page(s, from >> a.page_shift);
  if (pd < 0 || pf < 0) return;
  uint8_t* d = a.head_page(pd, h, L::head_bytes(T));
  const uint8_t* f = a.head_page(pf, h, L::head_bytes(T));
  const int td = to & (T - 1), tf = from & (T - 1);
  const uint32_t kw = *reinterpret_cast<const uint32_t*>(f + L::k_codes(tf) + 4 * sub);
  const uint32_t vw = get_v_word<D>(f, T, tf, sub);
  *reinterpret_cast<uint32_t*>(d + L::k_codes(td) + 4 * sub) = kw;
  put_v_word<D>(d, T, td, sub, vw);
  if ((sub & 3) == 0) {
    const int b = sub >> 2;
    d[L::k_scales(T, td) + b] = f[L::k_scales(T, tf) + b];
    d[L::v_scales(T, td, b)] = f[L::v_scales(T, tf, b)];
  }
}

bool wide_rows(const void* p, int64_t row, int64_t head) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && row % 8 == 0 && head % 8 == 0;
}

// blocks of kKvThreads lanes, D/8 lanes per row and head
lam_status row_grid(const lam_kv_view& v, unsigned* grid) {
  const int64_t items = v.rows * v.kv_heads * (v.head_dim / 8);
  const int64_t g = (items + kKvThreads - 1) / kKvThreads;
  LAM_CHECK(g < (1LL << 31), LAM_EINVAL, "too many rows for one launch");
  *grid = (unsigned)g;
  return LAM_OK;
}

}  // namespace

lam_status launch_kv_append(lam_ctx* ctx, const lam_kv_view& v, const void* k, int64_t k_row, int64_t k_head,
                            const void* val, int64_t v_row, int64_t v_head, const lam_kv_slots& weights,
                            const lam_kv_slots& positions, const int32_t* first, uint32_t* status) {
  unsigned grid;
  LAM_TRY(row_grid(v, &grid));
  const KvArgs a = KvArgs::of(v);
  const RowArgs ka{k, k_row, k_head, wide_rows(k, k_row, k_head)}, va{val, v_row, v_head, wide_rows(val, v_row, v_head)};
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_append", &e0, &e1));
#define LAM_GO(D, BF)                                                                                              \
  hipExtLaunchKernelGGL((k_kv_append<D, BF>), dim3(grid), dim3(kKvThreads), 0, ctx->stream, e0, e1, 0, a, ka, va,   \
                        weights, positions, first, status)
  LAM_KV_DISPATCH(v, LAM_GO);
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

lam_status launch_kv_read(lam_ctx* ctx, const lam_kv_view& v, void* k, void* val) {
  unsigned grid;
  LAM_TRY(row_grid(v, &grid));
  const KvArgs a = KvArgs::of(v);
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_read", &e0, &e1));
#define LAM_GO(D, BF)                                                                                            \
  hipExtLaunchKernelGGL((k_kv_read<D, BF>), dim3(grid), dim3(kKvThreads), 0, ctx->stream, e0, e1, 0, a,           \
                        static_cast<uint4*>(k), static_cast<uint4*>(val))
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
  DevBuf& buf = ctx->scratch[kScratchKv];
  LAM_TRY(buf.ensure((size_t)pairs * (2 * (size_t)e.moves + 1) * 4));
  e.n_moves = buf.as<int32_t>();
  e.holes = e.n_moves + pairs;
  e.extras = e.holes + pairs * e.moves;
  hipEvent_t e0, e1;
  LAM_TRY(prof_launch_events(ctx, "kv_select", &e0, &e1));
  hipExtLaunchKernelGGL(k_kv_select, dim3((unsigned)pairs), dim3(kSelThreads), 0, ctx->stream, e0, e1, 0, a, e);
  LAM_HIP(hipGetLastError());
  LAM_TRY(prof_launch_events(ctx, "kv_move", &e0, &e1));
  const int per = kKvThreads / (v.head_dim / 8);
  const dim3 grid((unsigned)std::max(1, (e.moves + per - 1) / per), (unsigned)pairs);
#define LAM_GO(D, BF) \
  hipExtLaunchKernelGGL((k_kv_move<D>), grid, dim3(kKvThreads), 0, ctx->stream, e0, e1, 0, a, e)
  if (v.head_dim == 64) LAM_GO(64, 0); else if (v.head_dim == 128) LAM_GO(128, 0); else LAM_GO(256, 0);
#undef LAM_GO
  LAM_HIP(hipGetLastError());
  return LAM_OK;
}

}  // namespace lam
