// C entry points of the 4-bit key/value cache (include/lam.h): argument checks.
// The kernels are in kv_cache.hip, kv_rotate.hip, kv_attend.hip and kv_chunk.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kv_rotate.h"
#include "lam_internal.h"

using namespace lam;

namespace {

constexpr size_t kKvLeastScratch = 1 << 20;

bool sizes_ok(int32_t head_dim, int32_t page_size) {
  return (head_dim == 64 || head_dim == 128 || head_dim == 256) && page_size >= 32 && page_size <= 1024 &&
         (page_size & (page_size - 1)) == 0;
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

lam_status check_view(const lam_kv_view* v) {
  LAM_CHECK(v != nullptr, LAM_EINVAL, "view is NULL");
  LAM_CHECK(sizes_ok(v->head_dim, v->page_size), LAM_EINVAL,
            "head_dim must be 64, 128 or 256 and page_size a power of two from 32 to 1024 (got %d, %d)", v->head_dim,
            v->page_size);
  LAM_CHECK(v->kv_heads >= 1 && v->kv_heads <= 4096, LAM_EINVAL, "kv_heads must be in [1, 4096]");
  LAM_CHECK(v->n_seqs >= 0 && v->n_seqs <= (1 << 20), LAM_EINVAL, "n_seqs must be in [0, 2^20]");
  LAM_CHECK(v->rows >= 0 && v->rows < (1LL << 31), LAM_EINVAL, "rows must be in [0, 2^31)");
  LAM_CHECK(v->table_cols >= 0 && (int64_t)v->table_cols * v->page_size <= (1LL << 30), LAM_EINVAL,
            "table_cols * page_size must be in [0, 2^30]");   // (strips ahead of a length are still 32-bit numbers)
  LAM_CHECK(v->n_pages >= 0 && v->n_pages < (1LL << 31), LAM_EINVAL, "n_pages must be in [0, 2^31)");
  LAM_CHECK(v->dtype == LAM_F16 || v->dtype == LAM_BF16, LAM_EINVAL, "dtype %d is not LAM_F16 or LAM_BF16", v->dtype);
  LAM_CHECK(v->pages_dev != nullptr || v->n_pages == 0, LAM_EINVAL, "pages is NULL");
  LAM_CHECK(aligned(v->pages_dev, 16), LAM_EINVAL, "pages must be 16-byte aligned");
  if (v->n_seqs > 0) {
    LAM_CHECK(v->lengths_dev != nullptr && (v->table_dev != nullptr || v->table_cols == 0), LAM_EINVAL,
              "lengths or table is NULL");
    LAM_CHECK(v->table_stride >= v->table_cols || v->n_seqs == 1, LAM_EINVAL, "table_stride is below table_cols");
  }
  LAM_CHECK(aligned(v->lengths_dev, 4) && aligned(v->table_dev, 4) && aligned(v->starts_dev, 4), LAM_EINVAL,
            "table, lengths and starts must be 4-byte aligned");
  return LAM_OK;
}

// the rows of calls that have some
lam_status check_rows(const lam_kv_view* v) {
  if (v->rows == 0) return LAM_OK;
  LAM_CHECK(v->n_seqs > 0, LAM_EINVAL, "rows without sequences");
  LAM_CHECK(v->starts_dev != nullptr || v->rows % v->n_seqs == 0, LAM_EINVAL,
            "without starts every sequence has the same number of rows (%lld rows, %d sequences)", (long long)v->rows,
            v->n_seqs);
  return LAM_OK;
}

lam_status check_slots(const lam_kv_slots* s, const char* name, uintptr_t align) {
  if (s == nullptr || s->p_dev == nullptr) return LAM_OK;
  LAM_CHECK(s->cols >= 0 && s->seq_stride >= 0 && s->head_stride >= 0, LAM_EINVAL, "%s has a negative size or stride",
            name);
  LAM_CHECK(aligned(s->p_dev, align), LAM_EINVAL, "%s must be %d-byte aligned", name, (int)align);
  return LAM_OK;
}

lam_kv_slots or_none(const lam_kv_slots* s) { return s ? *s : lam_kv_slots{nullptr, 0, 0, 0}; }

// slots that a call writes: one of its own for each sequence and head
lam_status check_own(const lam_kv_slots& s, const lam_kv_view* v, const char* name) {
  if (s.p_dev == nullptr) return LAM_OK;
  const int64_t n = v->n_seqs, heads = v->kv_heads, cols = s.cols, seq = s.seq_stride, head = s.head_stride;
  LAM_CHECK(head >= cols || heads == 1, LAM_EINVAL, "%s: heads overlap", name);
  LAM_CHECK(seq >= cols || n <= 1, LAM_EINVAL, "%s: sequences overlap", name);
  if (n <= 1 || heads == 1 || cols == 0) return LAM_OK;
  // heads within a sequence, as they lie mostly; else a head's slots are compared with those of
  // the sequences that begin next to them
  if (seq / heads >= head) return LAM_OK;
  for (int64_t h = 1; h < heads; ++h) {
    const int64_t at = h * head, q = at / seq;
    LAM_CHECK(!(q < n && at - q * seq < cols) && !(q + 1 < n && (q + 1) * seq - at < cols), LAM_EINVAL,
              "%s: heads of one sequence overlap those of another", name);
  }
  return LAM_OK;
}

// heads of rows as a strided array, for the question whether two of them share memory
struct Strided {
  const void* p;
  int64_t row, head, rows, heads, dim;
  uintptr_t begin() const { return reinterpret_cast<uintptr_t>(p); }
  int64_t span() const { return (heads - 1) * head + dim; }   // elements of a row, first to last
  uintptr_t end() const { return begin() + 2 * ((rows - 1) * row + span()); }
};

bool apart(const Strided& a, const Strided& b) {
  if (a.end() <= b.begin() || b.end() <= a.begin()) return true;
  // rows of the same stride, a's and b's in turn (parts of one product's result)
  if (a.row != b.row || a.span() > a.row || b.span() > b.row) return false;
  const int64_t step = 2 * a.row;
  int64_t off = (int64_t)(b.begin() - a.begin()) % step;
  if (off < 0) off += step;
  return off >= 2 * a.span() && off + 2 * b.span() <= step;
}

Strided in_of(const lam_heads& h, int64_t rows, int32_t dim) { return {h.x_dev, h.row_stride, h.head_stride, rows, h.heads, dim}; }
Strided out_of(const lam_heads& h, int64_t rows, int32_t dim) { return {h.y_dev, h.y_row_stride, h.y_head_stride, rows, h.heads, dim}; }

lam_status check_rotary(const lam_rotary* r, int32_t dim) {
  LAM_CHECK(r != nullptr, LAM_EINVAL, "rotary is NULL");
  LAM_CHECK(r->pairs >= 0 && 2 * (int64_t)r->pairs <= dim, LAM_EINVAL, "rotary pairs (%d) must be in [0, head_dim / 2]",
            r->pairs);
  LAM_CHECK(r->layout == LAM_ROTARY_HALF || r->layout == LAM_ROTARY_INTERLEAVED, LAM_EINVAL, "unknown rotary layout %d",
            r->layout);
  LAM_CHECK(r->pairs == 0 || r->freq_dev != nullptr, LAM_EINVAL, "rotary frequencies are NULL");
  LAM_CHECK(aligned(r->freq_dev, 8), LAM_EINVAL, "rotary frequencies must be 8-byte aligned");
  LAM_CHECK(std::isfinite(r->amplitude) && std::isfinite((float)r->amplitude), LAM_EINVAL, "amplitude must be finite");
  return LAM_OK;
}

lam_status check_heads(const lam_heads& h, const char* name, int64_t rows, int32_t dim, int32_t dtype, bool out) {
  LAM_CHECK(h.heads >= 0 && h.heads <= (1 << 20), LAM_EINVAL, "%s: heads must be in [0, 2^20]", name);
  LAM_CHECK(h.gain_dev == nullptr || h.gain_dtype == LAM_F32 || h.gain_dtype == dtype, LAM_EINVAL,
            "%s: gains must be LAM_F32 or of the rows' type", name);
  LAM_CHECK(aligned(h.gain_dev, h.gain_dtype == LAM_F32 ? 4 : 2), LAM_EINVAL, "%s: gains are not aligned", name);
  if (h.heads == 0 || rows == 0) return LAM_OK;
  LAM_CHECK(h.x_dev != nullptr, LAM_EINVAL, "%s is NULL", name);
  LAM_CHECK(aligned(h.x_dev, 2), LAM_EINVAL, "%s must be 2-byte aligned", name);
  LAM_CHECK(h.row_stride >= 0 && h.head_stride >= 0, LAM_EINVAL, "%s: strides must be >= 0", name);
  if (!out) return LAM_OK;
  LAM_CHECK(h.y_dev != nullptr, LAM_EINVAL, "%s: the result is NULL", name);
  LAM_CHECK(aligned(h.y_dev, 2), LAM_EINVAL, "%s: the result must be 2-byte aligned", name);
  const int64_t row = h.y_row_stride, head = h.y_head_stride;
  LAM_CHECK(row >= 0 && head >= 0, LAM_EINVAL, "%s: the result's strides must be >= 0", name);
  const bool by_row = (head >= dim || h.heads == 1) && (row >= (h.heads - 1) * head + dim || rows == 1);
  const bool by_head = (row >= dim || rows == 1) && (head >= (rows - 1) * row + dim || h.heads == 1);
  LAM_CHECK(by_row || by_head, LAM_EINVAL, "%s: rows or heads of the result overlap", name);
  const bool same = h.x_dev == h.y_dev && (row == h.row_stride || rows == 1) && (head == h.head_stride || h.heads == 1);
  LAM_CHECK(same || apart(in_of(h, rows, dim), out_of(h, rows, dim)), LAM_EINVAL,
            "%s: the result overlaps the rows in part (it may be the rows themselves)", name);
  return LAM_OK;
}

lam_status check_norm(double eps, int32_t norm_dim, int32_t dim) {
  LAM_CHECK(std::isfinite(eps) && eps > 0.0, LAM_EINVAL, "eps must be finite and above 0");
  LAM_CHECK(norm_dim >= 0 && norm_dim <= dim, LAM_EINVAL, "norm_dim must be in [0, head_dim], 0 for head_dim");
  return LAM_OK;
}

bool wide(const void* p, int64_t row, int64_t head) { return aligned(p, 16) && row % 8 == 0 && head % 8 == 0; }

RotateHeads heads_of(const lam_heads& h) {
  RotateHeads r{};
  r.x = static_cast<const uint16_t*>(h.x_dev);
  r.x_row = h.row_stride;
  r.x_head = h.head_stride;
  r.y = static_cast<uint16_t*>(h.y_dev);
  r.y_row = h.y_row_stride;
  r.y_head = h.y_head_stride;
  r.gain = h.gain_dev;
  r.gain_f32 = h.gain_dtype == LAM_F32;
  r.heads = h.heads;
  r.x_wide = wide(h.x_dev, h.row_stride, h.head_stride);
  r.y_wide = wide(h.y_dev, h.y_row_stride, h.y_head_stride);
  r.gain_wide = aligned(h.gain_dev, 16);
  return r;
}

RotateArgs rotate_args(const lam_rotary& r, const lam_heads& q, const lam_heads& k, int64_t rows, int32_t dim,
                       double eps, int32_t norm_dim) {
  RotateArgs a{};
  a.h[0] = heads_of(q);
  a.h[1] = heads_of(k);
  a.freq = r.freq_dev;
  a.pairs = r.pairs;
  a.interleaved = r.layout == LAM_ROTARY_INTERLEAVED;
  a.amplitude = (float)r.amplitude;
  a.amplitude64 = r.amplitude;
  a.eps = eps;
  a.inv_dim = 1.0 / (norm_dim ? norm_dim : dim);
  a.rows = rows;
  a.dim = dim;
  return a;
}

}  // namespace

namespace lam {

lam_status kv_scratch(lam_ctx* ctx, size_t need, void** out) {
  DevBuf& b = ctx->scratch[kScratchKv];
  if (need > b.bytes || b.p == nullptr) {
    DevBuf grown;
    LAM_TRY(grown.ensure(std::max({need, 2 * b.bytes, kKvLeastScratch})));
    if (b.p) {
      DevBuf* const end = ctx->kv_old + kKvOld;
      DevBuf* const slot = std::find_if(ctx->kv_old, end, [](const DevBuf& o) { return o.p == nullptr; });
      if (slot == end) grown.release();
      LAM_CHECK(slot != end, LAM_ENOMEM, "the context's scratch has grown too often");   // (31 doublings)
      *slot = b;
    }
    b = grown;
  }
  *out = b.p;
  return LAM_OK;
}

}  // namespace lam

extern "C" {

int64_t lam_kv_page_bytes(int32_t head_dim, int32_t page_size) {
  return sizes_ok(head_dim, page_size) ? (int64_t)page_size * (head_dim + head_dim / 16) : -1;
}

lam_status lam_kv_append(lam_ctx* ctx, const lam_kv_view* view, const void* k_dev, int64_t k_row_stride,
                         int64_t k_head_stride, const void* v_dev, int64_t v_row_stride, int64_t v_head_stride,
                         const lam_kv_slots* weights, const lam_kv_slots* positions, const int32_t* first_dev,
                         uint32_t* status_dev) {
  LAM_CHECK(ctx != nullptr, LAM_EINVAL, "ctx is NULL");
  LAM_TRY(check_view(view));
  LAM_TRY(check_rows(view));
  LAM_TRY(check_slots(weights, "weights", 4));
  LAM_TRY(check_slots(positions, "positions", 4));
  const lam_kv_slots w = or_none(weights), p = or_none(positions);
  LAM_TRY(check_own(w, view, "weights"));
  LAM_TRY(check_own(p, view, "positions"));
  LAM_CHECK(p.p_dev == nullptr || first_dev != nullptr || view->n_seqs == 0, LAM_EINVAL, "positions need first");
  LAM_CHECK(aligned(first_dev, 4) && aligned(status_dev, 4), LAM_EINVAL, "first and status must be 4-byte aligned");
  if (view->rows == 0) return LAM_OK;
  LAM_CHECK(k_dev != nullptr && v_dev != nullptr, LAM_EINVAL, "k or v is NULL");
  LAM_CHECK(aligned(k_dev, 2) && aligned(v_dev, 2), LAM_EINVAL, "k and v must be 2-byte aligned");
  LAM_CHECK(k_row_stride >= 0 && k_head_stride >= 0 && v_row_stride >= 0 && v_head_stride >= 0, LAM_EINVAL,
            "strides must be >= 0");
  DeviceGuard g(ctx->device);
  return launch_kv_append(ctx, *view, k_dev, k_row_stride, k_head_stride, v_dev, v_row_stride, v_head_stride, w, p,
                          first_dev, status_dev);
}

lam_status lam_rotary_frequencies(int32_t pairs, double base, int scaling, double factor, double length, double low,
                                  double high, double* freq, double* amplitude) {
  LAM_CHECK(pairs >= 0 && pairs <= (1 << 20), LAM_EINVAL, "pairs must be in [0, 2^20]");
  LAM_CHECK(std::isfinite(base) && base > 0.0, LAM_EINVAL, "base must be finite and above 0");
  LAM_CHECK(scaling >= LAM_ROTARY_PLAIN && scaling <= LAM_ROTARY_PARTS, LAM_EINVAL, "unknown rotary scaling %d", scaling);
  LAM_CHECK(freq != nullptr || pairs == 0, LAM_EINVAL, "freq is NULL");
  if (scaling != LAM_ROTARY_PLAIN)
    LAM_CHECK(std::isfinite(factor) && factor >= 1.0, LAM_EINVAL, "factor must be finite and at least 1");
  LAM_CHECK(scaling != LAM_ROTARY_BASE || pairs != 1, LAM_EINVAL, "a base for a longer context needs two pairs");
  if (scaling == LAM_ROTARY_PARTS)
    LAM_CHECK(std::isfinite(length) && length > 0.0 && std::isfinite(low) && std::isfinite(high) && low < high, LAM_EINVAL,
              "length must be above 0 and low below high");
  const long double two_pi = 6.283185307179586476925286766559L;
  const long double dim = 2.0L * pairs;
  long double b = base;
  if (scaling == LAM_ROTARY_BASE && pairs > 1) b *= powl(factor, dim / (dim - 2.0L));
  for (int32_t i = 0; i < pairs; ++i) {
    long double f = powl(b, -2.0L * i / dim);
    if (scaling == LAM_ROTARY_LINEAR) f /= factor;
    if (scaling == LAM_ROTARY_PARTS) {
      const long double turns = length * f / two_pi;
      const long double keep = std::min(1.0L, std::max(0.0L, (turns - low) / ((long double)high - low)));
      f = f / factor * (1.0L - keep) + f * keep;
    }
    freq[i] = (double)f;
  }
  if (amplitude) *amplitude = scaling == LAM_ROTARY_PARTS ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return LAM_OK;
}

lam_status lam_kv_rotate(lam_ctx* ctx, const lam_rotary* rotary, const lam_heads* q, const lam_heads* k, int64_t rows,
                         int32_t head_dim, int32_t dtype, const int32_t* positions_dev, double eps, int32_t norm_dim) {
  LAM_CHECK(ctx != nullptr, LAM_EINVAL, "ctx is NULL");
  LAM_CHECK(q != nullptr, LAM_EINVAL, "q is NULL");
  LAM_CHECK(head_dim >= 8 && head_dim <= 256 && head_dim % 8 == 0, LAM_EINVAL,
            "head_dim must be a multiple of 8 from 8 to 256 (got %d)", head_dim);
  LAM_CHECK(dtype == LAM_F16 || dtype == LAM_BF16, LAM_EINVAL, "dtype %d is not LAM_F16 or LAM_BF16", dtype);
  LAM_CHECK(rows >= 0 && rows < (1LL << 31), LAM_EINVAL, "rows must be in [0, 2^31)");
  LAM_TRY(check_rotary(rotary, head_dim));
  LAM_TRY(check_norm(eps, norm_dim, head_dim));
  const lam_heads none{};
  const lam_heads& kh = k ? *k : none;
  LAM_TRY(check_heads(*q, "q", rows, head_dim, dtype, true));
  LAM_TRY(check_heads(kh, "k", rows, head_dim, dtype, true));
  if (rows == 0 || (q->heads == 0 && kh.heads == 0)) return LAM_OK;
  if (q->heads > 0 && kh.heads > 0) {
    const Strided qx = in_of(*q, rows, head_dim), qy = out_of(*q, rows, head_dim);
    const Strided kx = in_of(kh, rows, head_dim), ky = out_of(kh, rows, head_dim);
    LAM_CHECK(apart(qy, kx) && apart(ky, qx) && apart(qy, ky), LAM_EINVAL,
              "a result overlaps the other's rows or result");
  }
  LAM_CHECK(rotary->pairs == 0 || positions_dev != nullptr, LAM_EINVAL, "positions is NULL");
  LAM_CHECK(aligned(positions_dev, 4), LAM_EINVAL, "positions must be 4-byte aligned");
  RotateArgs a = rotate_args(*rotary, *q, kh, rows, head_dim, eps, norm_dim);
  a.positions = positions_dev;
  DeviceGuard g(ctx->device);
  return launch_kv_rotate(ctx, a, dtype);
}

lam_status lam_kv_rotate_append(lam_ctx* ctx, const lam_kv_view* view, const lam_rotary* rotary, const lam_heads* q,
                                const lam_heads* k, const void* v_dev, int64_t v_row_stride, int64_t v_head_stride,
                                const lam_kv_slots* weights, const lam_kv_slots* positions, const int32_t* first_dev,
                                double eps, int32_t norm_dim, uint32_t* status_dev) {
  LAM_CHECK(ctx != nullptr, LAM_EINVAL, "ctx is NULL");
  LAM_TRY(check_view(view));
  LAM_TRY(check_rows(view));
  LAM_TRY(check_rotary(rotary, view->head_dim));
  LAM_TRY(check_norm(eps, norm_dim, view->head_dim));
  LAM_TRY(check_slots(weights, "weights", 4));
  LAM_TRY(check_slots(positions, "positions", 4));
  const lam_kv_slots w = or_none(weights), p = or_none(positions);
  LAM_TRY(check_own(w, view, "weights"));
  LAM_TRY(check_own(p, view, "positions"));
  LAM_CHECK(k != nullptr && k->heads == view->kv_heads, LAM_EINVAL, "k must have the view's heads");
  const lam_heads none{};
  const lam_heads& qh = q ? *q : none;
  LAM_TRY(check_heads(qh, "q", view->rows, view->head_dim, view->dtype, true));
  LAM_TRY(check_heads(*k, "k", view->rows, view->head_dim, view->dtype, false));
  if (view->rows > 0) {
    LAM_CHECK(v_dev != nullptr && aligned(v_dev, 2), LAM_EINVAL, "v must be 2-byte aligned and not NULL");
    LAM_CHECK(v_row_stride >= 0 && v_head_stride >= 0, LAM_EINVAL, "strides must be >= 0");
    if (qh.heads > 0) {
      const Strided y = out_of(qh, view->rows, view->head_dim);
      const Strided v{v_dev, v_row_stride, v_head_stride, view->rows, view->kv_heads, view->head_dim};
      LAM_CHECK(apart(y, in_of(*k, view->rows, view->head_dim)) && apart(y, v), LAM_EINVAL,
                "the queries' result overlaps k or v");
    }
  }
  LAM_CHECK(aligned(first_dev, 4) && aligned(status_dev, 4), LAM_EINVAL, "first and status must be 4-byte aligned");
  if (view->rows == 0) return LAM_OK;
  DeviceGuard g(ctx->device);
  return launch_kv_rotate_append(ctx, *view, rotate_args(*rotary, qh, *k, view->rows, view->head_dim, eps, norm_dim), v_dev,
                                 v_row_stride, v_head_stride, w, p, first_dev, status_dev);
}

lam_status lam_kv_read(lam_ctx* ctx, const lam_kv_view* view, void* k_dev, void* v_dev) {
  LAM_CHECK(ctx != nullptr, LAM_EINVAL, "ctx is NULL");
  LAM_TRY(check_view(view));
  LAM_TRY(check_rows(view));
  if (view->rows == 0) return LAM_OK;
  LAM_CHECK(k_dev != nullptr && v_dev != nullptr, LAM_EINVAL, "k or v is NULL");
  LAM_CHECK(aligned(k_dev, 16) && aligned(v_dev, 16), LAM_EINVAL, "k and v must be 16-byte aligned");
  DeviceGuard g(ctx->device);
  return launch_kv_read(ctx, *view, k_dev, v_dev);
}

lam_status lam_kv_attend(lam_ctx* ctx, const lam_kv_view* view, const void* q_dev, int64_t q_row_stride,
                         int64_t q_head_stride, int32_t q_heads, double scale, int causal, int64_t max_length,
                         const lam_kv_slots* mask, const lam_kv_slots* weights, void* out_dev, float* lse_dev) {
  return lam_kv_attend_window(ctx, view, q_dev, q_row_stride, q_head_stride, q_heads, scale, causal, max_length, 0, 0, mask,
                              weights, out_dev, lse_dev);
}

lam_status lam_kv_attend_window(lam_ctx* ctx, const lam_kv_view* view, const void* q_dev, int64_t q_row_stride,
                                int64_t q_head_stride, int32_t q_heads, double scale, int causal, int64_t max_length,
                                int64_t window, int64_t sinks, const lam_kv_slots* mask, const lam_kv_slots* weights,
                                void* out_dev, float* lse_dev) {
  LAM_CHECK(ctx != nullptr, LAM_EINVAL, "ctx is NULL");
  LAM_CHECK(window >= 0 && sinks >= 0, LAM_EINVAL, "window and sinks must be >= 0");
  LAM_CHECK(window > 0 || sinks == 0, LAM_EINVAL, "sinks without a window");
  LAM_TRY(check_view(view));
  LAM_TRY(check_rows(view));
  LAM_TRY(check_slots(mask, "mask", 1));
  LAM_TRY(check_slots(weights, "weights", 4));
  const lam_kv_slots m = or_none(mask), w = or_none(weights);
  LAM_TRY(check_own(w, view, "weights"));
  LAM_CHECK(q_heads >= 1 && q_heads % view->kv_heads == 0 && q_heads / view->kv_heads <= 1024, LAM_EINVAL,
            "q_heads (%d) must be a multiple of kv_heads (%d), at most 1024 of it", q_heads, view->kv_heads);
  LAM_CHECK(std::isfinite(scale) && std::isfinite((float)scale), LAM_EINVAL, "scale must be finite");
  LAM_CHECK(view->rows * (q_heads / view->kv_heads) < (1LL << 31), LAM_EINVAL, "too many query rows");
  if (view->rows == 0) return LAM_OK;
  LAM_CHECK(q_dev != nullptr && out_dev != nullptr, LAM_EINVAL, "q or out is NULL");
  LAM_CHECK(aligned(q_dev, 2) && aligned(out_dev, 16) && aligned(lse_dev, 4), LAM_EINVAL,
            "q must be 2-byte, out 16-byte and lse 4-byte aligned");
  LAM_CHECK(q_row_stride >= 0 && q_head_stride >= 0, LAM_EINVAL, "strides must be >= 0");
  // a workgroup reads its queries before it writes their results, in the same places where out is q
  const int64_t row = (int64_t)q_heads * view->head_dim;
  const uintptr_t q0 = reinterpret_cast<uintptr_t>(q_dev), o0 = reinterpret_cast<uintptr_t>(out_dev);
  const uintptr_t q1 = q0 + 2 * ((view->rows - 1) * q_row_stride + (q_heads - 1) * q_head_stride + view->head_dim);
  const bool apart = q1 <= o0 || o0 + 2 * view->rows * row <= q0;
  const bool same = q0 == o0 && (q_row_stride == row || view->rows == 1) && (q_head_stride == view->head_dim || q_heads == 1);
  LAM_CHECK(apart || same, LAM_EINVAL, "out overlaps q (it may be q itself, where that is contiguous)");
  DeviceGuard g(ctx->device);
  return launch_kv_attend(ctx, *view, q_dev, q_row_stride, q_head_stride, q_heads, (float)scale, causal != 0,
                          max_length, window, sinks, m, w, out_dev, lse_dev);
}

lam_status lam_kv_evict(lam_ctx* ctx, const lam_kv_view* view, const lam_kv_slots* scores,
                        const lam_kv_slots* positions, int32_t budget, int32_t recent, int32_t sinks,
                        int32_t* kept_dev, const lam_kv_slots* scores_out, const lam_kv_slots* positions_out,
                        int32_t* lengths_out_dev) {
  LAM_CHECK(ctx != nullptr, LAM_EINVAL, "ctx is NULL");
  LAM_TRY(check_view(view));
  LAM_CHECK(budget >= 1, LAM_EINVAL, "budget must be >= 1");
  LAM_CHECK(recent >= 0 && sinks >= 0 && (int64_t)recent + sinks <= budget, LAM_EINVAL,
            "recent and sinks must be >= 0 and together at most budget");
  LAM_TRY(check_slots(scores, "scores", 4));
  LAM_TRY(check_slots(positions, "positions", 4));
  LAM_TRY(check_slots(scores_out, "scores_out", 4));
  LAM_TRY(check_slots(positions_out, "positions_out", 4));
  const lam_kv_slots s = or_none(scores), p = or_none(positions), so = or_none(scores_out), po = or_none(positions_out);
  LAM_TRY(check_own(so, view, "scores_out"));
  LAM_TRY(check_own(po, view, "positions_out"));
  if (view->n_seqs == 0) return LAM_OK;
  LAM_CHECK(s.p_dev != nullptr && so.p_dev != nullptr && kept_dev != nullptr && lengths_out_dev != nullptr, LAM_EINVAL,
            "scores, scores_out, kept or lengths_out is NULL");
  LAM_CHECK(so.cols >= budget && (po.p_dev == nullptr || po.cols >= budget), LAM_EINVAL,
            "scores_out and positions_out need at least budget columns");
  LAM_CHECK(aligned(kept_dev, 4) && aligned(lengths_out_dev, 4), LAM_EINVAL,
            "kept and lengths_out must be 4-byte aligned");
  DeviceGuard g(ctx->device);
  return launch_kv_evict(ctx, *view, s, p, budget, recent, sinks, kept_dev, so, po, lengths_out_dev);
}

}  // extern "C"
