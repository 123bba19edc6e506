// C entry points of the 4-bit key/value cache (include/lam.h): argument checks.
// The kernels are in kv_cache.hip and kv_attend.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

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
  LAM_CHECK(ctx != nullptr, LAM_EINVAL, "ctx is NULL");
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
                          max_length, m, w, out_dev, lse_dev);
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
