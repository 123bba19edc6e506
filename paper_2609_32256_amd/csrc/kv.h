// The paged 4-bit key/value cache as its kernels see it: where a token's codes
// and scales lie, which rows and lengths a sequence has, and the conversions
// between codes and 16-bit values.  Everything read from the caller's device
// arrays (table, lengths, starts) is held to the sizes the host knows before it
// becomes an address.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lam.h"

namespace lam {

constexpr int kKvBlock = 32;        // channels that share a scale
constexpr int kKvExpLo = -23;       // 0.5 * 2^-23 is the smallest float16
constexpr int kKvExpHi = 13;        // 6 * 2^13 = 49152 is below float16's largest
constexpr int kKvStrip = 32;        // tokens a wave takes at a time; pages are multiples of it

// Offsets within one head's part of a page of T tokens.
template <int D>
struct KvLayout {
  static constexpr int kRun = D / 16;               // channels of a value run
  static constexpr int kRunBytes = D / 32;          // its codes, per token
  static constexpr int kBlocks = D / kKvBlock;      // scales per token
  __host__ __device__ static int64_t head_bytes(int T) { return (int64_t)T * (D + D / 16); }
  __device__ static int k_codes(int t) { return t * (D / 2); }
  __device__ static int v_codes(int T, int t, int run) {
    return T * (D / 2) + (((t >> 2) * 16 + run) * 4 + (t & 3)) * kRunBytes;
  }
  __device__ static int k_scales(int T, int t) { return T * D + t * kBlocks; }
  __device__ static int v_scales(int T, int t, int block) {
    return T * D + T * kBlocks + ((t >> 2) * kBlocks + block) * 4 + (t & 3);
  }
};

// The caller's index arrays do not change while a kernel reads them: through the
// constant address space, entries that a whole wave shares are scalar loads.
typedef const int32_t __attribute__((address_space(4)))* kv_const_i32;
__device__ __forceinline__ kv_const_i32 kv_const(const int32_t* p) { return (kv_const_i32)(uintptr_t)p; }

struct KvArgs {
  uint8_t* pages;
  int64_t n_pages;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* lengths;
  const int32_t* starts;
  int64_t rows;
  int32_t n_seqs, table_cols, heads, page_shift;
  int32_t per_seq;   // rows of each sequence where starts is NULL

  static KvArgs of(const lam_kv_view& v) {
    KvArgs a{};
    a.pages = v.pages_dev;
    a.n_pages = v.n_pages;
    a.table = v.table_dev;
    a.table_stride = v.table_stride;
    a.lengths = v.lengths_dev;
    a.starts = v.starts_dev;
    a.rows = v.rows;
    a.n_seqs = v.n_seqs;
    a.table_cols = v.table_cols;
    a.heads = v.kv_heads;
    while ((1 << a.page_shift) < v.page_size) ++a.page_shift;
    a.per_seq = v.n_seqs > 0 ? (int32_t)(v.rows / v.n_seqs) : 0;
    return a;
  }

  // first row of sequence s, s <= n_seqs
  __device__ int64_t start(int s) const {
    if (!starts) return (int64_t)s * per_seq;
    const int64_t r = starts[s];
    return r < 0 ? 0 : (r > rows ? rows : r);
  }
  // Cached tokens of sequence s, whose last are the call's rows: those past the table's
  // columns count in.  (Room above for the rows past the last of a tile; a sequence
  // has at most 2^30 tokens with a place, so no causal limit among them is another.)
  __device__ int tokens(int s) const { return min(max(kv_const(lengths)[s], 0), 0x7fff0000); }
  // those that the table has columns for
  __device__ int length(int s) const { return (int)min((int64_t)tokens(s), (int64_t)table_cols << page_shift); }
  // page of column c of sequence s, or -1
  __device__ int64_t page(int s, int c) const {
    const int64_t p = table[s * table_stride + c];
    return p >= 0 && p < n_pages ? p : -1;
  }
  __device__ uint8_t* head_page(int64_t page, int h, int64_t head_bytes) const {
    return pages + (page * heads + h) * head_bytes;
  }
};

typedef _Float16 kv_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 kv_h8 __attribute__((ext_vector_type(8)));
typedef __bf16 kv_b2 __attribute__((ext_vector_type(2)));
typedef __bf16 kv_b8 __attribute__((ext_vector_type(8)));
typedef uint32_t kv_u4 __attribute__((ext_vector_type(4)));
typedef float kv_f4 __attribute__((ext_vector_type(4)));

// scale byte -> 2^e as a float32 (a byte of a block never written may be anything)
__device__ __forceinline__ float kv_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes 2 SEL and 2 SEL + 1 of a word as two 16-bit values, scaled: one
// conversion instruction of CDNA4.
template <bool BF16, int SEL>
__device__ __forceinline__ uint32_t kv_values(uint32_t word, float scale) {
  if constexpr (BF16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, SEL));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, SEL));
}

// The eight values of a word.
template <bool BF16>
__device__ __forceinline__ uint4 kv_values8(uint32_t word, float scale) {
  return uint4{kv_values<BF16, 0>(word, scale), kv_values<BF16, 1>(word, scale), kv_values<BF16, 2>(word, scale),
               kv_values<BF16, 3>(word, scale)};
}

// Calls LAUNCH with the head size and the type as constants.
#define LAM_KV_DISPATCH(v, LAUNCH)                                                          \
  do {                                                                                      \
    const bool bf_ = (v).dtype == LAM_BF16;                                                 \
    if ((v).head_dim == 64) { if (bf_) LAUNCH(64, true); else LAUNCH(64, false); }          \
    else if ((v).head_dim == 128) { if (bf_) LAUNCH(128, true); else LAUNCH(128, false); }  \
    else { if (bf_) LAUNCH(256, true); else LAUNCH(256, false); }                           \
  } while (0)

}  // namespace lam
