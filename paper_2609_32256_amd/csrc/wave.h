// Wave-wide reductions by data-parallel primitive moves (DPP): lane moves that
// stay in the register file, where a butterfly of __shfl_xor steps goes
// through LDS and waits for each step.  The moves, on a 64-lane wave: swaps
// within quads (neighbours, then pairs), across the quads of each half row of
// 8 (row_half_mirror), across the halves of each row of 16 (row_mirror), then
// lane 15 of rows 0 and 2 into rows 1 and 3 (row_bcast:15), and lane 31 into
// rows 2 and 3 (row_bcast:31).  Each step combines disjoint partial results,
// so after it lane 63 holds the whole wave's; a lane that a move does not
// write gets the operation's identity.  Every lane of the wave must be active.
// Sums in binary64 are taken in this fixed order (different from a butterfly's,
// equally exact to within the usual bound for n terms).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace lam {

#define LAM_WAVE_DPP_STEPS(STEP) \
  STEP(0xb1, 0xf)                \
  STEP(0x4e, 0xf)                \
  STEP(0x141, 0xf)               \
  STEP(0x140, 0xf)               \
  STEP(0x142, 0xa)               \
  STEP(0x143, 0xc)

// move of a 32-bit lane value; `old` for lanes the move does not write
#define LAM_DPP_MOVE(old, v, ctrl, rmask) __builtin_amdgcn_update_dpp((int)(old), (int)(v), ctrl, rmask, 0xf, false)

__device__ __forceinline__ float wave_max_f32(float v) {
#define LAM_STEP(ctrl, rmask) v = fmaxf(v, __int_as_float(LAM_DPP_MOVE(__float_as_int(v), __float_as_int(v), ctrl, rmask)));
  LAM_WAVE_DPP_STEPS(LAM_STEP)
#undef LAM_STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#define LAM_STEP(ctrl, rmask) v = max(v, (uint32_t)LAM_DPP_MOVE(v, v, ctrl, rmask));
  LAM_WAVE_DPP_STEPS(LAM_STEP)
#undef LAM_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#define LAM_STEP(ctrl, rmask)                                                                     \
  {                                                                                               \
    const unsigned long long b = (unsigned long long)__double_as_longlong(v);                    \
    const uint32_t olo = (uint32_t)LAM_DPP_MOVE(0, (uint32_t)b, ctrl, rmask);                     \
    const uint32_t ohi = (uint32_t)LAM_DPP_MOVE(0, (uint32_t)(b >> 32), ctrl, rmask);             \
    v += __longlong_as_double((long long)(((unsigned long long)ohi << 32) | olo));                \
  }
  LAM_WAVE_DPP_STEPS(LAM_STEP)
#undef LAM_STEP
  const unsigned long long b = (unsigned long long)__double_as_longlong(v);
  const uint32_t rlo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63);
  const uint32_t rhi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
  return __longlong_as_double((long long)(((unsigned long long)rhi << 32) | rlo));
}

// Inclusive sums over the lanes of a wave, in lane order: within rows of 16 by
// shifts of 1, 2, 4 and 8 lanes (a lane past the row's edge gets 0), then the ends
// of rows 0 and 2 into rows 1 and 3, then lane 31's into rows 2 and 3.
__device__ __forceinline__ uint32_t wave_scan_u32(uint32_t v) {
  v += (uint32_t)LAM_DPP_MOVE(0, v, 0x111, 0xf);
  v += (uint32_t)LAM_DPP_MOVE(0, v, 0x112, 0xf);
  v += (uint32_t)LAM_DPP_MOVE(0, v, 0x114, 0xf);
  v += (uint32_t)LAM_DPP_MOVE(0, v, 0x118, 0xf);
  v += (uint32_t)LAM_DPP_MOVE(0, v, 0x142, 0xa);
  v += (uint32_t)LAM_DPP_MOVE(0, v, 0x143, 0xc);
  return v;
}

// The largest of each quad's four values, in all four lanes (which must be active together).
__device__ __forceinline__ uint32_t quad_max_u32(uint32_t v) {
  v = max(v, (uint32_t)LAM_DPP_MOVE(v, v, 0xb1, 0xf));
  return max(v, (uint32_t)LAM_DPP_MOVE(v, v, 0x4e, 0xf));
}

// Sums over groups of L consecutive lanes (8, 16 or 32), in all of them, by the same moves:
// the order is the same in every lane, so all get the same bits.
template <int L>
__device__ __forceinline__ float group_sum_f32(float v) {
  v += __int_as_float(LAM_DPP_MOVE(__float_as_int(v), __float_as_int(v), 0xb1, 0xf));
  v += __int_as_float(LAM_DPP_MOVE(__float_as_int(v), __float_as_int(v), 0x4e, 0xf));
  v += __int_as_float(LAM_DPP_MOVE(__float_as_int(v), __float_as_int(v), 0x141, 0xf));
  if constexpr (L >= 16) v += __int_as_float(LAM_DPP_MOVE(__float_as_int(v), __float_as_int(v), 0x140, 0xf));
  if constexpr (L >= 32) v += __shfl_xor(v, 16);
  return v;
}

template <int L>
__device__ __forceinline__ double group_sum_f64(double v) {
#define LAM_STEP(ctrl)                                                                                \
  {                                                                                                   \
    const unsigned long long b = (unsigned long long)__double_as_longlong(v);                         \
    const uint32_t lo = (uint32_t)LAM_DPP_MOVE((uint32_t)b, (uint32_t)b, ctrl, 0xf);                   \
    const uint32_t hi = (uint32_t)LAM_DPP_MOVE((uint32_t)(b >> 32), (uint32_t)(b >> 32), ctrl, 0xf);   \
    v += __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));                      \
  }
  LAM_STEP(0xb1)
  LAM_STEP(0x4e)
  LAM_STEP(0x141)
  if constexpr (L >= 16) LAM_STEP(0x140)
  if constexpr (L >= 32) v += __shfl_xor(v, 16);
#undef LAM_STEP
  return v;
}

#undef LAM_DPP_MOVE
#undef LAM_WAVE_DPP_STEPS

}  // namespace lam
