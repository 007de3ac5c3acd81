// The 4-bit form of a weight matrix [N, C] with groups of g columns (include/moehub.h, moe_w4_t): codes, 4 bits each, and a
// bf16 scale per group and row, stored [C / g, N] so that the scales of neighbouring rows are neighbours.
// A 32-bit word holds eight columns, the even ones in its low half: masking the word at bits 0-3 and 16-19 then gives
// columns 0 and 1 in the two halves of a register, which is how the tensor cores take pairs of bf16 numbers; shifted by
// 4, 8 and 12 the same mask gives columns 2 and 3, 4 and 5, 6 and 7.
#pragma once
#include "common.cuh"

namespace moehub {

__host__ __device__ constexpr int w4_shift(int column) { return 4 * (column % 2 * 4 + column / 2); }  // of a column's nibble in its word

__device__ __forceinline__ float w4_value(uint32_t word, int column) {
  return (float)((int)((word >> w4_shift(column)) & 15u) - 8);
}

// What the host checks of a matrix; returns MOE_OK or the error.
inline int w4_check(const moe_w4_t* w, int64_t experts, int64_t N, int64_t C, int group) {
  if (w == nullptr || w->codes == nullptr || w->scales == nullptr || experts <= 0 || N <= 0 || C <= 0) return MOE_ERR_ARG;
  if ((group != 32 && group != 64 && group != 128) || C > (1 << 25) || N > (1 << 30)) return MOE_ERR_UNSUPPORTED;
  if (C % group != 0) return MOE_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(w->codes) | reinterpret_cast<uintptr_t>(w->scales)) & 15) return MOE_ERR_ALIGN;
  return MOE_OK;
}

}  // namespace moehub
