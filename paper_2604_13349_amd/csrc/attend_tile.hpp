// Operands and places in LDS of the bf16 kernels of many query rows (v_mfma_f32_32x32x16_bf16, lane l: row l % 32, elements 8 (l / 32) .. + 7 of 16).
#pragma once
#include "attend.hpp"

namespace obf {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t TilePiece;

union TileFrag { TilePiece u; bf16x8 v; s16x4 h[2]; uint32_t w[4]; };

// Places in a tile of rows of 2 D bytes.
template <int D> __device__ __forceinline__ int place_k(const int row, const int piece) {       // 16-byte pieces
  return row * 2 * D + ((piece ^ (D == 128 ? row & 15 : (row >> 1) & 7)) << 4);
}
template <int D> __device__ __forceinline__ int swap_v(const int row) { return D == 128 ? row & 3 : (row >> 1) & 1; }   // of 64-byte pieces

}  // namespace obf
