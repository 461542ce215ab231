// The cache in 4 bits: what a page holds, and the pieces that the packing, the unpacking and the attention kernels share.
//
// A row (one token's key or value, 128 numbers) has two groups of 64.  A group keeps its smallest number `low`, a scale
// s = bf16((largest - low) / 15) and a code c of 4 bits for every number x: the count of borders low + (k + 1/2) s, k = 0..14, below x
// (on a border: the lower code).  It stands for low + c s.
//
// Pages are made of units of 16 rows, 1152 bytes of keys and 1152 of values behind them (so that one copy fetches both): 1024 of codes in the order in which a warp's lanes feed them to m16n8k16 MMAs, then
// [16 rows][2 groups] pairs (s, low) of bf16.  A 32-bit word holds eight codes as four pairs: pair e in the bits 4 e .. 4 e + 3 of both
// halves.  As the bits of an fp16 number a code c by itself is c 2^-24, and c << 4 is c 2^-20 (numbers without a leading one, which the tensor
// cores take as exactly as others): two masks and a shift by 8 make four operand registers of a word.
//   keys:   word (row, t, j) at row * 64 + t * 16 + j * 4: the numbers 32 j + 8 t .. + 7 of the row, pair e = numbers 2 e, 2 e + 1
//           (lane (row, t) of the first MMA operand; the contraction runs over the numbers in any order that q shares)
//   values: word (h, lane, m) at h * 512 + lane * 16 + m * 4, lane = 4 g + t: numbers d = 64 h + 8 g + 2 m and d + 1 of four rows;
//           pair 0: d of the rows 2 t, 2 t + 1; pair 1: d + 1 of those; pairs 2, 3: the same of the rows 2 t + 8, 2 t + 9
#pragma once
#include "common.cuh"
#include "kernels.h"

namespace kve {

constexpr int Q4_CODE_BYTES = Q4_UNIT_ROWS * D / 2;      // of a unit: 1024
static_assert(Q4_UNIT_BYTES == Q4_CODE_BYTES + Q4_UNIT_ROWS * 2 * 4, "codes, then a scale and a lowest number for two groups of each row");

// the four pairs of a word as fp16 numbers: c 2^-24, c 2^-20, c 2^-24, c 2^-20
__device__ __forceinline__ void q4_spread(uint32_t w, uint32_t (&pair)[4]) {
  const uint32_t x = w >> 8;
  pair[0] = w & 0x000f000fu;
  pair[1] = w & 0x00f000f0u;
  pair[2] = x & 0x000f000fu;
  pair[3] = x & 0x00f000f0u;
}

// 4 x 4 bytes: byte m of w[i] becomes byte i of w[m]
__device__ __forceinline__ void transpose_bytes(uint32_t (&w)[4]) {
  const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[2], w[3], 0x5140);      // (w0.0 w1.0 w0.1 w1.1)
  const uint32_t c = __byte_perm(w[0], w[1], 0x7362), d = __byte_perm(w[2], w[3], 0x7362);
  w[0] = __byte_perm(a, b, 0x5410); w[1] = __byte_perm(a, b, 0x7632);
  w[2] = __byte_perm(c, d, 0x5410); w[3] = __byte_perm(c, d, 0x7632);
}

}  // namespace kve
